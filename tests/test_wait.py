"""Bounded waits of the product kernels, compiled from the header that the kernels use and run against a simulated ring of stages (no GPU needed)."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2402_01798_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "tq_wait.h"

// wait LIMIT DONE_AT EVERY DEAD_AT: polls until DONE_AT, a stage filled every EVERY polls (0: never), another thread gives up at DEAD_AT (0: never)
static int wait_case(char** v) {
    const unsigned long limit = strtoul(v[0], 0, 0), done_at = strtoul(v[1], 0, 0), every = strtoul(v[2], 0, 0), dead_at = strtoul(v[3], 0, 0);
    unsigned long polls = 0;
    const bool ok = tq::wait_with_progress(limit, [&] { return ++polls == done_at; }, [&] { return dead_at && polls >= dead_at; },
                                           [&] { return static_cast<uint32_t>(every ? polls / every : 7); });
    std::printf("%d %lu\n", ok, polls);
    return 0;
}

// A ring whose stage `s` completes phase after phase.  Fillings 0 .. issued - 1 have been asked for, the first `landed` have landed and been read.
static int ring_case() {
    for (uint32_t stages = 1; stages <= 8; ++stages)
        for (uint32_t issued = 0; issued < 5 * stages; ++issued)
            for (uint32_t landed = issued > stages ? issued - stages : 0; landed <= issued; ++landed) {
                bool waited[64] = {};
                uint32_t completed[8] = {};                        // phases of each stage that are over
                for (uint32_t j = 0; j < landed; ++j) ++completed[j % stages];
                tq::for_outstanding(issued, stages, [&](uint32_t s, uint32_t parity) {
                    // the filling that this parity stands for: an over one if the stage's current phase has the other parity, else the current one
                    const uint32_t phase = (completed[s] & 1) != parity ? completed[s] - 1 : completed[s], j = phase * stages + s;
                    if (j >= issued) { std::printf("waits for a filling that nobody asked for\n"); std::exit(1); }
                    waited[j] = true;
                });
                for (uint32_t j = landed; j < issued; ++j)
                    if (!waited[j]) { std::printf("stages %u issued %u: filling %u not waited for\n", stages, issued, j); return 1; }
            }
    return 0;
}

// A pair: the barrier's phase ends when its one arrival (the first block's) and all expected bytes have come; one unit of bytes from each block.
static int pair_case() {
    for (uint32_t stages = 1; stages <= 6; ++stages)
        for (uint32_t read = 0; read < 3 * stages; ++read)          // fillings that both have asked for and that have been read
            for (uint32_t n0 = read; n0 <= read + stages; ++n0)
                for (uint32_t n1 = read; n1 <= read + stages; ++n1) {
                    struct Bar { uint32_t phase; int pending, tx; } bar[6];
                    bool settled[64] = {};
                    for (uint32_t s = 0; s < stages; ++s) bar[s] = Bar{0, 1, 0};
                    const auto over = [&](Bar& b) { if (b.pending == 0 && b.tx == 0) { ++b.phase; b.pending = 1; } };
                    const auto first = [&](uint32_t j) { Bar& b = bar[j % stages]; b.tx += 2; b.pending -= 1; b.tx -= 1; over(b); };
                    const auto second = [&](uint32_t j) { Bar& b = bar[j % stages]; b.tx -= 1; over(b); };
                    for (uint32_t j = 0; j < read; ++j) { first(j); second(j); }
                    for (uint32_t j = read; j < n1; ++j) second(j);   // the second's bytes may come before they are expected
                    for (uint32_t j = read; j < n0; ++j) first(j);
                    tq::for_outstanding_of_pair(n0, n1, stages, [&](uint32_t s, uint32_t parity, uint32_t by) {
                        Bar& b = bar[s];
                        if (by == 1) { b.tx -= 1; over(b); }                       // as if the second's had come
                        if (by == 2) { b.tx += 1; b.pending -= 1; over(b); }
                        if (by != 1 && by != 2 && by != 3) { std::printf("by %u\n", by); std::exit(1); }
                        if ((b.phase & 1) == parity) { std::printf("stages %u read %u n0 %u n1 %u: stage %u never ends\n", stages, read, n0, n1, s); std::exit(1); }
                        settled[s] = true;
                    });
                    for (uint32_t j = read; j < n0 || j < n1; ++j)
                        if (!settled[j % stages]) { std::printf("filling %u left\n", j); return 1; }
                    for (uint32_t s = 0; s < stages; ++s)
                        if (bar[s].tx != 0 || bar[s].pending != 1) { std::printf("stage %u: bytes left\n", s); return 1; }
                }
    return 0;
}

int main(int n, char** v) {
    if (n == 6 && !std::strcmp(v[1], "wait")) return wait_case(v + 2);
    if (n == 2 && !std::strcmp(v[1], "ring")) return ring_case();
    if (n == 2 && !std::strcmp(v[1], "pair")) return pair_case();
    return 2;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("wait")
    (where / "wait.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(where / "wait.cpp"), "-o", str(where / "wait")], check=True)

    def run(*args):
        return subprocess.run([str(where / "wait"), *map(str, args)], capture_output=True, text=True, timeout=120)
    return run


def wait(program, *args):
    ok, polls = map(int, program("wait", *args).stdout.split())
    return bool(ok), polls


def test_a_long_sum_has_its_time(program):
    """Many times the limit, while stages are filled: with 2^22 polls in all, a sum of 2^31 products gave up before its end."""
    assert wait(program, 5000, 1_000_000, 300, 0) == (True, 1_000_000)
    assert wait(program, 5000, 1_000_000, 4000, 0) == (True, 1_000_000)


def test_it_ends_without_progress(program):
    ok, polls = wait(program, 5000, 0, 0, 0)
    assert not ok and 5000 <= polls <= 5000 + 256 + 1              # the first look counts as one
    assert wait(program, 5000, 4999, 0, 0) == (True, 4999)
    ok, polls = wait(program, 5000, 0, 100_000, 0)                  # too slow
    assert not ok and polls <= 5000 + 256 + 1
    assert wait(program, 5000, 1, 0, 1) == (True, 1)                # what is done is done


def test_it_ends_when_another_thread_gave_up(program):
    ok, polls = wait(program, 1 << 22, 0, 300, 1000)
    assert not ok and 1000 <= polls < 1000 + 256


def test_every_filling_on_its_way_is_waited_for(program):
    r = program("ring")
    assert r.returncode == 0, r.stdout


def test_every_filling_of_a_pair_ends(program):
    r = program("pair")
    assert r.returncode == 0, r.stdout


def test_kernels_settle_before_memory_is_reused():
    """In each product kernel: after the roles have met and before the cluster's sums come into the stages, tensor memory is freed or the block ends."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tq_mx_product.cu")).read())
    bodies = {m.group(1): text[m.end():text.index("\n}\n", m.end())] for m in re.finditer(r"__global__[^;{]*?(mx_\w+_kernel)\(", text)}
    assert set(bodies) == {"mx_pair_kernel", "mx_split_kernel", "mx_token_kernel"}
    for name in ("mx_split_kernel", "mx_token_kernel"):
        b = bodies[name]
        assert "for_outstanding(issued, stages," in b
        assert re.search(r"__syncthreads\(\);\s*settle\(\);\s*cluster_sync\(\);", b), name
        assert re.search(r"__syncthreads\(\);\s*if constexpr \(SPLIT == 1\) settle\(\);.*tmem_free", b, re.S), name
        assert b.index("tell_block(&failed") > b.index("cluster_sync()"), name
    pair = bodies["mx_pair_kernel"]
    assert re.search(r"tell_block\(&ended.*cluster_sync\(\);.*for_outstanding_of_pair.*cluster_sync\(\);.*tmem_free", pair, re.S)
