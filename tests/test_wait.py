"""Bounded waits of the product kernels, compiled from the header that the kernels use and run on the CPU."""
import os
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

int main(int n, char** v) {
    if (n == 6 && !std::strcmp(v[1], "wait")) return wait_case(v + 2);
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
