"""Microscaled 4-bit operators without a GPU: sizes, refusals (found before any CUDA call is made), and the 64-bit reference that
the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import mx_reference as ref


@pytest.fixture(scope="module")
def tq():
    from paper_2402_01798_b200 import build
    build.build()
    from paper_2402_01798_b200 import binding
    binding.lib()
    return binding


# ---- the reference itself -------------------------------------------------------------------------------------------
def test_reference_random_bits_are_the_oracles(orc):
    seed, first = 0x0123456789ABCDEF, 11
    got = ref.random16(seed, 3, 21, first)
    for r in range(3):
        for g in range(3):
            w = orc.philox4x32_10((g, 0, first + r, 0), (seed & 0xFFFFFFFF, seed >> 32))
            slots = [v for x in w for v in (int(x) & 0xFFFF, int(x) >> 16)]
            n = min(8, 21 - 8 * g)
            assert got[r, 8 * g:8 * g + n].tolist() == slots[:n]


def test_reference_nearest_takes_the_nearest_value():
    """Against a search over all sixteen codes, ties to the even one."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 32)) * np.exp(rng.standard_normal((40, 1)) * 3)
    x[:, 3] = np.abs(x).max(1) * 0.3
    code, byte = ref.quantize(x)
    scale = np.ldexp(1.0, byte - 127)
    a = np.abs(x) / scale
    top = a.max(1)
    assert ((top >= 4) & (top < 8)).all()
    distance = np.abs(np.minimum(a, 6.0)[..., None] - ref.GRID)
    best = distance.min(-1)
    chosen = distance[np.arange(40)[:, None], np.arange(32), code[:, 0] & 7]
    assert np.array_equal(chosen, best)
    tied = (distance == best[..., None]).sum(-1) > 1
    assert (code[:, 0][tied] % 2 == 0).all()
    assert np.array_equal(code[:, 0] >> 3, np.signbit(x).astype(int))


def test_reference_stochastic_rounding_has_the_right_mean():
    """Over all 2^16 values of the random bits the mean is the element, to the resolution of 2^-16 of a step; nothing is cut off."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((1, 32)) * 3
    byte = ref.scale_byte(np.abs(x).max(-1), True)
    assert np.abs(x).max() <= 6 * np.ldexp(1.0, byte[0] - 127) and np.abs(x).max() > 3 * np.ldexp(1.0, byte[0] - 127)
    r = np.arange(65536)[:, None, None]
    codes = ref.codes_at(np.broadcast_to(x[:, None], (65536, 1, 32)), np.broadcast_to(byte[:, None], (65536, 1)), np.broadcast_to(r, (65536, 1, 32)))
    mean = ref.decode(codes, np.broadcast_to(byte[:, None], (65536, 1)), 32).mean(0)
    step = 2 * np.ldexp(1.0, byte[0] - 127)
    assert (np.abs(mean - x[0]) <= step * 2.0 ** -17 * (1 + 1e-9)).all()


def test_reference_activation_derivative_by_differences():
    g = np.linspace(-6, 6, 1001)
    for kind in ("silu", "gelu"):
        v, slope, _ = ref.activation(g, kind)
        h = 1e-5
        central = (ref.activation(g + h, kind)[0] - ref.activation(g - h, kind)[0]) / (2 * h)
        assert np.abs(central - slope).max() < 1e-9             # h^2 / 6 of a third derivative below 2, and 2^-52 / h
    assert np.allclose(ref.activation(g, "gelu")[0], 0.5 * g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3))), atol=1e-15)


# ---- sizes ------------------------------------------------------------------------------------------------------------
def test_strides(tq):
    for cols, codes, tiles, rows in ((0, 0, 0, 0), (1, 16, 512, 16), (32, 16, 512, 16), (33, 32, 512, 16), (128, 64, 512, 16), (129, 80, 1024, 16), (513, 272, 2560, 32)):
        assert tq.tq_mx_code_stride(cols) == codes
        assert tq.tq_mx_scale_stride(cols, tq.MX_TILES) == tiles
        assert tq.tq_mx_scale_stride(cols, tq.MX_ROWS) == rows


def test_record_is_plain_c(tq, tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "mx.c"
    src.write_text('''#include "tq.h"
int main(void) {
    tq_mx_t m = {0};
    if (sizeof(tq_mx_t) != 56) return 2;
    if (tq_mx_code_stride(100) != 64) return 3;
    if (tq_mx_product(&m, &m, 0, TQ_F32, 0, 0) != TQ_OK) return 4;          /* nothing to do */
    m.layout = TQ_MX_ROWS;
    return tq_mx_product(&m, &m, 0, TQ_F32, 0, 0) == TQ_ERR_INVALID_ARG ? 0 : 5;
}
''')
    libdir = os.path.dirname(tq.LIB_PATH)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "mx"), "-L", libdir,
                    "-ltq", "-Wl,-rpath," + libdir], check=True, capture_output=True)
    assert subprocess.run([str(tmp_path / "mx")], timeout=120).returncode == 0


# ---- refusals of the library: addresses are made up, nothing is launched ------------------------------------------------
BASE = 1 << 20


def record(tq, rows, cols, layout=0, /, **changes):
    m = tq.Mx(BASE, 2 * BASE, rows, cols, tq.tq_mx_code_stride(cols), tq.tq_mx_scale_stride(cols, layout), layout, 0)
    for k, v in changes.items():
        setattr(m, k, v)
    return m


BAD_RECORDS = [(dict(layout=2), "INVALID_ARG"), (dict(rows=1 << 31), "INVALID_ARG"), (dict(cols=(1 << 40) + 1), "INVALID_ARG"), (dict(codes=None), "INVALID_ARG"),
               (dict(scales=None), "INVALID_ARG"), (dict(codes=BASE + 8), "ALIGNMENT"), (dict(scales=BASE + 4), "ALIGNMENT"), (dict(code_stride=40), "ALIGNMENT"),
               (dict(scale_stride=520), "ALIGNMENT"), (dict(code_stride=16), "BUFFER_TOO_SMALL"), (dict(scale_stride=496), "BUFFER_TOO_SMALL"),
               (dict(code_stride=1 << 40), "INVALID_ARG")]


@pytest.mark.parametrize("changes,status", BAD_RECORDS)
def test_bad_records_are_refused_everywhere(tq, changes, status):
    L, want = tq.lib(), getattr(tq, "ERR_" + status)
    bad, good, square = record(tq, 64, 64, **changes), record(tq, 64, 64), record(tq, 64, 128)
    x = C.c_void_p(4 * BASE)
    r = C.byref
    assert L.tq_mx_quantize(x, tq.F32, 128, 0, 0, 0, r(bad), None) == want
    assert L.tq_mx_quantize_both(x, tq.F32, 128, 0, 0, 0, r(good), r(bad), None) == want
    assert L.tq_mx_dequantize(r(bad), x, tq.F32, 128, None) == want
    assert L.tq_mx_product(r(bad), r(good), x, tq.F32, 128, None) == want
    assert L.tq_mx_product(r(good), r(bad), x, tq.F32, 128, None) == want
    for at in range(4):
        ms = [good] * 4
        ms[at] = bad
        assert L.tq_mx_gated(r(ms[0]), r(ms[1]), r(ms[2]), 0, r(ms[3]), None, tq.F32, 0, None) == want
    tall = record(tq, 128, 64)
    for at in range(3):
        ms = [square, tall, good]
        ms[at] = bad
        assert L.tq_mx_gated_backward(x, 64, x, 128, tq.F32, 0, 0, 0, r(ms[0]), r(ms[1]), r(ms[2]), None) == want
    rows = record(tq, 8, 64, 1, **{k: v for k, v in changes.items() if k not in ("layout", "scale_stride")})
    if "layout" not in changes and "scale_stride" not in changes:
        assert L.tq_mx_decompress_aggregate(r(rows), None, x, None) == want


def test_other_refusals(tq):
    L, r = tq.lib(), C.byref
    x, inv, align, small = C.c_void_p(4 * BASE), tq.ERR_INVALID_ARG, tq.ERR_ALIGNMENT, tq.ERR_BUFFER_TOO_SMALL
    m, t, rows = record(tq, 64, 96), record(tq, 96, 64), record(tq, 64, 96, 1)
    null = C.POINTER(tq.Mx)()
    # quantisation
    assert L.tq_mx_quantize(x, tq.F32, 96, 0, 0, 0, null, None) == inv
    assert L.tq_mx_quantize(x, 2, 96, 0, 0, 0, r(m), None) == inv
    assert L.tq_mx_quantize(x, tq.F32, 96, 2, 0, 0, r(m), None) == inv
    assert L.tq_mx_quantize(None, tq.F32, 96, 0, 0, 0, r(m), None) == inv
    assert L.tq_mx_quantize(C.c_void_p(BASE + 2), tq.F32, 96, 0, 0, 0, r(m), None) == align
    assert L.tq_mx_quantize(C.c_void_p(BASE + 1), tq.BF16, 96, 0, 0, 0, r(m), None) == align
    assert L.tq_mx_quantize(x, tq.F32, 95, 0, 0, 0, r(m), None) == small
    assert L.tq_mx_quantize_both(x, tq.F32, 96, 0, 0, 0, r(m), r(m), None) == inv          # not the transposed shape
    # decoding and the mean
    assert L.tq_mx_dequantize(r(m), x, tq.F32, 95, None) == small
    assert L.tq_mx_dequantize(r(m), C.c_void_p(BASE + 2), tq.F32, 96, None) == align
    assert L.tq_mx_decompress_aggregate(r(m), None, x, None) == inv                        # scales in tiles
    assert L.tq_mx_decompress_aggregate(r(record(tq, 65, 96, 1)), None, x, None) == inv
    assert L.tq_mx_decompress_aggregate(r(record(tq, 0, 96, 1)), None, x, None) == inv
    assert L.tq_mx_decompress_aggregate(r(rows), None, C.c_void_p(BASE + 16), None) == align
    assert L.tq_mx_decompress_aggregate(r(rows), None, None, None) == inv
    # products
    assert L.tq_mx_product(r(m), r(t), x, tq.F32, 96, None) == inv                         # other columns
    assert L.tq_mx_product(r(rows), r(m), x, tq.F32, 96, None) == inv
    assert L.tq_mx_product(r(m), r(m), x, tq.F32, 63, None) == small
    assert L.tq_mx_product(r(m), r(m), None, tq.F32, 64, None) == inv
    assert L.tq_mx_product(r(m), r(m), x, 7, 64, None) == inv
    # the gated block
    xs, w, h = record(tq, 5, 96), record(tq, 64, 96), record(tq, 5, 64)
    gated = lambda xs=xs, wg=w, wu=w, act=0, h=h, p=None, dt=tq.F32, st=0: L.tq_mx_gated(r(xs), r(wg), r(wu), act, r(h), p, dt, st, None)  # noqa: E731
    assert gated(act=2) == inv
    assert gated(wu=record(tq, 96, 96)) == inv and gated(wg=record(tq, 64, 64)) == inv and gated(h=record(tq, 6, 64)) == inv
    assert gated(wg=record(tq, 40, 96), wu=record(tq, 40, 96), h=record(tq, 5, 40)) == inv                # features not a multiple of 32
    assert gated(xs=record(tq, 5, 0), wg=record(tq, 64, 0), wu=record(tq, 64, 0)) == inv
    assert gated(p=x, st=127) == small and gated(p=x, dt=3, st=128) == inv and gated(p=C.c_void_p(BASE + 1), st=128) == align
    back = lambda dh=x, dhs=64, gu=x, gus=128, dt=tq.F32, act=0, rnd=0, a=record(tq, 5, 128), b=record(tq, 128, 5), c=record(tq, 64, 5): \
        L.tq_mx_gated_backward(dh, dhs, gu, gus, dt, act, rnd, 0, r(a), r(b), r(c), None)  # noqa: E731
    assert back(act=2) == inv and back(rnd=2) == inv and back(dt=2) == inv and back(dh=None) == inv and back(gu=None) == inv
    assert back(dhs=63) == small and back(gus=127) == small and back(dh=C.c_void_p(BASE + 2)) == align
    assert back(a=record(tq, 5, 64)) == inv and back(b=record(tq, 128, 6)) == inv and back(c=record(tq, 96, 5)) == inv
    assert back(a=record(tq, 5, 80), b=record(tq, 80, 5), c=record(tq, 40, 5)) == inv


def test_nothing_to_do_is_fine(tq):
    """Empty matrices, without memory, before any CUDA call."""
    L, r = tq.lib(), C.byref
    for rows, cols in ((0, 0), (0, 64), (64, 0)):
        m, t = record(tq, rows, cols, codes=None, scales=None), record(tq, cols, rows, codes=None, scales=None)
        assert L.tq_mx_quantize(None, tq.F32, cols, 0, 0, 0, r(m), None) == tq.OK
        assert L.tq_mx_quantize_both(None, tq.BF16, cols, 1, 0, 0, r(m), r(t), None) == tq.OK
        assert L.tq_mx_dequantize(r(m), None, tq.F32, cols, None) == tq.OK
    assert L.tq_mx_product(r(record(tq, 0, 64)), r(record(tq, 5, 64)), None, tq.F32, 5, None) == tq.OK
    assert L.tq_mx_decompress_aggregate(r(record(tq, 3, 0, 1)), None, None, None) == tq.OK
    assert L.tq_mx_gated(r(record(tq, 0, 64)), r(record(tq, 32, 64)), r(record(tq, 32, 64)), 0, r(record(tq, 0, 32)), None, tq.F32, 0, None) == tq.OK


# ---- refusals of the binding ---------------------------------------------------------------------------------------------
def test_binding_refuses_what_it_can_see(tq):
    codes, scales = torch.zeros((64, 48), dtype=torch.uint8), torch.zeros((1, 512), dtype=torch.uint8)
    m = tq.MxMatrix(codes, scales, 64, 96)
    with pytest.raises(ValueError, match="CUDA tensor"):
        tq.tq_mx_product(m, m, out=torch.zeros(64, 64))
    with pytest.raises(ValueError, match="CUDA tensor"):
        tq.tq_mx_dequantize(m, out=torch.zeros(64, 96))
    with pytest.raises(TypeError):
        tq.tq_mx_product(m, m, torch.float16)
    with pytest.raises(AttributeError):
        tq.tq_mx_product(codes, codes, out=torch.zeros(64, 64))
    with pytest.raises(TypeError):
        tq._calls().mx_product()                                   # too few arguments
