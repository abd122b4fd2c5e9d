"""Microscaled 4-bit operators on the GPU against their definition in 64 bits (mx_reference)."""
import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def tq():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_01798_b200 import binding
    binding.lib()
    yield binding
    assert binding.tq_wait_expired_count() == 0


def host(m):
    return m.codes.cpu().numpy(), m.scales.cpu().numpy()


def held(m):
    c, s = host(m)
    return ref.held(c, s, m.rows, m.cols, m.layout)


def values(m):
    return ref.decode(*held(m), m.cols)


def assert_matrix(m, code, byte):
    """Codes and scales as expected, and zeros where the last block and the last scale tiles are filled up."""
    got_code, got_byte = held(m)
    assert np.array_equal(got_byte, byte)
    assert np.array_equal(got_code, code)
    if m.layout == ref.TILES:
        _, s = host(m)
        rest = np.ones(s.size, bool)
        rest[ref.scale_index(m.rows, byte.shape[1], ref.TILES, s.shape[1]).reshape(-1)] = False
        bands = -(-m.rows // 128)
        assert not s.reshape(-1)[rest][: bands * s.shape[1]].any()


def matrix(rng, rows, cols, dtype):
    """Values over many orders of magnitude, zeros and ties of the grid among them."""
    x = rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.75])
    pick = rng.random((rows, cols)) < 0.1
    x[pick] = (ties[rng.integers(0, len(ties), (rows, cols))] * rng.choice([-1, 1], (rows, cols)))[pick]
    return torch.tensor(x, dtype=torch.float32).to(dtype)


SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (64, 1024), (127, 129), (128, 128), (129, 255), (300, 1000), (33, 4096)]


@pytest.mark.parametrize("layout", [ref.TILES, ref.ROWS])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize(tq, rows, cols, dtype, stochastic, layout):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = matrix(rng, rows, cols, dtype)
    seed, first = 0x123456789ABCDEF, 7
    out = tq.new_mx(rows, cols, layout)
    out.codes.fill_(0xEE); out.scales.fill_(0xEE)
    tq.tq_mx_quantize(x.cuda(), tq.MX_STOCHASTIC if stochastic else tq.MX_NEAREST, seed, first, out=out)
    want = ref.quantize(x.double().numpy(), ref.random16(seed, rows, cols, first) if stochastic else None)
    assert_matrix(out, *want)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_both(tq, rows, cols, dtype, stochastic):
    rng = np.random.default_rng(rows * 1000 + cols + 1)
    x = matrix(rng, rows, cols, dtype)
    seed, first = 99, 2 ** 31
    out, out_t = tq.new_mx(rows, cols), tq.new_mx(cols, rows)
    for m in (out, out_t):
        m.codes.fill_(0xEE); m.scales.fill_(0xEE)
    tq.tq_mx_quantize_both(x.cuda(), tq.MX_STOCHASTIC if stochastic else tq.MX_NEAREST, seed, first, out, out_t)
    random = ref.random16(seed, rows, cols, first) if stochastic else None
    assert_matrix(out, *ref.quantize(x.double().numpy(), random))
    assert_matrix(out_t, *ref.quantize(x.double().numpy().T, random.T if stochastic else None))


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_extremes(tq, dtype, stochastic):
    """NaN, infinities, zeros of both signs, the type's largest and smallest numbers, scales at the ends of their range."""
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal
    rows = [[float("nan")] + [1.0] * 31, [1.0] * 31 + [float("inf")], [-float("inf")] + [0.0] * 31, [0.0] * 32, [-0.0] * 32, [top, -top, top / 2, 1.0] * 8,
            [tiny, tiny * 0.5, -tiny * 3, 0.0] * 8, [tiny * 2.0 ** k for k in range(-7, 25)], [6.0, 4.0, 3.0, 2.0, 1.5, 1.0, 0.5, 0.0] * 4,
            [7.9, 6.1, 5.0, -7.0, 6.0, -6.0, 5.9, 4.1] * 4, [1.5 * 2.0 ** -126] * 32, [2.0 ** -127] * 32]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype)
    random = ref.random16(5, *x.shape) if stochastic else None
    want = ref.quantize(x.double().numpy(), random)
    mode = tq.MX_STOCHASTIC if stochastic else tq.MX_NEAREST
    assert_matrix(tq.tq_mx_quantize(x.cuda(), mode, 5), *want)
    both, both_t = tq.tq_mx_quantize_both(x.cuda(), mode, 5)
    assert_matrix(both, *want)
    assert_matrix(both_t, *ref.quantize(x.double().numpy().T, random.T if stochastic else None))
    back = tq.tq_mx_dequantize(both, torch.float32).cpu().double().numpy()
    with np.errstate(over="ignore"):                               # 4 * 2^126 is past fp32
        assert np.array_equal(back, ref.decode(*want, 32).astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_strided_rows_and_columns(tq, dtype):
    """Rows on any boundary, a view of columns, outputs that are part of larger matrices: what lies beside them stays."""
    rng = np.random.default_rng(3)
    big = matrix(rng, 200, 777, dtype).cuda()
    for first_col, cols in ((0, 500), (3, 501), (8, 128)):
        x = big[:, first_col:first_col + cols]
        out, out_t = tq.new_mx(200, 1024), tq.new_mx(640, 384)
        for m in (out, out_t):
            m.codes.fill_(0xEE); m.scales.fill_(0xEE)
        part = tq.MxMatrix(out.codes[:, 128:], out.scales[:, 1024:], 200, cols)
        part_t = tq.MxMatrix(out_t.codes[128:, 64:], out_t.scales[1:, 512:], cols, 200)
        tq.tq_mx_quantize_both(x, out=part, out_t=part_t)
        want, want_t = ref.quantize(x.double().cpu().numpy()), ref.quantize(x.double().cpu().numpy().T)
        blocks = -(-cols // 32)
        code, byte = ref.held(out.codes.cpu().numpy()[:, 128:], out.scales.cpu().numpy(), 200, cols, ref.TILES)
        assert np.array_equal(code, want[0])
        at = ref.scale_index(200, blocks, ref.TILES, out.scales.shape[1]) + 1024
        assert np.array_equal(out.scales.cpu().numpy().reshape(-1)[at], want[1])
        code_t = out_t.codes.cpu().numpy()[128:128 + cols, 64:64 + 112]
        code_t = np.stack((code_t & 15, code_t >> 4), -1).reshape(cols, 7, 32)
        assert np.array_equal(code_t, want_t[0])
        assert (out.codes[:, :128] == 0xEE).all() and (out.codes[:, 128 + 16 * blocks:] == 0xEE).all()
        assert (out_t.codes[:128] == 0xEE).all() and (out_t.codes[:, :64] == 0xEE).all() and (out_t.codes[128 + cols:] == 0xEE).all()
        assert (out_t.scales[0] == 0xEE).all() and (out_t.scales[:, :512] == 0xEE).all() and (out.scales[:, :1024] == 0xEE).all()


@pytest.mark.parametrize("layout", [ref.TILES, ref.ROWS])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(2, 5003)])
def test_dequantize(tq, rows, cols, dtype, layout):
    rng = np.random.default_rng(cols)
    m = tq.new_mx(rows, cols, layout)
    m.codes.copy_(torch.from_numpy(rng.integers(0, 256, m.codes.shape, dtype=np.uint8)))
    m.scales.copy_(torch.from_numpy(rng.integers(0, 253, m.scales.shape, dtype=np.uint8)))        # 253 and up would overflow
    m.scales[:, ::5] = 255
    out = torch.full((rows + 1, cols + 3), -7.0, dtype=dtype, device="cuda")
    tq.tq_mx_dequantize(m, out=out[:rows, :cols])
    want = values(m)
    got = out.cpu().double().numpy()
    assert np.array_equal(got[:rows, :cols], want, equal_nan=True)
    assert (got[rows] == -7).all() and (got[:, cols:] == -7).all()
    assert np.array_equal(tq.tq_mx_dequantize(m, dtype).cpu().double().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("workers", [1, 2, 3, 8, 16, 64])
@pytest.mark.parametrize("d", [1, 31, 32, 1000, 100_003])
def test_aggregate(tq, workers, d, weighted):
    rng = np.random.default_rng(d + workers)
    m = tq.new_mx(workers, d, tq.MX_ROWS)
    m.codes.copy_(torch.from_numpy(rng.integers(0, 256, m.codes.shape, dtype=np.uint8)))
    m.scales.copy_(torch.from_numpy(rng.integers(100, 140, m.scales.shape, dtype=np.uint8)))
    w = [float(np.float32(v)) for v in rng.standard_normal(workers)] if weighted else None
    out = torch.full(((d + 7) // 8 * 8 + 8,), -7.0, device="cuda")
    tq.tq_mx_decompress_aggregate(m, w, out=out)
    v = values(m)
    want = (v * np.array(w)[:, None]).sum(0) if weighted else v.mean(0)
    # products rounded once, N additions and a division, each within 2^-24 of at most the sum of magnitudes
    bound = (workers + 1) * 2.0 ** -24 * np.abs(v * (np.array(w)[:, None] if weighted else 1 / workers)).sum(0) + 1e-300
    got = out.cpu().double().numpy()
    assert (np.abs(got[:d] - want) <= bound).all()
    assert (got[d:] == -7).all()


def random_mx(tq, rng, rows, cols, spread=4):
    """Any codes, scales over 2 * spread powers of two, the filling of the last tiles zero."""
    m = tq.new_mx(rows, cols)
    blocks = -(-cols // 32)
    code = rng.integers(0, 16, (rows, blocks * 32), dtype=np.uint8)
    code[:, cols:] = 0
    m.codes.copy_(torch.from_numpy(code[:, 0::2] | (code[:, 1::2] << 4)))
    s = np.zeros(m.scales.shape, np.uint8).reshape(-1)
    s[ref.scale_index(rows, blocks, ref.TILES, m.scales.shape[1])] = rng.integers(127 - spread, 128 + spread, (rows, blocks), dtype=np.uint8)
    m.scales.copy_(torch.from_numpy(s.reshape(m.scales.shape)))
    return m


def sum_bound(a, b, k):
    """What sums in fp32 may be off: products are exact; the tensor cores add 64 of them and the sum so far at a time, in 24 bits or more and cutting
    off, so each of the steps loses at most 2^-22 of the sum of magnitudes."""
    return (-(-k // 64) + 2) * 2.0 ** -22 * (np.abs(a) @ np.abs(b).T)


PRODUCTS = [(1, 1, 1), (1, 64, 32), (1, 1000, 4096), (3, 7, 64), (8, 128, 96), (16, 300, 256), (17, 129, 288), (64, 257, 130), (100, 512, 500), (127, 255, 512),
            (128, 256, 256), (129, 1, 1000), (130, 384, 2048), (256, 512, 777), (300, 700, 1056), (513, 130, 32), (1025, 1300, 384), (4096, 3000, 320), (2300, 4100, 96), (4000, 4099, 1000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(tq, m, n, k, dtype):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    a, b = random_mx(tq, rng, m, k), random_mx(tq, rng, n, k)
    out = torch.full((m + 1, n + 5), -7.0, dtype=dtype, device="cuda")
    tq.tq_mx_product(a, b, out=out[:m, :n])
    va, vb = values(a), values(b)
    want, got = va @ vb.T, out.cpu().double().numpy()
    bound = sum_bound(va, vb, k)
    bound = bound + torch.finfo(dtype).eps / 2 * (np.abs(want) + bound)
    assert (np.abs(got[:m, :n] - want) <= bound).all(), np.abs(got[:m, :n] - want).max()
    assert (got[m] == -7).all() and (got[:, n:] == -7).all()
    assert np.array_equal(tq.tq_mx_product(a, b, dtype).cpu().double().numpy(), got[:m, :n])


@pytest.mark.parametrize("m", [1, 8, 9, 24, 40, 47, 56, 64, 72, 96, 120, 127])
def test_few_rows_with_long_sums(tq, m):
    """Every number of rows that is loaded at a time, with more stages of k than fit the chip."""
    rng = np.random.default_rng(m)
    for n, k in ((520, 8192), (16_500, 2560)):
        a, b = random_mx(tq, rng, m, k, 1), random_mx(tq, rng, n, k, 1)
        va, vb = values(a), values(b)
        want, got = va @ vb.T, tq.tq_mx_product(a, b, torch.float32).cpu().double().numpy()
        bound = sum_bound(va, vb, k)
        assert (np.abs(got - want) <= bound + 2.0 ** -24 * (np.abs(want) + bound)).all()
    x, wg, wu = random_mx(tq, rng, m, 4096, 1), random_mx(tq, rng, 256, 4096, 1), random_mx(tq, rng, 256, 4096, 1)
    gu = torch.empty(m, 512, device="cuda")
    tq.tq_mx_gated(x, wg, wu, projections=gu)
    for half, w in ((gu[:, :256], wg), (gu[:, 256:], wu)):
        want, bound = values(x) @ values(w).T, sum_bound(values(x), values(w), 4096)
        assert (np.abs(half.cpu().double().numpy() - want) <= bound + 2.0 ** -24 * (np.abs(want) + bound)).all()


def test_product_with_operands_beyond_the_cache(tq):
    """Tiles in groups of rows, the last group ragged: the rows of one call are those of calls on parts of it, which take the tiles in another order.  The parts
    are tall enough for the same kernel, which adds k in one order whatever the tile's place."""
    rng = np.random.default_rng(12)
    a, b = random_mx(tq, rng, 5400, 16384, 1), random_mx(tq, rng, 5000, 16384, 1)
    whole = tq.tq_mx_product(a, b, torch.float32)
    assert (5400 + 5000) * 16384 * 17 // 32 > 80_000_000
    for first, rows in ((0, 2560), (2560, 2840)):
        part = tq.MxMatrix(a.codes[first:first + rows], a.scales[first // 128:], rows, 16384)
        assert torch.equal(whole[first:first + rows], tq.tq_mx_product(part, b, torch.float32))
    va, vb = values(a)[5300:], values(b)
    assert (np.abs(whole[5300:].cpu().double().numpy() - va @ vb.T) <= sum_bound(va, vb, 16384) * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(va @ vb.T)).all()


def test_product_scales_reach_the_ends(tq):
    """Every scale byte, and NaN blocks: a row of one operand that holds one is NaN, the others are untouched."""
    rng = np.random.default_rng(4)
    a, b = random_mx(tq, rng, 256, 128, 1), random_mx(tq, rng, 64, 128, 1)
    s = a.scales.cpu().numpy().reshape(-1)
    at = ref.scale_index(256, 4, ref.TILES, a.scales.shape[1])
    s[at] = np.arange(256, dtype=np.uint8)[:, None]               # byte 255: NaN
    a.scales.copy_(torch.from_numpy(s.reshape(a.scales.shape)))
    va, vb = values(a), values(b)
    got = tq.tq_mx_product(a, b, torch.float32).cpu().double().numpy()
    with np.errstate(over="ignore", invalid="ignore"):
        want = va @ vb.T
    assert np.isnan(got[255]).all()
    # a sum on its way reaches up to the sum of magnitudes: where that passes fp32, infinity is right although the result would fit
    fine = np.abs(np.nan_to_num(va)) @ np.abs(vb).T < 2.0 ** 127
    small = 2.0 ** -126                                           # subnormal results may be cut off
    fine[255] = False
    bound = sum_bound(np.nan_to_num(va), vb, 128) * 2 + small
    assert (np.abs(got - want)[fine] <= bound[fine]).all()


def bracket(x, delta, m, random=None):
    """`m` holds x quantised, where x is known to `delta` only: every code lies between those of the two ends."""
    code, byte = held(m)
    lo, hi = ref.blocks_of(x - delta), ref.blocks_of(x + delta)
    top = np.abs(ref.blocks_of(x)).max(-1)
    slack = ref.blocks_of(np.abs(delta)).max(-1)
    low_byte, high_byte = (ref.scale_byte(np.maximum(t, 0), random is not None) for t in (top - slack, top + slack))
    assert ((byte == low_byte) | (byte == high_byte)).all()
    r = None if random is None else ref.blocks_of(random)
    def value(z):
        return ref.decode(ref.codes_at(z, byte, r), byte, m.cols)
    got = ref.decode(code, byte, m.cols)
    if random is None:
        low, high = value(lo), value(hi)
    else:                                                          # rounding by magnitude: monotone on either side of zero
        low = np.minimum(value(lo), value(hi))
        high = np.maximum(value(lo), value(hi))
        cross = (x - delta < 0) & (x + delta > 0)
        step = 0.5 * np.repeat(np.ldexp(1.0, byte - 127), 32, 1)[:, :m.cols]
        low, high = np.where(cross, np.minimum(low, -step), low), np.where(cross, np.maximum(high, step), high)
    assert (got >= low).all() and (got <= high).all()


@pytest.mark.parametrize("dtype", [None] + DTYPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,d,f", [(1, 32, 32), (1, 256, 128), (2, 1000, 96), (5, 288, 352), (40, 512, 256), (128, 300, 160), (200, 640, 416), (300, 96, 1024), (4000, 288, 2080), (1300, 130, 8224)])
def test_gated(tq, tokens, d, f, act, dtype):
    rng = np.random.default_rng(tokens + d + f)
    x, wg, wu = random_mx(tq, rng, tokens, d, 1), random_mx(tq, rng, f, d, 1), random_mx(tq, rng, f, d, 1)
    for w in (wg, wu):                                             # bring the projections to the size of one
        s = w.scales.cpu().numpy()
        w.scales.copy_(torch.from_numpy(np.where(s > 8, s - 6, s).astype(np.uint8)))
    out = tq.new_mx(tokens, f)
    out.codes.fill_(0xEE); out.scales.fill_(0xEE)
    gu = None if dtype is None else torch.full((tokens + 1, 2 * f + 3), -7.0, dtype=dtype, device="cuda")
    kind = tq.MX_SILU if act == "silu" else tq.MX_GELU
    tq.tq_mx_gated(x, wg, wu, kind, None if gu is None else gu[:tokens, :2 * f], out)
    vx, vg, vu = values(x), values(wg), values(wu)
    g, u = vx @ vg.T, vx @ vu.T
    dg, du = sum_bound(vx, vg, d), sum_bound(vx, vu, d)
    a, slope, _ = ref.activation(g, act)
    # the activation in fp32: exp to (2 + 1.2 |z|) 2^-23 and z to 4 2^-24 of itself, |z| below 24 where s has not vanished, and a few roundings
    delta = 2.0 ** -16 * np.abs(a * u) + 1.2 * dg * np.abs(u) + np.abs(a) * du + 1.2 * dg * du
    bracket(a * u, delta, out)
    rest = out.scales.cpu().numpy().reshape(-1).copy()
    rest[ref.scale_index(tokens, f // 32, ref.TILES, out.scales.shape[1])] = 0
    assert not rest.any()
    if gu is not None:
        got = gu.cpu().double().numpy()
        want, bound = np.concatenate((g, u), 1), np.concatenate((dg, du), 1)
        assert (np.abs(got[:tokens, :2 * f] - want) <= bound + torch.finfo(dtype).eps / 2 * (np.abs(want) + bound)).all()
        assert (got[tokens] == -7).all() and (got[:, 2 * f:] == -7).all()


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,f", [(1, 32), (3, 96), (33, 128), (128, 160), (200, 352), (257, 512)])
def test_gated_backward(tq, tokens, f, dtype, act, stochastic):
    rng = np.random.default_rng(tokens * 3 + f)
    dh = torch.tensor(rng.standard_normal((tokens, f + 5)) * 1e-3).to(dtype)[:, :f]
    gu = torch.tensor(rng.standard_normal((tokens, 2 * f)) * 2).to(dtype)
    outs = tq.new_mx(tokens, 2 * f), tq.new_mx(2 * f, tokens), tq.new_mx(f, tokens)
    for m in outs:
        m.codes.fill_(0xEE); m.scales.fill_(0xEE)
    seed = 31337
    tq.tq_mx_gated_backward(dh.cuda(), gu.cuda(), tq.MX_SILU if act == "silu" else tq.MX_GELU, tq.MX_STOCHASTIC if stochastic else tq.MX_NEAREST, seed, *outs)
    g, u, e = gu[:, :f].double().numpy(), gu[:, f:].double().numpy(), dh.double().numpy()
    a, slope, size = ref.activation(g, act)
    x = np.concatenate((e * u * slope, e * a), 1)
    # fp32 arithmetic on inputs that are exact: as in the forward pass, relative to the terms of the derivative
    delta = 2.0 ** -16 * np.concatenate((np.abs(e * u) * size, np.abs(e * a)), 1)
    random = ref.random16(seed, tokens, 2 * f) if stochastic else None
    bracket(x, delta, outs[0], random)
    bracket(x.T, delta.T, outs[1], random.T if stochastic else None)
    bracket((a * u).T, 2.0 ** -16 * np.abs(a * u).T, outs[2])
    for m in outs:
        rest = m.scales.cpu().numpy().reshape(-1).copy()
        rest[ref.scale_index(m.rows, -(-m.cols // 32), ref.TILES, m.scales.shape[1])] = 0
        assert not rest.any()
