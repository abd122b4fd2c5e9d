"""Microscaled 4-bit operators where a last bit or a far address shows: the mean's one rounding, a training step code by code, matrices past 2^32 bytes."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from test_gpu_mx import bracket
from test_gpu_mx_gates import slope_error, value_error
from test_gpu_mx_use import block, step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_01798_b200 import binding
    binding.lib()
    yield binding
    assert binding.tq_wait_expired_count() == 0


def values(m):
    return ref.decode(*ref.held(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.rows, m.cols, m.layout), m.cols)


# (scale byte of the first row, of the last ones: 3 more each): ordinary sums, and sums so small that the quotient or its remainder is subnormal
@pytest.mark.parametrize("first_byte", [120, 30, 12, 0])
@pytest.mark.parametrize("d,workers", [(5000, list(range(1, 65))), (2_500_000, [3, 7, 8, 63])])
def test_the_mean_is_rounded_once(tq, d, workers, first_byte):
    """Rows at scales eight apart, whose sum in worker order is exact in fp32 (22 bits): the mean is that sum's IEEE quotient."""
    rng = np.random.default_rng(first_byte)
    for n in workers:
        m = tq.new_mx(n, d, tq.MX_ROWS)
        full = min(n, 7)
        m.codes.zero_()
        m.codes[:full].random_(0, 256, generator=torch.Generator("cuda").manual_seed(n))
        m.scales.copy_((first_byte + 3 * torch.arange(n).clamp_max(6)).to(torch.uint8)[:, None].expand(n, m.scales.shape[1]))
        total = values(m)[:full].sum(0) if d < 10_000 else tq.tq_mx_dequantize(m)[:full].double().sum(0).cpu().numpy()
        assert np.array_equal(total, total.astype(np.float32))
        want = total.astype(np.float32) / np.float32(n)
        got = tq.tq_mx_decompress_aggregate(m).cpu().numpy()
        assert np.array_equal(got, want), (n, np.abs(got - want).max())


@pytest.mark.parametrize("t,d,f,act", [(1, 96, 64, "silu"), (37, 200, 160, "gelu"), (300, 512, 384, "silu")])
def test_training_step_code_by_code(tq, t, d, f, act):
    """What the step's middle writes, against the formulas on the projections and gradients that it kept: every code, not the largest error alone."""
    rng = np.random.default_rng(t)
    x, w, wd, kind = block(tq, rng, t, d, f, act)
    dy = torch.tensor(rng.standard_normal((t, d)) * 1e-3).bfloat16().cuda()
    s = step(tq, x, w, wd, kind, dy, 17)
    g, u, e = (z.cpu().double().numpy() for z in (s["gu"][:, :f], s["gu"][:, f:], s["dh"]))
    a, slope, size = ref.activation(g, act)
    want = np.concatenate((e * u * slope, e * a), 1)
    delta = np.concatenate((np.abs(e * u) * size * (slope_error(g, act) + 2.0 ** -22), np.abs(e * a) * (value_error(g, act) + 2.0 ** -23)), 1)
    random = ref.random16(18, t, 2 * f)
    bracket(want, delta, s["dgu"], random)
    bracket(want.T, delta.T, s["dgu_t"], random.T)
    bracket((a * u).T, (np.abs(a * u) * (value_error(g, act) + 2.0 ** -23)).T, s["h_t"])


ROWS, COLS = 70_000, 131_072                                       # 9.2e9 elements
LAST = ROWS // 128 * 128 - 128                                     # a band of 128 rows near the end, and what follows


def cut(tq, m, first, rows):
    return tq.MxMatrix(m.codes[first:first + rows], m.scales[first // 128:], rows, m.cols)


def test_long_matrices_along_both_axes(tq):
    """Both copies of a matrix past 2^32 bytes: rows near the end, and columns near the end of the transposed copy, are those of a call on that part."""
    x = torch.empty((ROWS, COLS), dtype=torch.bfloat16, device="cuda").normal_()
    out, out_t = tq.tq_mx_quantize_both(x, tq.MX_STOCHASTIC, 9)
    part, part_t = tq.tq_mx_quantize_both(x[LAST:], tq.MX_STOCHASTIC, 9, first_row=LAST)
    view = cut(tq, out, LAST, ROWS - LAST)
    assert torch.equal(view.codes, part.codes) and torch.equal(view.scales, part.scales)
    width = part_t.codes.shape[1]
    assert torch.equal(out_t.codes[:, LAST // 2:LAST // 2 + width], part_t.codes)
    assert torch.equal(out_t.scales[:, LAST // 128 * 512:], part_t.scales)
    ragged = torch.empty((ROWS, COLS - 1), dtype=torch.bfloat16, device="cuda")
    tq.tq_mx_dequantize(tq.MxMatrix(out.codes, out.scales, ROWS, COLS - 1), out=ragged)
    assert torch.equal(ragged[LAST:], tq.tq_mx_dequantize(part, torch.bfloat16)[:, :-1])
    del x, out, out_t, ragged, view, part, part_t
    torch.cuda.empty_cache()


def test_long_gated_blocks(tq):
    """Projections past 2^32 elements, forward and backward."""
    t, d, f = ROWS, 96, 32_768
    x, wg, wu = (tq.tq_mx_quantize(torch.randn(n, d, device="cuda")) for n in (t, f, f))
    gu = torch.empty((t, 2 * f), dtype=torch.bfloat16, device="cuda")
    h = tq.tq_mx_gated(x, wg, wu, projections=gu)
    rows = t - LAST
    some = torch.empty((rows, 2 * f), dtype=torch.bfloat16, device="cuda")
    part = tq.tq_mx_gated(cut(tq, x, LAST, rows), wg, wu, projections=some)
    assert torch.equal(gu[LAST:], some)                            # sums of 96 terms in one order
    view = cut(tq, h, LAST, rows)
    assert torch.equal(view.codes, part.codes) and torch.equal(view.scales, part.scales)
    dh = torch.empty((t, f), dtype=torch.bfloat16, device="cuda").normal_()
    whole = tq.tq_mx_gated_backward(dh, gu, rounding=tq.MX_NEAREST)
    parts = tq.tq_mx_gated_backward(dh[LAST:], gu[LAST:], rounding=tq.MX_NEAREST)
    view = cut(tq, whole[0], LAST, rows)
    assert torch.equal(view.codes, parts[0].codes) and torch.equal(view.scales, parts[0].scales)
    for a, b in zip(whole[1:], parts[1:]):
        assert torch.equal(a.codes[:, LAST // 2:LAST // 2 + b.codes.shape[1]], b.codes) and torch.equal(a.scales[:, LAST // 128 * 512:], b.scales)
    del gu, dh, whole, h, some, part, parts, view, x
    torch.cuda.empty_cache()
