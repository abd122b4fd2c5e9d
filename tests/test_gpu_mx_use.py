"""Microscaled 4-bit operators as they are used together: a training step, a data-parallel round, graphs, streams, long matrices."""
import numpy as np
import pytest
import torch

import mx_reference as ref

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


def near(got, a, b, dtype=torch.bfloat16):
    """got = a b^T within the products' bound: steps of 64 in at least 24 bits, then one rounding to the type."""
    want = a @ b.T
    bound = (-(-a.shape[1] // 64) + 2) * 2.0 ** -22 * (np.abs(a) @ np.abs(b).T)
    bound = bound + torch.finfo(dtype).eps / 2 * (np.abs(want) + bound)
    assert (np.abs(got.cpu().double().numpy() - want) <= bound).all()


def block(tq, rng, t, d, f, act):
    """Inputs and weights of a gated feed-forward block."""
    x = torch.tensor(rng.standard_normal((t, d))).bfloat16().cuda()
    w = torch.tensor(rng.standard_normal((2 * f, d)) * d ** -0.5).bfloat16().cuda()
    wd = torch.tensor(rng.standard_normal((d, f)) * f ** -0.5).bfloat16().cuda()
    return x, w, wd, tq.MX_SILU if act == "silu" else tq.MX_GELU


def step(tq, x, w, wd, act, dy, seed):
    """Forward and backward pass of y = (act(x Wg^T) * (x Wu^T)) Wd^T; all that it makes."""
    f = wd.shape[1]
    q, q_t = tq.tq_mx_quantize_both(x)
    wq, wq_t = tq.tq_mx_quantize_both(w)
    wg, wu = tq.tq_mx_quantize(w[:f]), tq.tq_mx_quantize(w[f:])
    wdq, wdq_t = tq.tq_mx_quantize_both(wd)
    gu = torch.empty(x.shape[0], 2 * f, dtype=torch.bfloat16, device=x.device)
    h = tq.tq_mx_gated(q, wg, wu, act, projections=gu)
    y = tq.tq_mx_product(h, wdq)
    dyq, dyq_t = tq.tq_mx_quantize_both(dy, tq.MX_STOCHASTIC, seed)
    dh = tq.tq_mx_product(dyq, wdq_t)
    dgu, dgu_t, h_t = tq.tq_mx_gated_backward(dh, gu, act, tq.MX_STOCHASTIC, seed + 1)
    dx, dw, dwd = tq.tq_mx_product(dgu, wq_t), tq.tq_mx_product(dgu_t, q_t, torch.float32), tq.tq_mx_product(dyq_t, h_t, torch.float32)
    return dict(q=q, q_t=q_t, wq=wq, wq_t=wq_t, wg=wg, wu=wu, wdq=wdq, wdq_t=wdq_t, gu=gu, h=h, y=y, dyq=dyq, dyq_t=dyq_t, dh=dh, dgu=dgu, dgu_t=dgu_t, h_t=h_t, dx=dx,
                dw=dw, dwd=dwd)


@pytest.mark.parametrize("t,d,f,act", [(1, 96, 64, "silu"), (37, 200, 160, "gelu"), (300, 512, 384, "silu")])
def test_training_step(tq, t, d, f, act):
    rng = np.random.default_rng(t)
    x, w, wd, kind = block(tq, rng, t, d, f, act)
    dy = torch.tensor(rng.standard_normal((t, d)) * 1e-3).bfloat16().cuda()
    s = step(tq, x, w, wd, kind, dy, 17)
    v = {k: values(m) for k, m in s.items() if isinstance(m, tq.MxMatrix)}
    for name, source in (("q", x), ("wq", w), ("wdq", wd)):
        assert np.array_equal(v[name], ref.decode(*ref.quantize(source.cpu().double().numpy()), source.shape[1]))
        assert np.array_equal(v[name + "_t"], ref.decode(*ref.quantize(source.cpu().double().numpy().T), source.shape[0]))
    assert np.array_equal(v["wg"], v["wq"][:f]) and np.array_equal(v["wu"], v["wq"][f:])
    near(s["gu"][:, :f], v["q"], v["wg"])
    near(s["gu"][:, f:], v["q"], v["wu"])
    near(s["y"], v["h"], v["wdq"])
    near(s["dh"], v["dyq"], v["wdq_t"])
    near(s["dx"], v["dgu"], v["wq_t"])
    near(s["dw"], v["dgu_t"], v["q_t"], torch.float32)
    near(s["dwd"], v["dyq_t"], v["h_t"], torch.float32)
    # h and the gradients of the projections: the values behind the codes are within a step (2 scales at most) and the fp32 arithmetic of the formulas
    g, u, e = (z.cpu().double().numpy() for z in (s["gu"][:, :f], s["gu"][:, f:], s["dh"]))
    a, slope, size = ref.activation(g, act)
    for got, want in ((v["dgu"], np.concatenate((e * u * slope, e * a), 1)), (v["dgu_t"].T, np.concatenate((e * u * slope, e * a), 1)), (v["h_t"].T, a * u)):
        # a step is at most 2 scales, and the largest element of its block more than 3 of them
        assert np.abs(got - want).max() <= 2 / 3 * np.abs(want).max() * (1 + 2.0 ** -15)


def test_gradient_of_the_projections_by_differences(tq):
    """Stochastic rounding keeps the expectation: the mean of the decoded gradients over many seeds is the derivative of dh . (act(g) u), taken by differences."""
    rng = np.random.default_rng(5)
    t, f, seeds = 32, 64, 400
    dh, gu = torch.tensor(rng.standard_normal((t, f))).float(), torch.tensor(rng.standard_normal((t, 2 * f))).float()
    e, g, u = dh.double().numpy(), gu[:, :f].double().numpy(), gu[:, f:].double().numpy()
    for act, kind in (("silu", tq.MX_SILU), ("gelu", tq.MX_GELU)):
        step = 1e-5
        value = lambda g, u: e * ref.activation(g, act)[0] * u  # noqa: E731
        want = np.concatenate(((value(g + step, u) - value(g - step, u)) / (2 * step), (value(g, u + step) - value(g, u - step)) / (2 * step)), 1)
        total, total_t, scale = 0.0, 0.0, 0.0
        for seed in range(seeds):
            a, b, _ = tq.tq_mx_gated_backward(dh.cuda(), gu.cuda(), kind, tq.MX_STOCHASTIC, seed)
            total, total_t = total + values(a), total_t + values(b).T
        for got, blocks in ((total / seeds, ref.blocks_of(want)), (total_t / seeds, None)):
            top = np.repeat(np.abs(blocks).max(-1), 32, 1)[:, :2 * f] if blocks is not None else np.repeat(np.abs(ref.blocks_of(want.T)).max(-1), 32, 1)[:, :t].T
            # a step is at most 2 scales, a scale at most a third of the largest element; an element has at most a quarter of the squared step as variance:
            # six standard deviations of the mean, and the resolution of the random bits, the difference quotient and fp32 besides
            assert (np.abs(got - want) <= top * (2 / 3 * 0.5 * 6 / seeds ** 0.5 + 1e-4)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_round_with_mx_messages(tq, dtype):
    """Rows compressed where the workers are (first_row tells them apart) are the rows of one call; their mean is that of the values."""
    from paper_2402_01798_b200 import inputs
    n, d = 5, 100_003
    stride = inputs.worker_stride(d, dtype)
    g = torch.zeros((n, stride), dtype=dtype, device="cuda")
    for i in range(n):
        inputs.powerlaw_gradient(d, 3.0, 1e-3, 60 + i, "cuda", dtype, out=g[i, :d])
    m = tq.tq_mx_quantize(g, tq.MX_STOCHASTIC, 77, cols=d, layout=tq.MX_ROWS)
    for i in (0, 3):
        alone = tq.tq_mx_quantize(g[i], tq.MX_STOCHASTIC, 77, first_row=i, cols=d, layout=tq.MX_ROWS)
        assert torch.equal(alone.codes, m.codes[i:i + 1])
        assert torch.equal(alone.scales[:, :(d + 31) // 32], m.scales[i:i + 1, :(d + 31) // 32])
    out = tq.tq_mx_decompress_aggregate(m).cpu().double().numpy()
    v = values(m)
    assert (np.abs(out - v.mean(0)) <= (n + 1) * 2.0 ** -24 * np.abs(v).mean(0)).all()
    x = g[:, :d].cpu().double().numpy()
    assert np.array_equal(v, ref.decode(*ref.quantize(x, ref.random16(77, n, d)), d))


def test_captured_step_follows_its_inputs(tq):
    rng = np.random.default_rng(8)
    x, w, wd, kind = block(tq, rng, 70, 256, 192, "silu")
    dy = torch.tensor(rng.standard_normal((70, 256)) * 1e-3).bfloat16().cuda()
    step(tq, x, w, wd, kind, dy, 3)                                # first calls set function attributes
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(tq, x, w, wd, kind, dy, 3)
    for seed in (1, 2):
        other = np.random.default_rng(seed)
        for z in (x, w, wd, dy):
            z.copy_(torch.tensor(other.standard_normal(tuple(z.shape))).to(z.dtype))
        graph.replay()
        again = step(tq, x, w, wd, kind, dy, 3)
        for name in ("y", "dx", "dw", "dwd", "gu", "dh"):
            assert torch.equal(held[name], again[name]), name


def test_streams(tq):
    """Two streams at once, each with calls of its own; nothing is shared between them."""
    rng = np.random.default_rng(9)
    sets = [block(tq, rng, t, 512, 256, "silu") + (torch.tensor(rng.standard_normal((t, 512)) * 1e-3).bfloat16().cuda(),) for t in (3, 500)]
    want = [step(tq, x, w, wd, k, dy, 5) for x, w, wd, k, dy in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, (stream, (x, w, wd, k, dy)) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(stream):
                got[i].append(step(tq, x, w, wd, k, dy, 5))
    torch.cuda.synchronize()
    for i, runs in enumerate(got):
        for r in runs:
            for name in ("y", "dx", "dw", "dwd"):
                assert torch.equal(r[name], want[i][name])
    # a stream given by hand
    m = tq.tq_mx_quantize(sets[0][0], stream=streams[1])
    streams[1].synchronize()
    assert np.array_equal(values(m), ref.decode(*ref.quantize(sets[0][0].cpu().double().numpy()), 512))


def test_long_matrices(tq):
    """Codes, scales and values behind 2^32 bytes and elements."""
    rows, cols = 70_000, 131_072                                   # 9.2e9 elements: 4.6 GB of codes, 18 GB of bf16
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.fill_(1.0)
    tail = torch.randn(200, cols, device="cuda").bfloat16()
    x[-200:] = tail
    m = tq.tq_mx_quantize(x)
    last = rows // 128 * 128 - 128                                 # a band of 128 rows near the end
    part = tq.tq_mx_quantize(x[last:])
    view = tq.MxMatrix(m.codes[last:], m.scales[last // 128:], rows - last, cols)
    assert torch.equal(view.codes, part.codes) and torch.equal(view.scales, part.scales)
    b = tq.tq_mx_quantize(torch.randn(96, cols, device="cuda"))
    assert torch.equal(tq.tq_mx_product(m, b)[last:], tq.tq_mx_product(part, b))
    tq.tq_mx_dequantize(m, out=x)
    assert torch.equal(x[last:], tq.tq_mx_dequantize(part, torch.bfloat16))
    assert (x[0] == 1).all()
    del m, view, x
    torch.cuda.empty_cache()


def test_wrong_device_or_shape_is_refused(tq):
    m = tq.tq_mx_quantize(torch.ones(64, 96, device="cuda"))
    with pytest.raises(ValueError, match="smaller"):
        tq.tq_mx_product(m, m, out=torch.empty(63, 64, device="cuda"))
    with pytest.raises(ValueError, match="smaller"):
        tq.tq_mx_dequantize(m, out=torch.empty(64, 95, device="cuda"))
    with pytest.raises(ValueError, match="CUDA tensor"):
        tq.tq_mx_dequantize(m, out=torch.empty(64, 96))
    with pytest.raises(ValueError, match="smaller"):
        tq.tq_mx_product(tq.MxMatrix(m.codes, m.scales, 65, 96), m)
    with pytest.raises(ValueError, match="smaller"):
        tq.tq_mx_product(tq.MxMatrix(None, None, 500, 96, tq.MX_TILES, m.memory), m)
    with pytest.raises(ValueError, match="unit inner stride"):
        tq.tq_mx_quantize(torch.ones(64, 96, device="cuda").t())
    with pytest.raises(ValueError, match="overlap"):
        tq.tq_mx_quantize(torch.ones(1, 96, device="cuda").expand(64, 96))
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        tq.tq_mx_quantize(torch.ones(64, 96, device="cuda", dtype=torch.float16))
    with pytest.raises(tq.TqError) as e:
        tq.tq_mx_product(m, tq.tq_mx_quantize(torch.ones(64, 128, device="cuda")))
    assert e.value.status == tq.ERR_INVALID_ARG
    with pytest.raises(TypeError, match="one type"):
        tq.tq_mx_gated_backward(torch.ones(4, 32, device="cuda"), torch.ones(4, 64, device="cuda").bfloat16())
    # empty ones are fine
    none = tq.tq_mx_quantize(torch.empty(0, 96, device="cuda"))
    assert tq.tq_mx_product(none, m).shape == (0, 64) and tq.tq_mx_dequantize(none).shape == (0, 96)
    flat = tq.tq_mx_quantize(torch.empty(5, 0, device="cuda"))
    assert (tq.tq_mx_product(flat, tq.tq_mx_quantize(torch.empty(7, 0, device="cuda")), torch.float32, out=torch.full((5, 7), 3.0, device="cuda")) == 0).all()


def test_non_finite_values_stay_in_their_blocks(tq):
    """A NaN or an infinity makes its block NaN, in either copy and in the products that read it; nothing else."""
    x = torch.randn(130, 300, device="cuda")
    x[7, 40], x[129, 299] = float("nan"), -float("inf")
    q, q_t = tq.tq_mx_quantize_both(x, tq.MX_STOCHASTIC, 3)
    bad = np.isnan(values(q))
    assert bad[7, 32:64].all() and bad[129, 288:].all() and bad.sum() == 32 + 12
    bad_t = np.isnan(values(q_t))
    assert bad_t[40, :32].all() and bad_t[299, 128:].all() and bad_t.sum() == 32 + 2
    w = tq.tq_mx_quantize(torch.randn(200, 300, device="cuda"))
    y = tq.tq_mx_product(q, w, torch.float32)
    rows = torch.isnan(y).all(1).nonzero().flatten().tolist()
    assert rows == [7, 129] and torch.isnan(y).sum() == 400
    h = values(tq.tq_mx_gated(q, tq.tq_mx_quantize(torch.randn(64, 300, device="cuda")), tq.tq_mx_quantize(torch.randn(64, 300, device="cuda"))))
    assert np.isnan(h[[7, 129]]).all() and np.isnan(h).sum() == 128
    few = tq.MxMatrix(q.codes[:10], q.scales, 10, 300)             # the same by the path for single tokens
    h = values(tq.tq_mx_gated(few, tq.tq_mx_quantize(torch.randn(64, 300, device="cuda")), tq.tq_mx_quantize(torch.randn(64, 300, device="cuda"))))
    assert np.isnan(h[7]).all() and np.isnan(h).sum() == 64
