"""The gated block's activation over fp32's whole range, and its backward pass for every way that rows may lie, code by code against 64 bits."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from test_gpu_mx import bracket

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_01798_b200 import binding
    binding.lib()
    yield binding
    assert binding.tq_wait_expired_count() == 0


def kind_of(tq, act):
    return tq.MX_SILU if act == "silu" else tq.MX_GELU


def exponent(g, act):
    """z of x * sigmoid(z)."""
    return g if act == "silu" else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)


def value_error(g, act):
    """How far act(g) may be off, relative to itself, as tq.h says: 2^-20, and for GELU what six roundings of z, each of 2^-24 |z| at most, make of exp(z):
    6 |z| 2^-24 < |z| 2^-21.  Where the value is below 2^-126 its own rounding to a subnormal number comes on top (TINY)."""
    return 2.0 ** -20 + (2.0 ** -21 * np.minimum(np.abs(exponent(g, act)), 200) if act == "gelu" else 0.0)


TINY = 2.0 ** -148


def slope_error(g, act):
    """Relative to the sum of the two terms' magnitudes: s and x z' s (1 - s), which has a second factor of the kind and z' with five roundings."""
    return 2 * value_error(g, act) + 2.0 ** -21


# sums of four E2M1 values at scales of 16, 4, 1 and 1/4 are exact in fp32, as are their products with ones
def exact_projection(rng, features, largest):
    w = np.zeros((features, 128))
    for i, scale in enumerate((16, 4, 1, 0.25)):
        w[:, 32 * i] = ref.GRID[rng.integers(0, 8, features)] * scale
    w[:, 0] = np.where(largest, 96, np.minimum(w[:, 0], 64))
    return w


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens", [1, 16, 40, 4000])
def test_gates_of_large_magnitude(tq, tokens, act):
    """Blocks whose gates are all far below zero, where x * sigmoid(x) is a small normal number and not zero; far above, where it is x; and mixtures."""
    rng = np.random.default_rng(tokens)
    f = 2080
    x = np.zeros((tokens, 128))
    x[:, ::32] = 1.0
    # SiLU: -64 to -117; GELU reaches exp(-88) near -9
    wg = exact_projection(rng, f, rng.random(f) < 0.3) * (-1.0 if act == "silu" else -0.125)
    wg[:32] = 0.0                                                                              # a block of one value: -96, or -10
    wg[:32, 0], wg[:32, 32] = (-96, 0) if act == "silu" else (-8, -2)
    wg[32:64] *= -1
    wg[64:96] *= rng.choice([-1, 1], (32, 1))
    wu = exact_projection(rng, f, rng.random(f) < 0.5) * rng.choice([-1, 1], (f, 1))
    mats = [tq.tq_mx_quantize(torch.tensor(v, dtype=torch.float32, device="cuda")) for v in (x, wg, wu)]
    for m, v in zip(mats, (x, wg, wu)):
        assert np.array_equal(ref.decode(*ref.held(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.rows, m.cols, m.layout), m.cols), v)
    h = tq.tq_mx_gated(*mats, kind_of(tq, act))
    g, u = x @ wg.T, x @ wu.T
    a, _, _ = ref.activation(g, act)
    assert (np.abs(a[:, :32] * u[:, :32]).max() < 2.0 ** -100) and np.abs(a[:, :32]).min() > 0
    delta = (value_error(g, act) + 2.0 ** -23) * np.abs(a * u) + TINY * np.abs(u) + TINY
    bracket(a * u, delta, h)


def gates(rng, tokens, f):
    g = rng.standard_normal((tokens, f)) * 2
    for start, low, high in ((0, -103, -80), (32, -12, -8), (64, 80, 1e4)):
        g[:, start:start + 32] = rng.uniform(low, high, (tokens, 32))
    pick = rng.random((tokens, f)) < 0.01
    g[pick] = (rng.choice([-1, 1], (tokens, f)) * 10.0 ** rng.uniform(-30, 37, (tokens, f)))[pick]
    return g


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gates_of_large_magnitude_in_the_backward_pass(tq, dtype, act, stochastic):
    rng = np.random.default_rng(8)
    tokens, f = 96, 128
    gu = np.concatenate((gates(rng, tokens, f), rng.standard_normal((tokens, f))), 1)
    check_backward(tq, rng, gu, torch.tensor(rng.standard_normal((tokens, f))).to(dtype), act, stochastic, dtype)


def check_backward(tq, rng, gu, dh, act, stochastic, dtype, pad=(0, 0)):
    """Every code and scale of the three outputs lies where fp32 arithmetic of the formulas puts it."""
    tokens, f = dh.shape
    def laid(v, more):
        wide = torch.zeros((tokens, v.shape[1] + more), dtype=dtype, device="cuda")
        wide[:, :v.shape[1]] = v
        return wide[:, :v.shape[1]]
    gu = torch.tensor(gu).to(dtype)
    outs = tq.new_mx(tokens, 2 * f), tq.new_mx(2 * f, tokens), tq.new_mx(f, tokens)
    for m in outs:
        m.codes.fill_(0xEE); m.scales.fill_(0xEE)
    seed = 31337
    tq.tq_mx_gated_backward(laid(dh, pad[0]), laid(gu, pad[1]), kind_of(tq, act), tq.MX_STOCHASTIC if stochastic else tq.MX_NEAREST, seed, *outs)
    g, u, e = gu[:, :f].double().numpy(), gu[:, f:].double().numpy(), dh.double().numpy()
    with np.errstate(over="ignore"):
        a, slope, size = ref.activation(g, act)
    x = np.concatenate((e * u * slope, e * a), 1)
    # products of inputs that are exact: two roundings more, and subnormal numbers between them
    delta = np.concatenate((np.abs(e * u) * (size * (slope_error(g, act) + 2.0 ** -22) + TINY), np.abs(e) * (np.abs(a) * (value_error(g, act) + 2.0 ** -23) + TINY)), 1) + TINY
    random = ref.random16(seed, tokens, 2 * f) if stochastic else None
    bracket(x, delta, outs[0], random)
    bracket(x.T, delta.T, outs[1], random.T if stochastic else None)
    bracket((a * u).T, (np.abs(u) * (np.abs(a) * (value_error(g, act) + 2.0 ** -23) + TINY) + TINY).T, outs[2])
    for m in outs:
        rest = m.scales.cpu().numpy().reshape(-1).copy()
        rest[ref.scale_index(m.rows, -(-m.cols // 32), ref.TILES, m.scales.shape[1])] = 0
        assert not rest.any()


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [(0, 0), (8, 8), (5, 5), (16, 5)])
@pytest.mark.parametrize("tokens,f", [(65, 96), (200, 352)])
def test_backward_of_rows_on_every_boundary(tq, tokens, f, pad, dtype, stochastic):
    """Rows of both inputs on 32-byte boundaries, on 16-byte ones and on none: the inputs come ahead or do not."""
    rng = np.random.default_rng(tokens + pad[0])
    check_backward(tq, rng, rng.standard_normal((tokens, 2 * f)) * 2, torch.tensor(rng.standard_normal((tokens, f)) * 1e-3).to(dtype), "silu", stochastic, dtype, pad)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.bfloat16, "gelu"), (torch.float32, "gelu")])
def test_backward_with_several_tiles_a_block(tq, dtype, act, stochastic):
    """More tiles of 64 x 128 than two for each SM, so that blocks go on to a second one, both ends ragged."""
    rng = np.random.default_rng(77)
    tokens, f = 1300, 2080
    assert -(-tokens // 128) * 2 * -(-f // 128) > 2 * torch.cuda.get_device_properties(0).multi_processor_count
    check_backward(tq, rng, rng.standard_normal((tokens, 2 * f)) * 2, torch.tensor(rng.standard_normal((tokens, f)) * 1e-3).to(dtype), act, stochastic, dtype)
