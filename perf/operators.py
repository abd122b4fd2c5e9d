"""Timed cases of the microscaled 4-bit operators, each in a plain form (``own`` false) and through the calls of tq.h.

A microscaled matrix (MX) holds E2M1 codes, two in a byte, and one E8M0 scale (a power of two) for every 32 elements of a
row.  What a case does (``kind``):

  quantize   a matrix -> MX, along its rows and, with ``both``, along its columns as well (the transposed copy that a
             gradient product needs), and the values that the codes stand for.
  round      one data-parallel round with MX as the wire format: N workers' gradient rows -> MX with stochastic
             rounding -> mean of the N decoded rows.
  server     the mean alone, of rows that have arrived.
  product    A B^T of two MX matrices that lie in memory.
  gated      a gated feed-forward block: x -> MX -> act(x Wg^T) * (x Wu^T) -> MX -> times Wd^T.  ``save``: a training step's
             forward pass, which keeps both projections.
  gated_grad the block's backward pass from dy and what the forward pass kept: gradients of x, of [Wg; Wu] and of Wd,
             every product on MX operands with stochastically rounded gradients.

Nearest rounding: scale 2^(floor(log2 max) - 2), to even on ties, magnitudes above 6 become 6.  Stochastic rounding: the
smallest scale at which no element exceeds 6; element (row, col) goes up when its 16 random bits are below
rint(p * 2^16), the bits being those of Philox4x32-10 with key = seed, counter = (col >> 3, row), slot col & 7.  Blocks
that hold a NaN or an infinity decode as NaN.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"float32": torch.float32, "bfloat16": torch.bfloat16}
_MOST = {"quantize": 1 << 26, "round": 25_600_000 * 16, "server": 25_600_000 * 16, "product": 8192 ** 3,
         "gated": 4096 * 4096 * 8192, "gated_grad": 8192 * 4096 * 8192}


def listed():
    return [
        # activations of a few requests that are served together: the smallest call
        dict(name="quantize_64x1024", kind="quantize", rows=64, cols=1024, dtype="bfloat16", rounding="nearest", both=False),
        # a training step's activations, once along each axis
        dict(name="quantize_4k", kind="quantize", rows=4096, cols=4096, dtype="bfloat16", rounding="nearest", both=True),
        # output gradients in fp32 at a ragged size, rounded stochastically, once along each axis
        dict(name="quantize_ragged", kind="quantize", rows=8191, cols=5003, dtype="float32", rounding="stochastic", both=True),
        # a small model's gradient, three workers: latency
        dict(name="round_200k", kind="round", workers=3, d=200_003, dtype="float32"),
        # ResNet-50-sized gradients of 16 workers, the benchmark's default round
        dict(name="round_25m", kind="round", workers=16, d=25_600_000, dtype="float32"),
        # one token's projection while serving
        dict(name="product_token", kind="product", m=1, n=8192, k=4096, out="bfloat16"),
        # a ragged batch, sizes that fill no tile
        dict(name="product_ragged", kind="product", m=777, n=1000, k=4000, out="float32"),
        # a long prompt's or a training step's projection
        dict(name="product_8k", kind="product", m=8192, n=8192, k=8192, out="bfloat16"),
        # four requests, one token each
        dict(name="gated_tokens", kind="gated", tokens=4, d=4096, f=8192, act="silu", save=False),
        # a training step's forward pass
        dict(name="gated_4k", kind="gated", tokens=4096, d=4096, f=8192, act="silu", save=True),
        # the backward pass of a small block on a short ragged batch
        dict(name="gated_grad_small", kind="gated_grad", tokens=250, d=1024, f=2048, act="gelu"),
        # the backward pass of a training step
        dict(name="gated_grad_8k", kind="gated_grad", tokens=8192, d=4096, f=8192, act="silu"),
    ]


def _spread(rng, lo, hi):
    """A size from lo to hi, even over the logarithm; every other one a power of two or a multiple of 128 nearby."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 256:
        v = v // 128 * 128
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "round", "server", "product", "product", "gated", "gated_grad"])
    for _ in range(1000):
        if kind == "quantize":
            c = dict(rows=_spread(rng, 1, 16384), cols=_spread(rng, 16, 16384), dtype=rng.choice(["bfloat16", "float32"]),
                     rounding=rng.choice(["nearest", "stochastic"]), both=rng.random() < 0.5)
            size = c["rows"] * c["cols"]
        elif kind in ("round", "server"):
            c = dict(workers=_spread(rng, 1, 64), d=_spread(rng, 10_000, 100_000_000), dtype=rng.choice(["bfloat16", "float32"]))
            size = c["workers"] * c["d"]
        elif kind == "product":
            c = dict(m=_spread(rng, 1, 8192), n=_spread(rng, 64, 8192), k=_spread(rng, 64, 8192), out=rng.choice(["bfloat16", "float32"]))
            size = c["m"] * c["n"] * c["k"]
        else:
            c = dict(tokens=_spread(rng, 1, 8192), d=_spread(rng, 8, 256) * 32, f=_spread(rng, 8, 512) * 32, act=rng.choice(["silu", "gelu"]))
            if kind == "gated":
                c["save"] = rng.random() < 0.5
            size = c["tokens"] * c["d"] * c["f"]
        if size <= _MOST[kind]:
            return dict(kind=kind, **c)
    raise ValueError("no size in range")


# ---- plain forms ------------------------------------------------------------------------------------------------------
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)
_M32 = 0xFFFFFFFF


def _philox16(seed, rows, cols, device, first_row=0):
    """16 random bits for every element of a rows x cols matrix, as int32."""
    groups = (cols + 7) // 8
    x0 = torch.arange(groups, device=device, dtype=torch.int64).expand(rows, groups)
    x2 = (first_row + torch.arange(rows, device=device, dtype=torch.int64)).unsqueeze(1).expand(rows, groups)
    x1, x3 = torch.zeros_like(x0), torch.zeros_like(x0)
    k0, k1 = seed & _M32, (seed >> 32) & _M32
    for _ in range(10):
        p0, p1 = x0 * 0xD2511F53, x2 * 0xCD9E8D57          # the low 64 bits of a signed product are those of the unsigned one
        x0, x1, x2, x3 = ((p1 >> 32) & _M32) ^ x1 ^ k0, p1 & _M32, ((p0 >> 32) & _M32) ^ x3 ^ k1, p0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    words = torch.stack((x0, x1, x2, x3), -1)
    bits = torch.stack((words & 0xFFFF, words >> 16), -1).to(torch.int32)
    return bits.reshape(rows, groups * 8)[:, :cols]


def _blocks(x):
    """[rows, cols] -> [rows, blocks, 32], the last block filled up with zeros."""
    pad = -x.shape[1] % 32
    if pad:
        x = torch.nn.functional.pad(x, (0, pad))
    return x.reshape(x.shape[0], -1, 32)


def _codes(x, bits=None):
    """fp32 [rows, cols] (and random bits of the same shape) -> codes [rows, blocks, 32] and scale bytes [rows, blocks]."""
    x = _blocks(x)
    top = x.abs().amax(-1)
    pattern = top.view(torch.int32)
    scale = (((pattern if bits is None else pattern + 0x3FFFFF) >> 23) - 2).clamp_min(0)
    a = x.abs() * ((254 - scale) << 23).view(torch.float32).unsqueeze(-1)
    step = 0.5 + 0.5 * (a >= 2) + (a >= 4)
    if bits is None:
        q = torch.round(a / step)
    else:
        u = a / step
        low = torch.floor(u)
        q = low + (_blocks(bits) < torch.round((u - low) * 65536))
    q = torch.clamp_max(q * step, 6.0)
    code = (q * 2 - (q - 2).clamp_min(0) - (q > 4).float()).to(torch.uint8) | (torch.signbit(x).to(torch.uint8) << 3)
    bad = ~torch.isfinite(top)
    return torch.where(bad.unsqueeze(-1), 0, code), torch.where(bad, 255, scale).to(torch.uint8)


def _scale_values(scale):
    s = scale.to(torch.int32)
    v = torch.where(s == 0, 0x00400000, s << 23).view(torch.float32)      # byte 0 is 2^-127, a subnormal number
    return torch.where(s == 255, float("nan"), v)


def _values(code, scale, cols):
    """Codes [rows, blocks, 32] and scale bytes -> fp32 [rows, cols]."""
    table = torch.tensor(_E2M1, device=code.device)
    v = table[code.int()] * _scale_values(scale).unsqueeze(-1)
    return v.reshape(v.shape[0], -1)[:, :cols]


def _rounded(x, bits=None):
    """What x stands for after quantisation along its rows, fp32."""
    x = x.float()
    return _values(*_codes(x, bits), x.shape[1])


def _pack(code, scale, tiles=True):
    """Bytes as they lie in memory: two codes in a byte; scales in tiles of 128 rows x 4 blocks, or row after row."""
    rows = code.shape[0]
    flat = code.reshape(rows, -1)
    codes = flat[:, 0::2] | (flat[:, 1::2] << 4)
    if not tiles:
        scales = torch.nn.functional.pad(scale, (0, -scale.shape[1] % 16))
    else:
        s = torch.nn.functional.pad(scale, (0, -scale.shape[1] % 4, 0, -rows % 128))
        s = s.reshape(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4)
        scales = s.reshape(s.shape[0], -1)
    return codes.contiguous(), scales.contiguous()


def _unpack(codes, scales, rows, cols, tiles=True):
    """fp32 [rows, cols] from the bytes in memory."""
    blocks = (cols + 31) // 32
    code = torch.stack((codes & 15, codes >> 4), -1).reshape(rows, blocks, 32)
    if tiles:
        s = scales.reshape(scales.shape[0], -1, 32, 4, 4).permute(0, 3, 2, 1, 4)
        scales = s.reshape(s.shape[0] * 128, -1)
    return _values(code, scales[:rows, :blocks], cols)


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(c * (g + b * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * b * g * g)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, rows, cols, dtype=torch.bfloat16):
    """Normal values whose channels differ in size, some by a lot."""
    spread = torch.exp(torch.randn(cols, generator=g, device="cuda"))
    return (torch.randn(rows, cols, generator=g, device="cuda") * spread).to(dtype)


def _gradients(g, rows, cols, dtype, scale):
    """Heavy-tailed: magnitudes of a power law with density exponent 3, random signs."""
    u = torch.rand(rows, cols, generator=g, device="cuda")
    x = scale * (torch.rsqrt(1 - u) - 1)
    return torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.5, -x, x).to(dtype)


def _weights(g, rows, cols):
    return torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) & 0xFFFFFFFFFFFFFFFF}
    if kind == "quantize":
        dt = _DT[case["dtype"]]
        make = _activations if case["rounding"] == "nearest" else lambda *a: _gradients(*a, 1e-3)
        s["x"] = make(g, case["rows"], case["cols"], dt)
    elif kind in ("round", "server"):
        # rows start on a 32-byte boundary, as the gradient calls want them
        n, d = case["workers"], case["d"]
        x = torch.zeros(n, (d + 15) // 16 * 16, dtype=_DT[case["dtype"]], device="cuda")
        for i in range(n):
            x[i, :d] = _gradients(g, 1, d, _DT[case["dtype"]], 5e-4)[0]
        s["x"] = x
        if kind == "server":
            parts = [_pack(*_codes(x[i:i + 1, :d].float()), tiles=False) for i in range(n)]
            s["codes"], s["scales"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
            del s["x"]
    elif kind == "product":
        s["a"] = _pack(*_codes(_activations(g, case["m"], case["k"]).float()))
        s["b"] = _pack(*_codes(_weights(g, case["n"], case["k"])))
    else:
        t, d, f = case["tokens"], case["d"], case["f"]
        wg, wu, wd = _weights(g, f, d), _weights(g, f, d), _weights(g, d, f)
        if kind == "gated":
            s["x"] = torch.randn(t, d, generator=g, device="cuda").bfloat16()
            s["wg"], s["wu"], s["wd"] = (_pack(*_codes(w)) for w in (wg, wu, wd))
        else:
            s["dy"] = _gradients(g, t, d, torch.bfloat16, 1e-3)
            s["gu"] = torch.randn(t, 2 * f, generator=g, device="cuda").bfloat16()
            x = torch.randn(t, d, generator=g, device="cuda")
            s["x_t"] = _pack(*_codes(x.t()))
            s["w_t"] = _pack(*_codes(torch.cat((wg, wu)).t()))
            s["wd_t"] = _pack(*_codes(wd.t()))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "quantize":
        x = s["x"].float()
        bits = _philox16(s["seed"], *x.shape, x.device) if c["rounding"] == "stochastic" else None
        out = [_rounded(x, bits).bfloat16()]
        if c["both"]:
            out.append(_rounded(x.t(), bits.t() if bits is not None else None).bfloat16())
        return out
    if kind == "round":
        n, d = c["workers"], c["d"]
        return _rounded(s["x"][:, :d], _philox16(s["seed"], n, d, s["x"].device)).sum(0) / n
    if kind == "server":
        return _unpack(s["codes"], s["scales"], c["workers"], c["d"], tiles=False).sum(0) / c["workers"]
    if kind == "product":
        return (_unpack(*s["a"], c["m"], c["k"]) @ _unpack(*s["b"], c["n"], c["k"]).t()).to(_DT[c["out"]])
    t, d, f = c["tokens"], c["d"], c["f"]
    if kind == "gated":
        x = _rounded(s["x"])
        g, u = x @ _unpack(*s["wg"], f, d).t(), x @ _unpack(*s["wu"], f, d).t()
        h = _rounded(_act(g, c["act"])[0] * u)
        y = (h @ _unpack(*s["wd"], d, f).t()).bfloat16()
        return [y, torch.cat((g, u), 1).bfloat16()] if c["save"] else [y]
    seed = s["seed"]
    dy = s["dy"].float()
    bits = _philox16(seed, t, d, dy.device)
    dh = (_rounded(dy, bits) @ _unpack(*s["wd_t"], f, d).t()).bfloat16().float()
    gu = s["gu"].float()
    a, da = _act(gu[:, :f], c["act"])
    h, dgu = a * gu[:, f:], torch.cat((dh * gu[:, f:] * da, dh * a), 1)
    more = _philox16(seed + 1, t, 2 * f, dy.device)
    dx = _rounded(dgu, more) @ _unpack(*s["w_t"], d, 2 * f).t()
    dw = _rounded(dgu.t(), more.t()) @ _unpack(*s["x_t"], d, t).t()
    dwd = _rounded(dy.t(), bits.t()) @ _rounded(h.t()).t()
    return [dx.bfloat16(), dw.bfloat16(), dwd.bfloat16()]


def _run_own(s):
    from paper_2402_01798_b200 import binding as tq
    c = s["case"]
    kind = c["kind"]
    if kind == "quantize":
        rounding = tq.MX_STOCHASTIC if c["rounding"] == "stochastic" else tq.MX_NEAREST
        if not c["both"]:
            return [tq.tq_mx_dequantize(tq.tq_mx_quantize(s["x"], rounding, s["seed"]), torch.bfloat16)]
        q, q_t = tq.tq_mx_quantize_both(s["x"], rounding, s["seed"])
        return [tq.tq_mx_dequantize(q, torch.bfloat16), tq.tq_mx_dequantize(q_t, torch.bfloat16)]
    if kind == "round":
        q = tq.tq_mx_quantize(s["x"], tq.MX_STOCHASTIC, s["seed"], cols=c["d"], layout=tq.MX_ROWS)
        return tq.tq_mx_decompress_aggregate(q)
    if kind == "server":
        return tq.tq_mx_decompress_aggregate(tq.MxMatrix(s["codes"], s["scales"], c["workers"], c["d"], tq.MX_ROWS))
    if kind == "product":
        return tq.tq_mx_product(tq.MxMatrix(*s["a"], c["m"], c["k"]), tq.MxMatrix(*s["b"], c["n"], c["k"]), _DT[c["out"]])
    t, d, f = c["tokens"], c["d"], c["f"]
    act = tq.MX_SILU if c["act"] == "silu" else tq.MX_GELU
    if kind == "gated":
        x = tq.tq_mx_quantize(s["x"])
        gu = torch.empty(t, 2 * f, dtype=torch.bfloat16, device=s["x"].device) if c["save"] else None
        h = tq.tq_mx_gated(x, tq.MxMatrix(*s["wg"], f, d), tq.MxMatrix(*s["wu"], f, d), act, projections=gu)
        y = tq.tq_mx_product(h, tq.MxMatrix(*s["wd"], d, f), torch.bfloat16)
        return [y, gu] if c["save"] else [y]
    seed = s["seed"]
    dy, dy_t = tq.tq_mx_quantize_both(s["dy"], tq.MX_STOCHASTIC, seed)
    dh = tq.tq_mx_product(dy, tq.MxMatrix(*s["wd_t"], f, d), torch.bfloat16)
    dgu, dgu_t, h_t = tq.tq_mx_gated_backward(dh, s["gu"], act, tq.MX_STOCHASTIC, seed + 1)
    dx = tq.tq_mx_product(dgu, tq.MxMatrix(*s["w_t"], d, 2 * f), torch.bfloat16)
    dw = tq.tq_mx_product(dgu_t, tq.MxMatrix(*s["x_t"], d, t), torch.bfloat16)
    dwd = tq.tq_mx_product(dy_t, h_t, torch.bfloat16)
    return [dx, dw, dwd]


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case):
    """Bytes: inputs, outputs and the 4.25-bit copies in between, each once.  FLOPs: two for each term of a product."""
    kind, mx = case["kind"], 4.25 / 8
    if kind == "quantize":
        n, copies = case["rows"] * case["cols"], 2 if case["both"] else 1
        return {"bytes": n * ((2 if case["dtype"] == "bfloat16" else 4) + copies * (2 * mx + 2)), "flops": 0}
    if kind in ("round", "server"):
        n, d = case["workers"], case["d"]
        size = 2 if case["dtype"] == "bfloat16" else 4
        return {"bytes": n * d * ((size + 2 * mx) if kind == "round" else mx) + 4 * d, "flops": 0}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * k * mx + m * n * (2 if case["out"] == "bfloat16" else 4), "flops": 2 * m * n * k}
    t, d, f = case["tokens"], case["d"], case["f"]
    if kind == "gated":
        return {"bytes": t * d * (2 + 2 * mx) + 3 * d * f * mx + t * f * (2 * mx + (4 if case["save"] else 0)) + t * d * 2,
                "flops": 6 * t * d * f}
    return {"bytes": t * d * (2 + 4 * mx) + 3 * d * f * mx + t * f * (2 + 2 + 4) + t * f * 5 * 2 * mx + t * d * (mx + 2) + 3 * d * f * 2,
            "flops": 12 * t * d * f}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _random64(seed, rows, cols):
    """The same 16 random bits: Philox4x32-10 as published, counter (group, 0, row, 0), 32-bit words as int64 halves of products."""
    def mulhilo(a, b):          # by 16-bit parts, so that nothing leaves 63 bits
        al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = ah * bl + ((al * bl) >> 16)
        mid2 = al * bh + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((al * bl) & 0xFFFF)

    groups = -(-cols // 8)
    c = [torch.arange(groups, device="cuda").repeat(rows, 1), torch.zeros(rows, groups, dtype=torch.int64, device="cuda"),
         torch.arange(rows, device="cuda").unsqueeze(1).repeat(1, groups), torch.zeros(rows, groups, dtype=torch.int64, device="cuda")]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for r in range(10):
        hi0, lo0 = mulhilo(c[0], 0xD2511F53)
        hi1, lo1 = mulhilo(c[2], 0xCD9E8D57)
        c = [hi1 ^ c[1] ^ key[0], lo1, hi0 ^ c[3] ^ key[1], lo0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = torch.empty(rows, groups, 8, dtype=torch.float64, device="cuda")
    for w in range(4):
        out[..., 2 * w], out[..., 2 * w + 1] = (c[w] % 65536).double(), (c[w] // 65536).double()
    return out.reshape(rows, -1)[:, :cols]


def _mx64(x, random=None):
    """Values after quantisation of a finite matrix along its rows, by search in the grid of magnitudes."""
    rows, cols = x.shape
    wide = -(-cols // 32) * 32
    v = torch.zeros(rows, wide, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, wide // 32, 32)
    top = v.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)                               # top = mantissa 2^exponent, mantissa in [1/2, 1)
    e = exponent - 3 if random is None else exponent - 3 + (mantissa > 0.75)
    e = torch.where(top > 0, e, -127).clamp_min(-127)
    scale = torch.ldexp(torch.ones_like(top), e)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    a = (v.abs() / scale).clamp_max(6.0)
    lower = (torch.searchsorted(grid, a, right=True) - 1).clamp(0, 6)
    low, high = grid[lower], grid[lower + 1]
    p = (a - low) / (high - low)
    if random is None:
        up = (p > 0.5) | ((p == 0.5) & (lower % 2 == 1))
    else:
        r = torch.zeros(rows, wide, dtype=torch.float64, device=x.device)
        r[:, :cols] = random
        up = r.view_as(v) < torch.round(p * 65536)
    return (torch.where(up, high, low) * torch.sign(v) * scale).view(rows, wide)[:, :cols]


def _held64(held, rows, cols, tiled=True):
    """The matrix that bytes in memory stand for: every byte's place from the layout's own index formula."""
    codes, scales = held
    j = torch.arange(cols, device="cuda")
    i = torch.arange(rows, device="cuda").unsqueeze(1)
    nibble = (codes[:, j // 2] >> (j % 2 * 4).to(torch.uint8)) & 15
    grid = torch.tensor(_GRID, dtype=torch.float64, device="cuda")
    b = j // 32
    if tiled:
        at = (i // 128) * scales.shape[1] + (b // 4) * 512 + (i % 32) * 16 + (i // 32 % 4) * 4 + b % 4
    else:
        at = i * scales.shape[1] + b
    s = scales.reshape(-1)[at].double()
    return grid[(nibble & 7).long()] * (1 - 2 * (nibble >> 3).double()) * torch.exp2(s - 127)


def _act64(g, act):
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig + g * sig * (1 - sig)
    c = math.sqrt(2 / math.pi)
    inner = c * (g + 0.044715 * g ** 3)
    sig = 1 / (1 + torch.exp(-2 * inner))
    return g * sig, sig + g * 2 * sig * (1 - sig) * c * (1 + 3 * 0.044715 * g ** 2)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "quantize":
        x = s["x"].double()
        r = _random64(s["seed"], *x.shape) if case["rounding"] == "stochastic" else None
        out = [_mx64(x, r)]
        if case["both"]:
            out.append(_mx64(x.t(), None if r is None else r.t()))
        return out
    if kind in ("round", "server"):
        n, d = case["workers"], case["d"]
        total = torch.zeros(d, dtype=torch.float64, device="cuda")
        for i in range(n):
            if kind == "server":
                total += _held64((s["codes"][i:i + 1], s["scales"][i:i + 1]), 1, d, tiled=False)[0]
                continue
            # row i's random bits alone
            total += _mx64(s["x"][i:i + 1, :d].double(), _random64_row(s["seed"], i, d))[0]
        return total / n
    if kind == "product":
        return _held64(s["a"], case["m"], case["k"]) @ _held64(s["b"], case["n"], case["k"]).t()
    t, d, f, act = case["tokens"], case["d"], case["f"], case["act"]
    if kind == "gated":
        x = _mx64(s["x"].double())
        g, u = x @ _held64(s["wg"], f, d).t(), x @ _held64(s["wu"], f, d).t()
        y = _mx64(_act64(g, act)[0] * u) @ _held64(s["wd"], d, f).t()
        return [y, torch.cat((g, u), 1)] if case["save"] else [y]
    dy, gu = s["dy"].double(), s["gu"].double()
    r = _random64(s["seed"], t, d)
    # dh is handed over in bf16: that rounding belongs to the definition
    dh = (_mx64(dy, r) @ _held64(s["wd_t"], f, d).t()).float().bfloat16().double()
    a, da = _act64(gu[:, :f], act)
    dgu = torch.cat((dh * gu[:, f:] * da, dh * a), 1)
    r2 = _random64(s["seed"] + 1, t, 2 * f)
    dx = _mx64(dgu, r2) @ _held64(s["w_t"], d, 2 * f).t()
    dw = _mx64(dgu.t(), r2.t()) @ _held64(s["x_t"], d, t).t()
    return [dx, dw, _mx64(dy.t(), r.t()) @ _mx64((a * gu[:, f:]).t()).t()]


def _random64_row(seed, row, cols):
    """One row's bits, from the same counter scheme, in pieces that keep memory small."""
    part = 1 << 24
    out = torch.empty(1, cols, dtype=torch.float64, device="cuda")
    for at in range(0, cols, part):
        n = min(part, cols - at)
        out[0, at:at + n] = _row_piece(seed, row, at // 8, n)
    return out


def _row_piece(seed, row, group0, n):
    m0, m1 = 0xD2511F53, 0xCD9E8D57
    groups = -(-n // 8)
    a = torch.arange(group0, group0 + groups, device="cuda")
    b, c, d = torch.zeros_like(a), torch.full_like(a, row), torch.zeros_like(a)
    k = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]

    def high_low(x, m):
        low_part = x * (m % 65536)                                       # below 2^48
        high_part = x * (m // 65536) + low_part // 65536                 # below 2^49
        return high_part // 65536, high_part % 65536 * 65536 + low_part % 65536

    for _ in range(10):
        h0, l0 = high_low(a, m0)
        h1, l1 = high_low(c, m1)
        a, b, c, d = h1 ^ b ^ k[0], l1, h0 ^ d ^ k[1], l0
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    w = torch.stack((a, b, c, d), 1)
    return torch.stack((w % 65536, w // 65536), 2).reshape(-1)[:n].double()
