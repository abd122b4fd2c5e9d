"""Microscaled 4-bit floating point in 64 bits, from its definition: what the GPU tests compare with (no torch, no GPU)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TILES, ROWS = 0, 1


def random16(seed, rows, cols, first_row=0):
    """Philox4x32-10 (Salmon et al., SC'11), key = seed, counter = (c >> 3, first_row + r, 0), 16 bits in slot c & 7."""
    groups = -(-cols // 8)
    m = np.uint64(0xFFFFFFFF)
    g = np.arange(groups, dtype=np.uint64)
    c = [np.broadcast_to(g & m, (rows, groups)), np.broadcast_to(g >> np.uint64(32), (rows, groups)),
         np.broadcast_to(((np.uint64(first_row) + np.arange(rows, dtype=np.uint64)) & m)[:, None], (rows, groups)), np.zeros((rows, groups), np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack(c, -1)
    return np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), -1).reshape(rows, -1)[:, :cols].astype(np.int64)


def blocks_of(x, fill=0):
    rows, cols = x.shape
    out = np.full((rows, -(-cols // 32) * 32), fill, x.dtype)
    out[:, :cols] = x
    return out.reshape(rows, -1, 32)


def scale_byte(top, stochastic):
    """The scale bytes for blocks of largest magnitude `top` (fp64; NaN and infinity give 255)."""
    good = np.isfinite(top) & (top > 0)
    mantissa, e = np.frexp(np.where(good, top, 1.0))                # mantissa in [1/2, 1)
    e = e - 3 + ((mantissa > 0.75) if stochastic else 0)
    return np.where(np.isfinite(top), np.where(top > 0, np.maximum(e + 127, 0), 0), 255).astype(np.int64)


def codes_at(x, byte, random=None):
    """Codes of blocks x [.., 32] at given scale bytes [..]; monotone in x."""
    scale = np.ldexp(1.0, np.minimum(byte, 254) - 127)[..., None]
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)) / scale, 6.0)
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    p = (a - GRID[low]) / (GRID[low + 1] - GRID[low])
    up = (p > 0.5) | ((p == 0.5) & (low % 2 == 1)) if random is None else random < np.rint(p * 65536)
    code = low + up + 8 * np.signbit(x)
    return np.where(byte[..., None] == 255, 0, code)


def quantize(x, random=None):
    """fp64 [rows, cols] -> codes [rows, blocks, 32], scale bytes [rows, blocks]."""
    x = blocks_of(np.asarray(x, np.float64))
    with np.errstate(invalid="ignore"):
        byte = scale_byte(np.abs(x).max(-1), random is not None)
    return codes_at(x, byte, None if random is None else blocks_of(random)), byte


def decode(code, byte, cols):
    scale = np.where(byte == 255, np.nan, np.ldexp(1.0, np.minimum(byte, 254) - 127))
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * scale[..., None]
    return v.reshape(v.shape[0], -1)[:, :cols]


def scale_index(rows, blocks, layout, stride):
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    if layout == ROWS:
        return r * stride + b
    return r // 128 * stride + b // 4 * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4


def held(codes, scales, rows, cols, layout):
    """Codes [rows, blocks, 32] and scale bytes [rows, blocks] from the bytes in memory (2-d uint8 arrays as the binding keeps them)."""
    blocks = -(-cols // 32)
    c = codes[:rows, :16 * blocks].astype(np.int64)
    code = np.stack((c & 15, c >> 4), -1).reshape(rows, blocks, 32)
    return code, scales.reshape(-1)[scale_index(rows, blocks, layout, scales.shape[1])].astype(np.int64)


def activation(g, kind):
    """Value, derivative, and the size of the derivative's terms."""
    if kind == "silu":
        z, dz = g, np.ones_like(g)
    else:
        c = 2 * np.sqrt(2 / np.pi)
        z, dz = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g ** 2)
    s = 1 / (1 + np.exp(-z))
    v = g * s
    return v, s + v * (1 - s) * dz, s + np.abs(v * (1 - s) * dz)
