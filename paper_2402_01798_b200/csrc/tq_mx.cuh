// Microscaled 4-bit floating point on the device: scales, codes and where they lie (format: include/tq.h).
#pragma once
#include "tq_device.cuh"

namespace tq {

// One MX matrix as a kernel sees it.
struct MxView {
    uint8_t* codes;
    uint8_t* scales;
    uint64_t rows, cols, code_stride, scale_stride;
    uint32_t tiles;                // layout of the scales: 1 tiles, 0 row after row
};
inline MxView mx_view(const tq_mx_t& m) {
    return MxView{m.codes, m.scales, m.rows, m.cols, m.code_stride, m.scale_stride, m.layout == TQ_MX_TILES};
}
__host__ __device__ __forceinline__ uint64_t mx_blocks(uint64_t cols) { return (cols + 31) / 32; }
__device__ __forceinline__ uint64_t mx_scale_at(const MxView& m, uint64_t row, uint64_t block) {
    if (!m.tiles) return row * m.scale_stride + block;
    return (row >> 7) * m.scale_stride + (block >> 2) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

constexpr uint32_t kInfBits = 0x7F800000u;

// max(|a|, |b|, |c|), NaN if one is
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
    float r; asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r;
}
__device__ __forceinline__ float max_abs_32(const float (&v)[32]) {
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = max_abs3(v[4 * i], v[4 * i + 1], v[4 * i + 2]);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = max_abs3(m[i], m[i + 4], v[4 * i + 3]);
    m[0] = max_abs3(m[0], v[19], v[23]);
    m[1] = max_abs3(m[1], v[27], v[31]);
    m[2] = max_abs3(m[2], m[3], m[0]);
    return max_abs3(m[1], m[2], 0.0f);
}

// The scale byte of a block whose largest magnitude is `top`; 255 where the block holds a NaN or an infinity.
//   nearest:    2^(floor(log2 top) - 2): top / scale lies in [4, 8), what exceeds 6 is rounded to 6;
//   stochastic: the smallest power of two with top <= 6 scale, so that nothing is cut off and the expectation is the element.
//               With top = m 2^e that is e - 2 for m <= 3/2 and e - 1 above: the carry of 0x3FFFFF into the exponent.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t mx_scale_byte(float top) {
    const uint32_t p = __float_as_uint(top);
    const int e = static_cast<int>((STOCHASTIC ? p + 0x3FFFFFu : p) >> 23) - 2;
    return p >= kInfBits ? 255u : static_cast<uint32_t>(e > 0 ? e : 0);
}
// 1 / scale, exact: 2^(127 - byte), a normal number for every byte that mx_scale_byte gives a finite block (0 .. 253)
__device__ __forceinline__ float mx_inv_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Eight scaled elements -> eight codes, to nearest, ties to the even code, 6 at most; the sign of a zero stays.
__device__ __forceinline__ uint32_t e2m1_nearest8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// Stochastic rounding of scaled magnitudes a <= 6.  On the grid's own scale, where neighbours are one apart, a lies at
//     F(a) = 2a (a < 2),  a + 2 (2 <= a < 4),  a / 2 + 4 (4 <= a)  =  min(2a, a + 2, a / 2 + 4),
// the code below it being floor F(a) and p the rest.  P = rint(2^16 F(a)) is the smallest of three fused multiply-adds onto a magic number (the
// products are exact, each is rounded once to an integer, 2^17 and 2^18 are even, and rounding keeps the order).  The code is
// (P + 65535 - r) >> 16, one up when r < rint(p 2^16): byte 2 of the sum.  (By the exponent of a it takes four operations of the integer pipe, here one: rows
// of 8192 x 4096 bf16 30 -> 27 us; with three scalar multiply-adds an element instead of half as many packed ones 1 us more.)
__device__ __forceinline__ float min3(float a, float b, float c) { float r; asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// Byte 3 of four words.
__device__ __forceinline__ uint32_t byte3_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073u), __byte_perm(c, d, 0x0073u), 0x5410u);
}
// Where the inverted bits of an element are: in which word, and in which half of it (0x0001 the lower, 0x0100 the upper one).
struct RowBits {                   // of 8 neighbours, two in a word
    uint32_t w[4];
    __device__ __forceinline__ uint32_t word(int e) const { return w[e >> 1]; }
    __device__ __forceinline__ uint32_t half(int e) const { return e & 1 ? 0x0100u : 0x0001u; }
};
struct ColumnBits {                // of 8 elements in a column, each beside that of the next or last column
    uint32_t w[8], side;
    __device__ __forceinline__ uint32_t word(int e) const { return w[e]; }
    __device__ __forceinline__ uint32_t half(int) const { return side; }
};
// Eight elements x, to be scaled by `inv`.
template <class Bits>
__device__ __forceinline__ uint32_t e2m1_stochastic8(const float* x, float inv, const Bits& bits) {
    uint32_t s[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 a = pair(fabsf(x[2 * i]) * inv, fabsf(x[2 * i + 1]) * inv);
        float l[3], h[3];
        unpair(fma2(a, both(131072.0f), both(kMagic)), l[0], h[0]);
        unpair(fma2(a, both(65536.0f), both(kMagic + 131072.0f)), l[1], h[1]);
        unpair(fma2(a, both(32768.0f), both(kMagic + 262144.0f)), l[2], h[2]);
        s[2 * i] = dot_halves(bits.word(2 * i), bits.half(2 * i), __float_as_uint(min3(l[0], l[1], l[2])));
        s[2 * i + 1] = dot_halves(bits.word(2 * i + 1), bits.half(2 * i + 1), __float_as_uint(min3(h[0], h[1], h[2])));
    }
    const uint32_t even = byte3_of(__float_as_uint(x[0]), __float_as_uint(x[2]), __float_as_uint(x[4]), __float_as_uint(x[6]));
    const uint32_t odd = byte3_of(__float_as_uint(x[1]), __float_as_uint(x[3]), __float_as_uint(x[5]), __float_as_uint(x[7]));
    return pack_byte2<4>(s) | ((even >> 4) & 0x08080808u) | (odd & 0x80808080u);
}

// Eight codes -> fp32, before the scale.
__device__ __forceinline__ void e2m1_values8(uint32_t codes, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "r"(h[i]));
}

// Random bits of the elements (row, 8 * group .. 8 * group + 7), inverted: word i holds those of elements 2i (low half) and 2i + 1.
// `run` belongs to the row and the group's upper half.
__device__ __forceinline__ void mx_random8(const PhiloxRun& run, uint64_t group, const RoundKeys& keys, RowBits& out) {
    philox_block(static_cast<uint32_t>(group), run, keys, out.w);
#pragma unroll
    for (int i = 0; i < 4; ++i) out.w[i] = ~out.w[i];
}

// 32 elements -> their 32 codes, element 0 in the lowest nibble.  `random(q)` gives the bits of elements 8q .. 8q + 7 (RowBits or
// ColumnBits); it is not called for nearest rounding.
template <bool STOCHASTIC, class Random>
__device__ __forceinline__ uint4 mx_encode32(const float (&v)[32], uint32_t byte, Random random) {
    uint32_t w[4];
    const float inv = mx_inv_scale(byte);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (STOCHASTIC) {
            w[q] = e2m1_stochastic8(&v[8 * q], inv, random(q));
        } else {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; e += 2) unpair(mul2(pair(v[8 * q + e], v[8 * q + e + 1]), both(inv)), y[e], y[e + 1]);
            w[q] = e2m1_nearest8(y);
        }
        w[q] = byte == 255u ? 0u : w[q];
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r;
}
__device__ __forceinline__ void stg128(void* p, uint4 v) {
    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void stg256_words(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                 :: "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "l"(p) : "memory");
}
__device__ __forceinline__ uint4 ldg128(const void* p) {
    uint4 v; asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory"); return v;
}
__device__ __forceinline__ void ldg256(const void* p, uint32_t (&v)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ uint32_t ldg8(const void* p) {
    uint32_t v; asm volatile("ld.global.b8 %0, [%1];" : "=r"(v) : "l"(p) : "memory"); return v;
}

// ---- activations of the gated block ------------------------------------------------------------------------
// x * s with s = sigmoid(z): SiLU has z = x, the tanh form of GELU z = 2 sqrt(2/pi) (x + 0.044715 x^3), since
// (1 + tanh t) / 2 = sigmoid(2 t).
// With h = exp(-|z| / 2), r = 1 / (1 + h^2), s is h^2 r below zero and r above, and 1 - s the other one.  The products take one h after the
// other, so that no factor is subnormal before the product is: x s is a normal number down to x = -92, where exp(x) has not been one since -87.3.
// Errors, relative: expf 2 ulp, rcp.approx 1 ulp, so that x s is off by less than 2^-20; GELU's z, six roundings, adds 6 |z| 2^-24 below zero.
constexpr float kGeluC = 1.5957691216057308f;      // 2 sqrt(2/pi)
constexpr float kGeluB = 0.044715f;
struct GateParts {
    float h, r, a;                 // a: h below zero, 1 above: s = a (a r)
};
template <bool GELU>
__device__ __forceinline__ GateParts gate_parts(float x) {
    float z = x;
    if constexpr (GELU) z = kGeluC * x * fmaf(kGeluB * x, x, 1.0f);
    GateParts p;
    p.h = expf(-0.5f * fabsf(z));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p.r) : "f"(fmaf(p.h, p.h, 1.0f)));       // of a number from 1 to 2
    p.a = z < 0.0f ? p.h : 1.0f;
    return p;
}
template <bool GELU>
__device__ __forceinline__ float gate_value(float x) {
    const GateParts p = gate_parts<GELU>(x);
    return (x * p.a) * (p.a * p.r);
}
// value and derivative: s + x z' s (1 - s)
template <bool GELU>
__device__ __forceinline__ void gate_value_slope(float x, float& value, float& slope) {
    const GateParts p = gate_parts<GELU>(x);
    const float s = p.a * (p.a * p.r);
    float t = x * p.h;
    if constexpr (GELU) t *= fminf(kGeluC * fmaf(3.0f * kGeluB * x, x, 1.0f), 1e30f);    // where it would overflow, h is 0
    value = (x * p.a) * (p.a * p.r);
    slope = fmaf(t, p.h * p.r * p.r, s);
}

}  // namespace tq
