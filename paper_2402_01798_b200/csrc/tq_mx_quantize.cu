// Microscaled 4-bit floating point: quantisation along one or both axes, decoding, the mean of decoded rows, and the backward
// pass of the gated block's activation, which ends in three quantised matrices.
#include "tq_mx.cuh"

namespace tq {

namespace {

struct MxInput {
    const void* data;
    uint64_t stride;               // elements from row to row
    uint32_t wide;                 // 1: every row starts on a 16-byte boundary
};

// ---- along the rows ----------------------------------------------------------------------------------------
// One thread makes one block: 64 or 128 bytes in, 16 bytes of codes and a byte of scale out, no exchange between threads.
// A block of 256 threads covers 2^shift MX blocks of 256 >> shift rows.  Bound by memory where rounding is to nearest.
template <bool BF16, bool STOCHASTIC>
__global__ void __launch_bounds__(kThreads) mx_rows_kernel(MxInput in, MxView out, uint32_t shift, uint64_t col_groups, RoundKeys keys, uint32_t first_row) {
    pdl_wait();
    const uint64_t row = (blockIdx.x / col_groups) * (kThreads >> shift) + (threadIdx.x >> shift);
    const uint64_t block = (blockIdx.x % col_groups << shift) + (threadIdx.x & ((1u << shift) - 1));
    const uint64_t blocks = mx_blocks(out.cols);
    if (row >= out.rows || block >= blocks) {
        // the tile layout is filled up to whole tiles
        if (out.tiles && row < (out.rows + 127) / 128 * 128 && block < (blocks + 3) / 4 * 4) out.scales[mx_scale_at(out, row, block)] = 0;
        return;
    }
    const char* src = static_cast<const char*>(in.data) + (row * in.stride + block * 32) * (BF16 ? 2 : 4);
    float v[32];
    if (block * 32 + 32 <= out.cols) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
            const uint4 w = ldg128(src + 16 * i);
            if constexpr (BF16) {
                const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) { v[8 * i + 2 * k] = __uint_as_float(x[k] << 16); v[8 * i + 2 * k + 1] = __uint_as_float(x[k] & 0xFFFF0000u); }
            } else {
                v[4 * i] = __uint_as_float(w.x); v[4 * i + 1] = __uint_as_float(w.y); v[4 * i + 2] = __uint_as_float(w.z); v[4 * i + 3] = __uint_as_float(w.w);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = block * 32 + i < out.cols ? load1<BF16>(src, i) : 0.0f;
    }
    const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
    const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q, uint32_t (&r)[4]) { mx_random8(first_row + static_cast<uint32_t>(row), block * 4 + q, keys, r); });
    stg128(out.codes + row * out.code_stride + block * 16, codes);
    out.scales[mx_scale_at(out, row, block)] = static_cast<uint8_t>(byte);
}

// ---- tiles in shared memory ------------------------------------------------------------------------------------
// 128 x 128 elements in fp32.  32 elements are followed by 4 words of padding: a thread that reads 32 elements of a row in
// 16-byte steps then meets no other thread of its quarter warp in a bank, and neither do 32 threads that read down 32 columns.
constexpr int kTile = 128;
constexpr int kTilePitch = 4 * 36;
struct MxTile {
    float v[kTile * kTilePitch];
    uint32_t random[kTile * 64];           // 16 bits an element, in 16-byte chunks of 8; see random_chunk
};
__device__ __forceinline__ int tile_at(int r, int c) { return r * kTilePitch + (c >> 5) * 36 + (c & 31); }
// Word of the 16-byte chunk with the bits of row r, columns 8g .. 8g + 7.  The exchange of chunks keeps eight threads that write (two rows,
// four blocks) in different banks.
__device__ __forceinline__ int random_chunk(int r, int g) { return r * 64 + ((g ^ ((g >> 3) | ((r & 1) << 1))) << 2); }

// Codes and scales of the tile's rows: rows r0 .., columns c0 .. of the matrix `out`, both multiples of 32; `width` columns of the tile count
// and `height` rows.  `fill`: the tile ends the matrix on the right, and its row of scales is filled up with zeros.
template <bool STOCHASTIC, bool KEEP>
__device__ __forceinline__ void tile_rows(MxTile& t, const MxView& out, uint64_t r0, uint64_t c0, int height, int width, bool fill, const RoundKeys& keys,
                                          uint32_t first_row, uint64_t random_c0) {
    const uint64_t blocks = mx_blocks(out.cols);
    for (int item = threadIdx.x; item < kTile * 4; item += blockDim.x) {
        const int r = item >> 2, b = item & 3;
        const uint64_t block = c0 / 32 + b;
        const bool inside = r < height && b * 32 < width;
        float v[32];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 x = *reinterpret_cast<const float4*>(&t.v[tile_at(r, b * 32 + 4 * i)]);
            v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
        }
        const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
        const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q, uint32_t (&w)[4]) {
            mx_random8(first_row + static_cast<uint32_t>(r0) + r, (random_c0 >> 3) + b * 4 + q, keys, w);
            if constexpr (KEEP) *reinterpret_cast<uint4*>(&t.random[random_chunk(r, b * 4 + q)]) = make_uint4(w[0], w[1], w[2], w[3]);
        });
        if (inside) {
            stg128(out.codes + (r0 + r) * out.code_stride + block * 16, codes);
            out.scales[mx_scale_at(out, r0 + r, block)] = static_cast<uint8_t>(byte);
        } else if (out.tiles && (b * 32 < width || (fill && block < (blocks + 3) / 4 * 4))) {
            out.scales[mx_scale_at(out, r0 + r, block)] = 0;
        }
    }
}

// The same along the columns: the tile's column c becomes row q0 + c of `out`, whose blocks run over the tile's rows from r0 on.
// `fill`: the tile ends `out` below, and the rest of its last 128 rows gets zero scales.
template <bool STOCHASTIC>
__device__ __forceinline__ void tile_cols(const MxTile& t, const MxView& out, uint64_t q0, uint64_t r0, int height, int width, bool fill) {
    const uint64_t blocks = mx_blocks(out.cols);
    for (int item = threadIdx.x; item < kTile * 4; item += blockDim.x) {
        const int c = item & (kTile - 1), b = item >> 7;
        const uint64_t block = r0 / 32 + b, row = q0 + c;
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = t.v[tile_at(b * 32 + i, c)];
        const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
        const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q, uint32_t (&w)[4]) {
            const unsigned short* random = reinterpret_cast<const unsigned short*>(t.random);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = b * 32 + q * 8 + 2 * i;
                const uint32_t lo = random[2 * random_chunk(r, c >> 3) + (c & 7)], hi = random[2 * random_chunk(r + 1, c >> 3) + (c & 7)];
                w[i] = lo | (hi << 16);
            }
        });
        if (c < width && b * 32 < height) {
            stg128(out.codes + row * out.code_stride + block * 16, codes);
            out.scales[mx_scale_at(out, row, block)] = static_cast<uint8_t>(byte);
        } else if (out.tiles && block < (blocks + 3) / 4 * 4 && (c < width || (fill && row < (out.rows + 127) / 128 * 128))) {
            out.scales[mx_scale_at(out, row, block)] = 0;
        }
    }
}

// The tile's elements from memory, zeros outside.  `wide`: 16 bytes a thread at a time, consecutive threads in consecutive places; else one
// element, for rows on any boundary.
template <bool BF16>
__device__ __forceinline__ void load_tile(float* tile, const MxInput& in, uint64_t r0, uint64_t c0, int height, int width) {
    constexpr int kSize = BF16 ? 2 : 4, kPer = 16 / kSize, kLanes = kTile / kPer;      // threads in a row
    const char* base = static_cast<const char*>(in.data) + (r0 * in.stride + c0) * kSize;
    if (in.wide) {
        const int c = (threadIdx.x % kLanes) * kPer;
#pragma unroll 8
        for (int r = threadIdx.x / kLanes; r < kTile; r += kThreads / kLanes) {
            float x[kPer];
            const char* p = base + (static_cast<uint64_t>(r) * in.stride + c) * kSize;
            if (r < height && c + kPer <= width) {
                const uint4 w4 = ldg128(p);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (BF16) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
                    else x[k] = __uint_as_float(w[k]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kPer; ++k) x[k] = r < height && c + k < width ? load1<BF16>(p, k) : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kPer; k += 4) *reinterpret_cast<float4*>(&tile[tile_at(r, c + k)]) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
        }
    } else {
        const int c = threadIdx.x % kTile;
#pragma unroll 16
        for (int r = threadIdx.x / kTile; r < kTile; r += kThreads / kTile)
            tile[tile_at(r, c)] = r < height && c < width ? load1<BF16>(base, static_cast<uint64_t>(r) * in.stride + c) : 0.0f;
    }
}

template <bool BF16, bool STOCHASTIC, bool BOTH>
__global__ void __launch_bounds__(kThreads) mx_tile_kernel(MxInput in, MxView out, MxView out_t, uint32_t tiles_across, RoundKeys keys, uint32_t first_row) {
    extern __shared__ __align__(16) unsigned char raw[];
    MxTile& t = *reinterpret_cast<MxTile*>(raw);
    pdl_wait();
    const uint64_t r0 = static_cast<uint64_t>(blockIdx.x / tiles_across) * kTile, c0 = static_cast<uint64_t>(blockIdx.x % tiles_across) * kTile;
    const int height = static_cast<int>(out.rows - r0 < kTile ? out.rows - r0 : kTile), width = static_cast<int>(out.cols - c0 < kTile ? out.cols - c0 : kTile);
    load_tile<BF16>(t.v, in, r0, c0, height, width);
    __syncthreads();
    tile_rows<STOCHASTIC, BOTH>(t, out, r0, c0, height, width, true, keys, first_row, c0);
    if constexpr (BOTH) {
        if constexpr (STOCHASTIC) __syncthreads();
        tile_cols<STOCHASTIC>(t, out_t, c0, r0, height, width, true);
    }
}

// ---- decoding ----------------------------------------------------------------------------------------------------
// A thread makes 8 elements.  WIDE: it stores them in one piece; else the warp passes its codes around so that consecutive threads store
// consecutive elements, for rows on any boundary.
template <bool BF16, bool WIDE>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(MxView m, void* out, uint64_t stride, uint32_t chunks) {
    pdl_wait();
    const uint64_t row = blockIdx.x / chunks;
    const uint64_t first = (static_cast<uint64_t>(blockIdx.x % chunks) * kThreads + (threadIdx.x & ~31u)) * 8;      // the warp's first element
    if (first >= m.cols) return;
    const uint64_t col = first + (threadIdx.x & 31) * 8;
    const bool any = col < m.cols;
    uint32_t codes = 0, byte = 0;
    if (any) {
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(codes) : "l"(m.codes + row * m.code_stride + col / 2) : "memory");
        byte = ldg8(m.scales + mx_scale_at(m, row, col / 32));
    }
    const float scale = mx_scale_value(byte);
    char* const to = static_cast<char*>(out) + row * stride * (BF16 ? 2 : 4);
    if constexpr (WIDE) {
        if (!any) return;
        float v[8];
        e2m1_values8(codes, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        if (col + 8 <= m.cols) {
            if constexpr (BF16) {
                stg128(to + col * 2, make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
            } else {
                stg128(to + col * 4, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
                stg128(to + col * 4 + 16, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < m.cols) {
                    if constexpr (BF16) reinterpret_cast<unsigned short*>(to)[col + e] = static_cast<unsigned short>(__float_as_uint(v[e]) >> 16);   // exact
                    else reinterpret_cast<float*>(to)[col + e] = v[e];
                }
        }
    } else {
        const uint32_t lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = __shfl_sync(0xFFFFFFFFu, codes, 4 * i + lane / 8);
            const float s = __shfl_sync(0xFFFFFFFFu, scale, 4 * i + lane / 8);
            float v[8];
            e2m1_values8(w >> (4 * (lane & 7)), v);
            const uint64_t c = first + 32 * i + lane;
            if (c < m.cols) {
                if constexpr (BF16) reinterpret_cast<unsigned short*>(to)[c] = static_cast<unsigned short>(__float_as_uint(v[0] * s) >> 16);
                else reinterpret_cast<float*>(to)[c] = v[0] * s;
            }
        }
    }
}

// ---- mean of decoded rows --------------------------------------------------------------------------------------------
struct MxWeights {
    float w[TQ_MAX_WORKERS];
};
// A thread decodes the same block of 32 elements of every worker's row and keeps the 32 sums.  fp32, in worker order.
template <bool WEIGHTED>
__global__ void __launch_bounds__(kThreads) mx_aggregate_kernel(MxView m, float* out, uint32_t n, float divisor, MxWeights weights) {
    pdl_wait();
    const uint64_t block = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (block * 32 >= m.cols) return;
    float sum[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) sum[e] = 0.0f;
#pragma unroll 4
    for (uint32_t i = 0; i < n; ++i) {
        const uint4 c = ldg128(m.codes + i * m.code_stride + block * 16);
        const float scale = mx_scale_value(ldg8(m.scales + i * m.scale_stride + block));
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[8];
            e2m1_values8(w[q], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = v[e] * scale;
                sum[8 * q + e] += WEIGHTED ? x * weights.w[i] : x;
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = WEIGHTED ? sum[8 * q + e] : __fdiv_rn(sum[8 * q + e], divisor);
        const uint64_t col = block * 32 + 8 * q;
        if (col + 8 <= m.cols) stg256(out + col, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < m.cols) out[col + e] = v[e];
    }
}

// ---- backward pass of the gated block's activation ----------------------------------------------------------------------
// A block owns 128 tokens x 128 features and goes through it three times: dg = dh u a'(g), du = dh a(g), h = a(g) u, each made in fp32
// in the tile and quantised from there, so that none of the three goes to memory in a wide type.
struct MxGatedInput {
    const void* dh;
    const void* gu;                // [tokens][>= 2 features]: g, then u
    uint64_t dh_stride, gu_stride, features;
};
template <bool BF16, bool GELU, int PART>
__device__ __forceinline__ void gated_tile(float* tile, const MxGatedInput& in, uint64_t r0, uint64_t c0, int height, int width) {
    const int c = threadIdx.x % kTile;
#pragma unroll 8
    for (int r = threadIdx.x / kTile; r < kTile; r += kThreads / kTile) {
        float x = 0.0f;
        if (r < height && c < width) {
            const uint64_t at = (r0 + r) * in.gu_stride + c0 + c;
            const float g = load1<BF16>(in.gu, at);
            float a, da;
            gate_value_slope<GELU>(g, a, da);
            if constexpr (PART == 2) x = a * load1<BF16>(in.gu, at + in.features);
            else {
                const float dh = load1<BF16>(in.dh, (r0 + r) * in.dh_stride + c0 + c);
                x = PART == 1 ? dh * a : dh * load1<BF16>(in.gu, at + in.features) * da;
            }
        }
        tile[tile_at(r, c)] = x;
    }
}
template <bool BF16, bool GELU, bool STOCHASTIC>
__global__ void __launch_bounds__(kThreads) mx_gated_backward_kernel(MxGatedInput in, MxView dgu, MxView dgu_t, MxView h_t, uint32_t tiles_across, RoundKeys keys) {
    extern __shared__ __align__(16) unsigned char raw[];
    MxTile& t = *reinterpret_cast<MxTile*>(raw);
    pdl_wait();
    const uint64_t r0 = static_cast<uint64_t>(blockIdx.x / tiles_across) * kTile, c0 = static_cast<uint64_t>(blockIdx.x % tiles_across) * kTile;
    const int height = static_cast<int>(dgu.rows - r0 < kTile ? dgu.rows - r0 : kTile);
    const int width = static_cast<int>(in.features - c0 < kTile ? in.features - c0 : kTile);
    const bool last = c0 + kTile >= in.features;
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        const uint64_t at = part ? in.features + c0 : c0;
        if (part) gated_tile<BF16, GELU, 1>(t.v, in, r0, c0, height, width);
        else gated_tile<BF16, GELU, 0>(t.v, in, r0, c0, height, width);
        __syncthreads();
        tile_rows<STOCHASTIC, true>(t, dgu, r0, at, height, width, false, keys, 0, at);
        if constexpr (STOCHASTIC) __syncthreads();
        tile_cols<STOCHASTIC>(t, dgu_t, at, r0, height, width, false);
        __syncthreads();
    }
    // [dg | du] ends anywhere in its last scale tiles, since du starts behind dg: fill them up from there
    if (last && dgu.tiles)
        for (uint64_t block = mx_blocks(dgu.cols) + threadIdx.x / kTile; block < (mx_blocks(dgu.cols) + 3) / 4 * 4; block += kThreads / kTile)
             dgu.scales[mx_scale_at(dgu, r0 + threadIdx.x % kTile, block)] = 0;
    if (last && dgu_t.tiles)
        for (uint64_t row = dgu_t.rows + threadIdx.x / 4; row < (dgu_t.rows + 127) / 128 * 128; row += kThreads / 4) dgu_t.scales[mx_scale_at(dgu_t, row, r0 / 32 + threadIdx.x % 4)] = 0;
    gated_tile<BF16, GELU, 2>(t.v, in, r0, c0, height, width);
    __syncthreads();
    tile_cols<false>(t, h_t, c0, r0, height, width, last);
}

template <class K>
cudaError_t allow_smem(K* kernel, size_t bytes) {
    return cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
}

template <bool BF16, bool STOCHASTIC>
cudaError_t launch_quantize_as(const MxQuantizeCall& c) {
    const uint64_t rows = c.out->rows, cols = c.out->cols;
    const MxInput in{c.x, c.x_stride, (reinterpret_cast<uintptr_t>(c.x) | (rows > 1 ? c.x_stride * (BF16 ? 2 : 4) : 0)) % 16 == 0};
    const MxView out = mx_view(*c.out), out_t = c.out_t ? mx_view(*c.out_t) : MxView{};
    const RoundKeys keys = round_keys(c.seed);
    if (!c.out_t && in.wide) {
        uint32_t shift = 2;
        while (shift < 8 && (32ull << shift) < cols) ++shift;
        const uint64_t across = (mx_blocks(cols) + (1u << shift) - 1) >> shift, high = kThreads >> shift;
        const uint64_t rows_out = out.tiles ? (rows + 127) / 128 * 128 : rows;
        return launch_kernel(mx_rows_kernel<BF16, STOCHASTIC>, dim3(static_cast<unsigned>(across * ((rows_out + high - 1) / high))), kThreads, 0, c.stream, in, out, shift,
                             across, keys, c.first_row);
    }
    const uint64_t across = (cols + kTile - 1) / kTile, down = (rows + kTile - 1) / kTile;
    const dim3 grid(static_cast<unsigned>(across * down));
    if (c.out_t) {
        if (const cudaError_t e = allow_smem(mx_tile_kernel<BF16, STOCHASTIC, true>, sizeof(MxTile))) return e;
        return launch_kernel(mx_tile_kernel<BF16, STOCHASTIC, true>, grid, kThreads, sizeof(MxTile), c.stream, in, out, out_t, static_cast<uint32_t>(across), keys, c.first_row);
    }
    if (const cudaError_t e = allow_smem(mx_tile_kernel<BF16, STOCHASTIC, false>, sizeof(MxTile))) return e;
    return launch_kernel(mx_tile_kernel<BF16, STOCHASTIC, false>, grid, kThreads, sizeof(MxTile), c.stream, in, out, out_t, static_cast<uint32_t>(across), keys, c.first_row);
}

template <bool BF16, bool GELU, bool STOCHASTIC>
cudaError_t launch_gated_backward_as(const MxGatedBackwardCall& c) {
    const uint64_t features = c.h_t->rows, across = (features + kTile - 1) / kTile, down = (c.dgu->rows + kTile - 1) / kTile;
    const MxGatedInput in{c.dh, c.gu, c.dh_stride, c.gu_stride, features};
    auto* kernel = mx_gated_backward_kernel<BF16, GELU, STOCHASTIC>;
    if (const cudaError_t e = allow_smem(kernel, sizeof(MxTile))) return e;
    return launch_kernel(kernel, dim3(static_cast<unsigned>(across * down)), kThreads, sizeof(MxTile), c.stream, in, mx_view(*c.dgu), mx_view(*c.dgu_t), mx_view(*c.h_t),
                         static_cast<uint32_t>(across), round_keys(c.seed));
}
template <bool BF16, bool GELU>
cudaError_t launch_gated_backward_as(const MxGatedBackwardCall& c) {
    return c.stochastic ? launch_gated_backward_as<BF16, GELU, true>(c) : launch_gated_backward_as<BF16, GELU, false>(c);
}

}  // namespace

cudaError_t launch_mx_quantize(const MxQuantizeCall& c) {
    if (c.bf16) return c.stochastic ? launch_quantize_as<true, true>(c) : launch_quantize_as<true, false>(c);
    return c.stochastic ? launch_quantize_as<false, true>(c) : launch_quantize_as<false, false>(c);
}

cudaError_t launch_mx_dequantize(const tq_mx_t& m, void* out, bool bf16, uint64_t stride, cudaStream_t stream) {
    const uint64_t chunks = (m.cols + kThreads * 8 - 1) / (kThreads * 8);
    const dim3 grid(static_cast<unsigned>(chunks * m.rows));
    const bool wide = (reinterpret_cast<uintptr_t>(out) | (m.rows > 1 ? stride * (bf16 ? 2 : 4) : 0)) % 16 == 0;
    auto* kernel = bf16 ? (wide ? mx_dequantize_kernel<true, true> : mx_dequantize_kernel<true, false>)
                        : (wide ? mx_dequantize_kernel<false, true> : mx_dequantize_kernel<false, false>);
    return launch_kernel(kernel, grid, kThreads, 0, stream, mx_view(m), out, stride, static_cast<uint32_t>(chunks));
}

cudaError_t launch_mx_aggregate(const tq_mx_t& m, const float* weights, float* out, cudaStream_t stream) {
    MxWeights w{};
    const uint32_t n = static_cast<uint32_t>(m.rows);
    if (weights)
        for (uint32_t i = 0; i < n; ++i) w.w[i] = weights[i];
    const dim3 grid(static_cast<unsigned>((mx_blocks(m.cols) + kThreads - 1) / kThreads));
    auto* kernel = weights ? mx_aggregate_kernel<true> : mx_aggregate_kernel<false>;
    return launch_kernel(kernel, grid, kThreads, 0, stream, mx_view(m), out, n, static_cast<float>(n), w);
}

cudaError_t launch_mx_gated_backward(const MxGatedBackwardCall& c) {
    if (c.bf16) return c.gelu ? launch_gated_backward_as<true, true>(c) : launch_gated_backward_as<true, false>(c);
    return c.gelu ? launch_gated_backward_as<false, true>(c) : launch_gated_backward_as<false, false>(c);
}

}  // namespace tq
