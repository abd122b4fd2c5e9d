// Microscaled 4-bit floating point: quantisation along one or both axes, decoding, the mean of decoded rows, and the backward
// pass of the gated block's activation, which ends in three quantised matrices.
#include <cstddef>

#include "tq_mx.cuh"

namespace tq {

namespace {

struct MxInput {
    const void* data;
    uint64_t stride;               // elements from row to row
    uint32_t wide;                 // the boundary that every row starts on: 32 bytes, 16, or 0 for any
};

// A row block of 32 elements of the matrix from memory, zeros outside.  `wide`: the boundary that rows start on, 32 bytes, 16 or 0 for any.
template <bool BF16>
__device__ __forceinline__ void load_row_block(const void* data, uint64_t at, uint32_t wide, int count, float (&v)[32]) {
    const char* src = static_cast<const char*>(data) + at * (BF16 ? 2 : 4);
    if (wide == 32 && count >= 32) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) {
            uint32_t x[8];
            ldg256(src + 32 * i, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if constexpr (BF16) { v[16 * i + 2 * k] = __uint_as_float(x[k] << 16); v[16 * i + 2 * k + 1] = __uint_as_float(x[k] & 0xFFFF0000u); }
                else v[8 * i + k] = __uint_as_float(x[k]);
            }
        }
    } else if (wide && count >= 32) {
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
        for (int i = 0; i < 32; ++i) v[i] = i < count ? load1<BF16>(src, i) : 0.0f;
    }
}

// ---- along the rows ----------------------------------------------------------------------------------------
// One thread makes one block: 64 or 128 bytes in, 16 bytes of codes and a byte of scale out, no exchange between threads.
// A block of 256 threads covers 2^shift MX blocks of 256 >> shift rows.  16 x 25.6 M fp32, stochastic: 304 us, 6.1 TB/s, with four blocks an SM (64
// registers); 383 us with three.
template <bool BF16, bool STOCHASTIC>
__global__ void __launch_bounds__(kThreads, 4) mx_rows_kernel(MxInput in, MxView out, uint32_t shift, uint64_t col_groups, RoundKeys keys, uint32_t first_row) {
    pdl_wait();
    const uint64_t row = (blockIdx.x / col_groups) * (kThreads >> shift) + (threadIdx.x >> shift);
    const uint64_t block = (blockIdx.x % col_groups << shift) + (threadIdx.x & ((1u << shift) - 1));
    const uint64_t blocks = mx_blocks(out.cols);
    if (row >= out.rows || block >= blocks) {
        // the tile layout is filled up to whole tiles
        if (out.tiles && row < (out.rows + 127) / 128 * 128 && block < (blocks + 3) / 4 * 4) out.scales[mx_scale_at(out, row, block)] = 0;
        return;
    }
    float v[32];
    load_row_block<BF16>(in.data, row * in.stride + block * 32, in.wide, out.cols - block * 32 < 32 ? static_cast<int>(out.cols - block * 32) : 32, v);
    const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
    const PhiloxRun run = philox_run(static_cast<uint32_t>(block * 4 >> 32), first_row + static_cast<uint32_t>(row), keys);
    const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q) {
        RowBits r;
        mx_random8(run, block * 4 + q, keys, r);
        return r;
    });
    stg128(out.codes + row * out.code_stride + block * 16, codes);
    out.scales[mx_scale_at(out, row, block)] = static_cast<uint8_t>(byte);
}

// ---- tiles in shared memory ------------------------------------------------------------------------------------
// 64 x 128 elements, one block of 32 along a row and one along a column for each of 256 threads.  The thread makes its row block from
// registers and leaves the elements in shared memory in fp32 for the thread that makes the column block.  32 elements are followed by
// 4 words of padding, 32 rows by 16: the 16-byte accesses of eight threads (two rows, four blocks) then touch different banks, as do those of 32
// threads down 16 columns in both halves of the rows.  Two threads so hold the neighbouring 16 bytes of a transposed row, and stores fill sectors.
// 53 KB with the random bits: four blocks an SM, so that loads of one run beside the arithmetic of others.
constexpr int kTileRows = 64, kTileCols = 128;
constexpr int kTilePitch = 4 * 36;
struct MxTile {
    float v[kTileRows * kTilePitch + 16];
    uint32_t random[kTileRows * 64 + 8];   // 16 bits an element, inverted, in 16-byte chunks of 8; see random_chunk.  Not there where rounding is to nearest
};
__host__ __device__ constexpr size_t tile_bytes(bool stochastic) { return stochastic ? sizeof(MxTile) : offsetof(MxTile, random); }
__device__ __forceinline__ int tile_at(int r, int c) { return r * kTilePitch + (r >> 5) * 16 + (c >> 5) * 36 + (c & 31); }
// Word of the 16-byte chunk with the bits of row r, columns 8g .. 8g + 7.  The exchange of chunks keeps eight threads that write (two rows,
// four blocks) in different banks.
__device__ __forceinline__ int random_chunk(int r, int g) { return r * 64 + (r >> 5) * 8 + ((g ^ ((g >> 3) | ((r & 1) << 1))) << 2); }

// This thread's row block: row r, block b of the tile.
struct MxItem {
    int r, b;
};
__device__ __forceinline__ MxItem row_item() { return MxItem{static_cast<int>(threadIdx.x) >> 2, static_cast<int>(threadIdx.x) & 3}; }

__device__ __forceinline__ void put_row(MxTile& t, const MxItem& it, const float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<float4*>(&t.v[tile_at(it.r, it.b * 32 + 4 * i)]) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}
__device__ __forceinline__ void get_row(const MxTile& t, const MxItem& it, float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(&t.v[tile_at(it.r, it.b * 32 + 4 * i)]);
        v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
    }
}

// The thread's row block -> codes and scale of `out`: the tile starts at row r0, column c0 (a multiple of 32) of that matrix and `height` x `width`
// of it count.  `fill`: the tile ends the matrix on the right, and its row of scales is filled up with zeros.
template <bool STOCHASTIC, bool KEEP>
__device__ __forceinline__ void encode_row(MxTile& t, const MxItem& it, const float (&v)[32], const MxView& out, uint64_t r0, uint64_t c0, int height, int width, bool fill,
                                           const RoundKeys& keys, uint32_t first_row) {
    const uint64_t blocks = mx_blocks(out.cols), block = c0 / 32 + it.b;
    const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
    const PhiloxRun run = philox_run(static_cast<uint32_t>(block * 4 >> 32), first_row + static_cast<uint32_t>(r0) + it.r, keys);
    const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q) {
        RowBits r;
        mx_random8(run, block * 4 + q, keys, r);
        if constexpr (KEEP) *reinterpret_cast<uint4*>(&t.random[random_chunk(it.r, it.b * 4 + q)]) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        return r;
    });
    if (it.r < height && it.b * 32 < width) {
        stg128(out.codes + (r0 + it.r) * out.code_stride + block * 16, codes);
        out.scales[mx_scale_at(out, r0 + it.r, block)] = static_cast<uint8_t>(byte);
    } else if (out.tiles && (it.b * 32 < width || (fill && block < (blocks + 3) / 4 * 4))) {
        out.scales[mx_scale_at(out, r0 + it.r, block)] = 0;
    }
}

// The thread's column block: column c of the tile becomes row q0 + c of `out`, whose blocks run over the tile's rows from r0 on.
// `fill`: the tile ends `out` below, and the rest of its last 128 rows gets zero scales.
template <bool STOCHASTIC>
__device__ __forceinline__ void encode_col(const MxTile& t, const MxView& out, uint64_t q0, uint64_t r0, int height, int width, bool fill) {
    const int c = threadIdx.x >> 1, b = threadIdx.x & 1;
    const uint64_t blocks = mx_blocks(out.cols), block = r0 / 32 + b, row = q0 + c;
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = t.v[tile_at(b * 32 + i, c)];
    const uint32_t byte = mx_scale_byte<STOCHASTIC>(max_abs_32(v));
    const uint4 codes = mx_encode32<STOCHASTIC>(v, byte, [&](int q) {
        ColumnBits r;
        r.side = c & 1 ? 0x0100u : 0x0001u;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = t.random[random_chunk(b * 32 + q * 8 + i, c >> 3) + ((c & 7) >> 1)];
        return r;
    });
    if (c < width && b * 32 < height) {
        stg128(out.codes + row * out.code_stride + block * 16, codes);
        out.scales[mx_scale_at(out, row, block)] = static_cast<uint8_t>(byte);
    } else if (out.tiles && block < (blocks + 3) / 4 * 4 && (c < width || (fill && row < (out.rows + 127) / 128 * 128))) {
        out.scales[mx_scale_at(out, row, block)] = 0;
    }
}

__device__ __forceinline__ int within(uint64_t size, uint64_t from, int most) {
    return from >= size ? 0 : size - from < static_cast<uint64_t>(most) ? static_cast<int>(size - from) : most;
}

// 8192 x 4096 bf16 along both axes: nearest 23.5 us (4.4 TB/s), where warps wait for memory and the shared-memory pipe is 67 % busy; stochastic 44, 32 instructions an
// element: 72 % of the issue slots, the integer and fma-heavy pipes 60 % each, none of them full; warps wait for a pipe or to be dispatched, hardly for memory.
// Rows on any boundary: 8191 x 5003 fp32 along rows 32 us nearest, 52 stochastic, bf16 50 and 85.  A tile is 64 rows high whether there are so many or not: 16 messages of 25.6 M
// fp32 that follow one another without padding take 3.2 ms, on 16-byte boundaries 0.32.
template <bool BF16, bool STOCHASTIC, bool BOTH>
__global__ void __launch_bounds__(kThreads, 4) mx_tile_kernel(MxInput in, MxView out, MxView out_t, uint32_t tiles_across, RoundKeys keys, uint32_t first_row) {
    extern __shared__ __align__(16) unsigned char raw[];
    MxTile& t = *reinterpret_cast<MxTile*>(raw);
    pdl_wait();
    const uint64_t r0 = static_cast<uint64_t>(blockIdx.x / tiles_across) * kTileRows, c0 = static_cast<uint64_t>(blockIdx.x % tiles_across) * kTileCols;
    const int height = within(out.rows, r0, kTileRows), width = within(out.cols, c0, kTileCols);
    const MxItem it = row_item();
    float v[32];
    // fp32: 16 bytes a thread, a warp in whole lines, by way of the tile (8192 x 4096, stochastic: 62 us with 128 bytes a thread, 52 so; bf16 rows, half as
    // long, go straight to the registers: 23.5 us nearest, 25 by way of the tile)
    if (BOTH && !BF16 && in.wide && width == kTileCols) {
        constexpr int kIn = kTileCols / 4, kEach = kTileRows * kIn / kThreads;
        const int r = threadIdx.x / kIn, c = threadIdx.x % kIn * 4;
        const char* src = static_cast<const char*>(in.data) + ((r0 + r) * in.stride + c0 + c) * 4;
        uint4 w[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            w[i] = make_uint4(0, 0, 0, 0);
            if (r + i * (kThreads / kIn) < height) w[i] = ldg128(src);
            src += in.stride * (kThreads / kIn) * 4;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            *reinterpret_cast<float4*>(&t.v[tile_at(r + i * (kThreads / kIn), c)]) =
                make_float4(__uint_as_float(w[i].x), __uint_as_float(w[i].y), __uint_as_float(w[i].z), __uint_as_float(w[i].w));
        __syncthreads();
        get_row(t, it, v);
    } else if (BOTH && in.wide) {
        load_row_block<BF16>(in.data, (r0 + it.r) * in.stride + c0 + it.b * 32, in.wide, it.r < height ? width - it.b * 32 : 0, v);
        put_row(t, it, v);
    } else {                               // rows on any boundary (for the copy along rows alone, no others come here): one element a thread at a time
        const int c = threadIdx.x % kTileCols, first = threadIdx.x / kTileCols;
        const char* src = static_cast<const char*>(in.data) + ((r0 + first) * in.stride + c0 + c) * (BF16 ? 2 : 4);
#pragma unroll
        for (int half = 0; half < 2; ++half) {             // 16 loads, then 16 stores: in turn they took 91 us for 8191 x 5003 fp32 along both axes, so 67
            float x[kTileRows / 4];
#pragma unroll
            for (int i = 0; i < kTileRows / 4; ++i) {
                x[i] = 0.0f;
                if (first + (half * kTileRows / 4 + i) * 2 < height && c < width) x[i] = load1<BF16>(src, 0);
                src += in.stride * (BF16 ? 4 : 8);
            }
#pragma unroll
            for (int i = 0; i < kTileRows / 4; ++i) t.v[tile_at(first + (half * kTileRows / 4 + i) * 2, c)] = x[i];
        }
        __syncthreads();
        get_row(t, it, v);
    }
    encode_row<STOCHASTIC, BOTH>(t, it, v, out, r0, c0, height, width, true, keys, first_row);
    if constexpr (BOTH) {
        __syncthreads();
        encode_col<STOCHASTIC>(t, out_t, c0, r0, height, width, true);
    }
}

// ---- decoding ----------------------------------------------------------------------------------------------------
// Row and column of this thread, which makes EACH elements in each of ROWS rows: a block covers EACH << shift columns and ROWS * (256 >> shift) rows.
template <int EACH, int ROWS>
struct DecodePlace {
    uint32_t high, row;
    uint64_t col;
    __device__ __forceinline__ DecodePlace(uint32_t chunks, uint32_t shift) {
        high = kThreads >> shift;
        row = blockIdx.x / chunks * (high * ROWS) + (threadIdx.x >> shift);
        col = (static_cast<uint64_t>(blockIdx.x % chunks) * EACH << shift) + (threadIdx.x & ((1u << shift) - 1)) * EACH;
    }
};
__device__ __forceinline__ uint64_t mx_scale_row(const MxView& m, uint32_t row) {              // where row's first scale is
    return m.tiles ? (row >> 7) * m.scale_stride + (row & 31) * 16 + ((row >> 5) & 3) * 4 : row * m.scale_stride;
}

// Rows that start on 16-byte boundaries (`wide`: 32): 16 elements of 2 rows, stored in pieces of 32 or 16 bytes.  8192 x 4096 to bf16: 11.8 us, 7.2 TB/s of the L2
// and memory (with 8 elements of 4 rows, more of it addresses, 15).
constexpr int kWideEach = 16, kWideRows = 2;
template <bool BF16>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(MxView m, void* out, uint64_t stride, uint32_t chunks, uint32_t shift, uint32_t wide) {
    pdl_wait();
    const DecodePlace<kWideEach, kWideRows> at(chunks, shift);
    if (at.col >= m.cols) return;
    const uint64_t scale_at = m.tiles ? (at.col >> 7) * 512 + ((at.col >> 5) & 3) : at.col >> 5;
    uint32_t codes[kWideRows][2], byte[kWideRows];
#pragma unroll
    for (int i = 0; i < kWideRows; ++i) {
        const uint32_t row = at.row + i * at.high;
        codes[i][0] = codes[i][1] = byte[i] = 0;
        if (row < m.rows) {
            asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(codes[i][0]), "=r"(codes[i][1]) : "l"(m.codes + row * m.code_stride + at.col / 2) : "memory");
            byte[i] = ldg8(m.scales + mx_scale_row(m, row) + scale_at);
        }
    }
#pragma unroll
    for (int i = 0; i < kWideRows; ++i) {
        const uint32_t row = at.row + i * at.high;
        if (row >= m.rows) continue;
        char* const to = static_cast<char*>(out) + (row * stride + at.col) * (BF16 ? 2 : 4);
        const f32x2 scale = both(mx_scale_value(byte[i]));
        float v[16];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float x[8];
            e2m1_values8(codes[i][q], x);
#pragma unroll
            for (int e = 0; e < 8; e += 2) unpair(mul2(pair(x[e], x[e + 1]), scale), v[8 * q + e], v[8 * q + e + 1]);
        }
        if (at.col + kWideEach <= m.cols) {
            if constexpr (BF16) {
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                if (wide == 32) stg256_words(to, w);
                else { stg128(to, make_uint4(w[0], w[1], w[2], w[3])); stg128(to + 16, make_uint4(w[4], w[5], w[6], w[7])); }
            } else {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(v[e]);
                if (wide == 32) {
                    const uint32_t lo[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]}, hi[8] = {w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]};
                    stg256_words(to, lo);
                    stg256_words(to + 32, hi);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) stg128(to + 16 * e, make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]));
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (at.col + e < m.cols) {
                    if constexpr (BF16) reinterpret_cast<unsigned short*>(to)[e] = static_cast<unsigned short>(__float_as_uint(v[e]) >> 16);   // exact
                    else reinterpret_cast<float*>(to)[e] = v[e];
                }
        }
    }
}

// Rows on any boundary: 8 elements of 4 rows; a warp's 256 go through shared memory, so that consecutive threads store consecutive words.  bf16 rows may
// start in the middle of a word: two elements a thread all the same, the first and last alone.  8191 x 5003: to fp32 32 us (5.8 TB/s), to bf16 27 (3.9 TB/s), bound by
// instructions, some 19 an element.  (Two words of codes shifted to the output's own 16-byte pieces, without shared memory: 39 and 31 us.)
constexpr int kRaggedEach = 8, kRaggedRows = 4;
template <bool BF16>
__global__ void __launch_bounds__(kThreads) mx_dequantize_ragged_kernel(MxView m, void* out, uint64_t stride, uint32_t chunks, uint32_t shift) {
    constexpr int kWords = BF16 ? 128 : 256;
    __shared__ __align__(16) uint32_t staged[kThreads / 32][kWords];
    pdl_wait();
    const DecodePlace<kRaggedEach, kRaggedRows> at(chunks, shift);
    const uint32_t lane = threadIdx.x & 31;
    uint32_t* const words = staged[threadIdx.x / 32];
    const uint64_t first = at.col - lane * kRaggedEach;          // shift >= 5: a warp lies in one row
    if (first >= m.cols) return;
    const bool any = at.col < m.cols;
    const int count = m.cols - first < 256 ? static_cast<int>(m.cols - first) : 256;
    const uint64_t scale_at = m.tiles ? (at.col >> 7) * 512 + ((at.col >> 5) & 3) : at.col >> 5;
    uint32_t codes[kRaggedRows], byte[kRaggedRows];
#pragma unroll
    for (int i = 0; i < kRaggedRows; ++i) {
        const uint32_t row = at.row + i * at.high;
        codes[i] = byte[i] = 0;
        if (any && row < m.rows) {
            asm volatile("ld.global.b32 %0, [%1];" : "=r"(codes[i]) : "l"(m.codes + row * m.code_stride + at.col / 2) : "memory");
            byte[i] = ldg8(m.scales + mx_scale_row(m, row) + scale_at);
        }
    }
#pragma unroll
    for (int i = 0; i < kRaggedRows; ++i) {
        const uint32_t row = at.row + i * at.high;
        if (row >= m.rows) break;                                // a whole warp's
        const f32x2 scale = both(mx_scale_value(byte[i]));
        float v[8];
        e2m1_values8(codes[i], v);
#pragma unroll
        for (int e = 0; e < 8; e += 2) unpair(mul2(pair(v[e], v[e + 1]), scale), v[e], v[e + 1]);
        __syncwarp();
        if constexpr (BF16) {
            unsigned short* const to = static_cast<unsigned short*>(out) + row * stride + first;
            const int off = static_cast<int>(reinterpret_cast<uintptr_t>(to) >> 1 & 1);      // 1: the row starts in the middle of a word, and words hold elements 2t - 1 and 2t
            const float before = __shfl_up_sync(0xFFFFFFFFu, v[7], 1);
            *reinterpret_cast<uint4*>(&words[4 * lane]) = off ? make_uint4(pack_bf16(before, v[0]), pack_bf16(v[1], v[2]), pack_bf16(v[3], v[4]), pack_bf16(v[5], v[6]))
                                                              : make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            __syncwarp();
            unsigned short* const mine = to + 2 * static_cast<int>(lane) - off;
            if (off && lane == 31 && count == 256) to[255] = static_cast<unsigned short>(__float_as_uint(v[7]) >> 16);
            if (count == 256 && !(off && lane == 0)) {
#pragma unroll
                for (int k = 0; k < 4; ++k) asm volatile("st.global.b32 [%0], %1;" ::"l"(mine + 64 * k), "r"(words[32 * k + lane]) : "memory");
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int e = 2 * (32 * k + static_cast<int>(lane)) - off;
                    const uint32_t two = words[32 * k + lane];
                    if (e >= 0 && e + 1 < count) asm volatile("st.global.b32 [%0], %1;" ::"l"(to + e), "r"(two) : "memory");
                    else if (e >= 0 && e < count) to[e] = static_cast<unsigned short>(two);
                    else if (e == -1) to[0] = static_cast<unsigned short>(two >> 16);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q)
                *reinterpret_cast<float4*>(&words[8 * lane + 4 * q]) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            __syncwarp();
            float* const to = static_cast<float*>(out) + row * stride + first + lane;
            if (count == 256) {
#pragma unroll
                for (int k = 0; k < 8; ++k) to[32 * k] = __uint_as_float(words[32 * k + lane]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (32 * k + static_cast<int>(lane) < count) to[32 * k] = __uint_as_float(words[32 * k + lane]);
            }
        }
    }
}

// ---- mean of decoded rows --------------------------------------------------------------------------------------------
struct MxWeights {
    float w[TQ_MAX_WORKERS];
};
// Eight sums over n, each rounded once.  inv = 1 / n rounded; for a power of two the product is all there is to it.  Else one step of Markstein's (IBM J. Res. Dev. 34,
// 1990): with q = x inv, the remainder x - q n is exact in a fused operation, and q + remainder * inv is x / n correctly rounded as long as nothing
// underflows.  Tiny sums, infinities and NaN take the division itself (for all, 2 rows of 50 M took 140 us instead of 54).
__device__ __forceinline__ void divide8(float (&v)[8], float n, float inv, bool exact) {
    if (exact) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= inv;
        return;
    }
    bool plain = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) plain = plain && ((__float_as_uint(v[e]) & 0x7FFFFFFFu) - 0x10000000u < 0x6F800000u || v[e] == 0.0f);      // 2^-95 <= |x| < infinity
    if (plain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = v[e] * inv;
            v[e] = fmaf(fmaf(-q, n, v[e]), inv, q);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fdiv_rn(v[e], n);
    }
}
// A thread decodes the same EACH elements of every worker's row (32, a block; 8 where the rows are too short to fill the GPU so) and keeps their sums.
// fp32, in worker order; code * scale is exact, so that one fused operation adds it.  16 x 25.6 M: 63 us, 5.1 TB/s; four workers' codes are asked for at a time
// (two 66 us, eight 69).
template <bool WEIGHTED, int EACH>
__global__ void __launch_bounds__(kThreads) mx_aggregate_kernel(MxView m, float* out, uint32_t n, float divisor, float inv, bool exact, MxWeights weights) {
    pdl_wait();
    const uint64_t first = (static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x) * EACH;
    if (first >= m.cols) return;
    f32x2 sum[EACH / 2];
#pragma unroll
    for (int e = 0; e < EACH / 2; ++e) sum[e] = both(0.0f);
    const uint8_t* codes = m.codes + first / 2;
    const uint8_t* scales = m.scales + first / 32;
    constexpr uint32_t kAhead = EACH == 8 ? 16 : 4;          // workers whose codes are asked for at a time
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < n; i0 += kAhead) {
        uint32_t w[kAhead][EACH / 8], byte[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
            if (i0 + i < n) {
                if constexpr (EACH == 32) {
                    const uint4 c = ldg128(codes);
                    w[i][0] = c.x; w[i][1] = c.y; w[i][2] = c.z; w[i][3] = c.w;
                } else {
                    asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[i][0]) : "l"(codes) : "memory");
                }
                byte[i] = ldg8(scales);
            }
            codes += m.code_stride; scales += m.scale_stride;
        }
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
            if (i0 + i >= n) break;
            const f32x2 scale = both(mx_scale_value(byte[i]));
#pragma unroll
            for (int q = 0; q < EACH / 8; ++q) {
                float v[8];
                e2m1_values8(w[i][q], v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x2& to = sum[4 * q + e];
                    if constexpr (WEIGHTED) to = add2(to, mul2(mul2(pair(v[2 * e], v[2 * e + 1]), scale), both(weights.w[i0 + i])));
                    else to = fma2(pair(v[2 * e], v[2 * e + 1]), scale, to);
                }
            }
        }
    }
#pragma unroll
    for (int q = 0; q < EACH / 8; ++q) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            unpair(sum[4 * q + e], v[2 * e], v[2 * e + 1]);
        }
        if constexpr (!WEIGHTED) divide8(v, divisor, inv, exact);
        const uint64_t col = first + 8 * q;
        if (col + 8 <= m.cols) stg256(out + col, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < m.cols) out[col + e] = v[e];
    }
}

// ---- backward pass of the gated block's activation ----------------------------------------------------------------------
// A block owns 64 tokens x 128 features: dg = dh u a'(g), du = dh a(g) and h = a(g) u are made in fp32 in registers and go through the
// tile one after another, so that none of the three goes to memory in a wide type.
struct MxGatedInput {
    const void* dh;
    const void* gu;                // [tokens][>= 2 features]: g, then u
    uint64_t dh_stride, gu_stride, features;
    uint32_t wide;                 // the boundary that all rows start on: 32 bytes, 16, or 0 for any
};
// bf16 rows on 16-byte boundaries come ahead: while a block works on one tile, its 64 x 128 of dh, g and u for the next are copied into shared memory
// (asynchronously, whole lines by neighbouring threads, chunks of 16 bytes exchanged as in random_chunk).
constexpr int kInputs = 3;
struct MxAhead {
    uint4 v[kInputs][kTileRows * 16];
};
__device__ __forceinline__ int ahead_chunk(int r, int g) { return r * 16 + (g ^ ((g >> 3) | ((r & 1) << 1))); }
__device__ __forceinline__ void copy_ahead(MxAhead& a, const MxGatedInput& in, uint64_t r0, uint64_t c0, int height, int width) {
#pragma unroll
    for (int j = 0; j < kInputs; ++j) {
        const char* const base = static_cast<const char*>(j == 0 ? in.dh : in.gu);
        const uint64_t stride = j == 0 ? in.dh_stride : in.gu_stride, from = r0 * stride + c0 + (j == 2 ? in.features : 0);
#pragma unroll
        for (int i = 0; i < kTileRows * 16 / kThreads; ++i) {
            const int at = threadIdx.x + i * kThreads, r = at >> 4, g = at & 15;
            const bool inside = r < height && g * 8 < width;
            const char* const src = base + (inside ? (from + r * stride + g * 8) * 2 : 0);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(&a.v[j][ahead_chunk(r, g)])), "l"(src), "r"(inside ? 16 : 0) : "memory");
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void take_ahead(const MxAhead& a, int j, const MxItem& it, float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 w = a.v[j][ahead_chunk(it.r, it.b * 4 + i)];
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[8 * i + 2 * k] = __uint_as_float(x[k] << 16); v[8 * i + 2 * k + 1] = __uint_as_float(x[k] & 0xFFFF0000u); }
    }
}

// A block takes tile after tile.  AHEAD: as above, 102 KB of shared memory, two blocks an SM.  8192 x 8192 bf16: stochastic 286 us, 106 instructions a feature at 0.7 a
// clock and scheduler; nearest 183 (3.2 TB/s), 67 instructions; GELU 313 and 204.  (With an exponential that is flushed below 2^-126 250 and 154, but gates below -87 came out as zeros.)
// Three blocks a tile, one for each of dg, du and h, with half the registers, took 331 where this took 274.
template <bool BF16, bool AHEAD, bool GELU, bool STOCHASTIC>
__global__ void __launch_bounds__(kThreads, 2) mx_gated_backward_kernel(MxGatedInput in, MxView dgu, MxView dgu_t, MxView h_t, uint32_t tiles_across, uint32_t tiles, RoundKeys keys) {
    extern __shared__ __align__(16) unsigned char raw[];
    MxTile& t = *reinterpret_cast<MxTile*>(raw);
    MxAhead& ahead = *reinterpret_cast<MxAhead*>(raw + tile_bytes(STOCHASTIC));
    pdl_wait();
    const MxItem it = row_item();
    const auto row_of = [&](uint32_t tile) { return static_cast<uint64_t>(tile / tiles_across) * kTileRows; };
    const auto col_of = [&](uint32_t tile) { return static_cast<uint64_t>(tile % tiles_across) * kTileCols; };
    const auto ask = [&](uint32_t tile) {
        copy_ahead(ahead, in, row_of(tile), col_of(tile), within(dgu.rows, row_of(tile), kTileRows), within(in.features, col_of(tile), kTileCols));
    };
    if constexpr (AHEAD) ask(blockIdx.x);
#pragma unroll 1
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t r0 = row_of(tile), c0 = col_of(tile);
        const int height = within(dgu.rows, r0, kTileRows), width = within(in.features, c0, kTileCols);
        const bool last = c0 + kTileCols >= in.features;
        float dh[32], g[32], u[32];                // become du, dg and h
        if constexpr (AHEAD) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncthreads();                       // also: the tile's last reader is through
            take_ahead(ahead, 0, it, dh); take_ahead(ahead, 1, it, g); take_ahead(ahead, 2, it, u);
        } else {
            const int count = it.r < height ? width - it.b * 32 : 0;
            const uint64_t row = r0 + it.r, col = c0 + it.b * 32;
            load_row_block<BF16>(in.dh, row * in.dh_stride + col, in.wide, count, dh);
            load_row_block<BF16>(in.gu, row * in.gu_stride + col, in.wide, count, g);
            load_row_block<BF16>(in.gu, row * in.gu_stride + in.features + col, in.wide, count, u);
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float a, slope;
            gate_value_slope<GELU>(g[i], a, slope);
            g[i] = dh[i] * u[i] * slope;
            dh[i] = dh[i] * a;
            u[i] = a * u[i];
        }
        // h first: it takes no random numbers, whose registers beside those of all three would not do
        put_row(t, it, u);
        __syncthreads();
        if constexpr (AHEAD)
            if (tile + gridDim.x < tiles) ask(tile + gridDim.x);
        encode_col<false>(t, h_t, c0, r0, height, width, last);
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
            const uint64_t at = part ? in.features + c0 : c0;
            __syncthreads();
            put_row(t, it, g);
            encode_row<STOCHASTIC, true>(t, it, g, dgu, r0, at, height, width, false, keys, 0);
            __syncthreads();
            encode_col<STOCHASTIC>(t, dgu_t, at, r0, height, width, false);
#pragma unroll
            for (int i = 0; i < 32; ++i) g[i] = dh[i];
        }
        // [dg | du] ends anywhere in its last scale tiles, since du starts behind dg: fill them up from there
        if (last && dgu.tiles)
            for (uint64_t block = mx_blocks(dgu.cols) + threadIdx.x / kTileRows; block < (mx_blocks(dgu.cols) + 3) / 4 * 4; block += kThreads / kTileRows)
                dgu.scales[mx_scale_at(dgu, r0 + threadIdx.x % kTileRows, block)] = 0;
        if (last && dgu_t.tiles)
            for (uint64_t q = dgu_t.rows + threadIdx.x / 2; q < (dgu_t.rows + 127) / 128 * 128; q += kThreads / 2)
                dgu_t.scales[mx_scale_at(dgu_t, q, r0 / 32 + threadIdx.x % 2)] = 0;
    }
}

uint32_t boundary(uint64_t at) { return at % 32 == 0 ? 32 : at % 16 == 0 ? 16 : 0; }

template <auto KERNEL, class... A>
cudaError_t launch_tiled(dim3 grid, size_t smem, cudaStream_t stream, const A&... args) {
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared_memory(KERNEL, smem, allowed)) return e;
    return launch_kernel(KERNEL, grid, kThreads, smem, stream, args...);
}

template <bool BF16, bool STOCHASTIC>
cudaError_t launch_quantize_as(const MxQuantizeCall& c) {
    const uint64_t rows = c.out->rows, cols = c.out->cols;
    const MxInput in{c.x, c.x_stride, boundary(reinterpret_cast<uintptr_t>(c.x) | (rows > 1 ? c.x_stride * (BF16 ? 2 : 4) : 0))};
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
    const uint64_t across = (cols + kTileCols - 1) / kTileCols, down = (rows + 127) / 128 * 2;       // whole scale tiles
    const dim3 grid(static_cast<unsigned>(across * down));
    if (c.out_t) return launch_tiled<mx_tile_kernel<BF16, STOCHASTIC, true>>(grid, tile_bytes(STOCHASTIC), c.stream, in, out, out_t, static_cast<uint32_t>(across), keys, c.first_row);
    return launch_tiled<mx_tile_kernel<BF16, STOCHASTIC, false>>(grid, tile_bytes(STOCHASTIC), c.stream, in, out, out_t, static_cast<uint32_t>(across), keys, c.first_row);
}

template <bool BF16, bool GELU, bool STOCHASTIC>
cudaError_t launch_gated_backward_as(const MxGatedBackwardCall& c) {
    const uint64_t features = c.h_t->rows, across = (features + kTileCols - 1) / kTileCols, down = (c.dgu->rows + 127) / 128 * 2;
    const uint64_t size = BF16 ? 2 : 4;
    const MxGatedInput in{c.dh, c.gu, c.dh_stride, c.gu_stride, features,
                          boundary(reinterpret_cast<uintptr_t>(c.dh) | reinterpret_cast<uintptr_t>(c.gu) | (c.dgu->rows > 1 ? (c.dh_stride | c.gu_stride) * size : 0))};
    const uint64_t tiles = across * down, room = 2 * static_cast<uint64_t>(sm_count());
    const dim3 grid(static_cast<unsigned>(tiles < room ? tiles : room));
    if constexpr (BF16)
        if (in.wide)
            return launch_tiled<mx_gated_backward_kernel<true, true, GELU, STOCHASTIC>>(grid, tile_bytes(STOCHASTIC) + sizeof(MxAhead), c.stream, in, mx_view(*c.dgu),
                                                                                       mx_view(*c.dgu_t), mx_view(*c.h_t), static_cast<uint32_t>(across), static_cast<uint32_t>(tiles),
                                                                                       round_keys(c.seed));
    return launch_tiled<mx_gated_backward_kernel<BF16, false, GELU, STOCHASTIC>>(grid, tile_bytes(STOCHASTIC), c.stream, in, mx_view(*c.dgu), mx_view(*c.dgu_t), mx_view(*c.h_t),
                         static_cast<uint32_t>(across), static_cast<uint32_t>(tiles), round_keys(c.seed));
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
    const uint32_t wide = boundary(reinterpret_cast<uintptr_t>(out) | (m.rows > 1 ? stride * (bf16 ? 2 : 4) : 0));
    const uint64_t each = wide ? kWideEach : kRaggedEach;
    uint32_t shift = wide ? 1 : 5;
    while (shift < 8 && (each << shift) < m.cols) ++shift;
    const uint64_t chunks = (m.cols + (each << shift) - 1) / (each << shift), high = static_cast<uint64_t>(kThreads >> shift) * (wide ? kWideRows : kRaggedRows);
    const dim3 grid(static_cast<unsigned>(chunks * ((m.rows + high - 1) / high)));
    if (wide) return launch_kernel(bf16 ? mx_dequantize_kernel<true> : mx_dequantize_kernel<false>, grid, kThreads, 0, stream, mx_view(m), out, stride, static_cast<uint32_t>(chunks), shift, wide);
    return launch_kernel(bf16 ? mx_dequantize_ragged_kernel<true> : mx_dequantize_ragged_kernel<false>, grid, kThreads, 0, stream, mx_view(m), out, stride, static_cast<uint32_t>(chunks), shift);
}

cudaError_t launch_mx_aggregate(const tq_mx_t& m, const float* weights, float* out, cudaStream_t stream) {
    MxWeights w{};
    const uint32_t n = static_cast<uint32_t>(m.rows);
    if (weights)
        for (uint32_t i = 0; i < n; ++i) w.w[i] = weights[i];
    const bool shortened = mx_blocks(m.cols) < static_cast<uint64_t>(sm_count()) * kThreads * 2;
    const uint64_t each = shortened ? 8 : 32;
    const dim3 grid(static_cast<unsigned>((m.cols + each * kThreads - 1) / (each * kThreads)));
    auto* kernel = shortened ? (weights ? mx_aggregate_kernel<true, 8> : mx_aggregate_kernel<false, 8>)
                             : (weights ? mx_aggregate_kernel<true, 32> : mx_aggregate_kernel<false, 32>);
    return launch_kernel(kernel, grid, kThreads, 0, stream, mx_view(m), out, n, static_cast<float>(n), 1.0f / static_cast<float>(n), (n & (n - 1)) == 0, w);
}

cudaError_t launch_mx_gated_backward(const MxGatedBackwardCall& c) {
    if (c.bf16) return c.gelu ? launch_gated_backward_as<true, true>(c) : launch_gated_backward_as<true, false>(c);
    return c.gelu ? launch_gated_backward_as<false, true>(c) : launch_gated_backward_as<false, false>(c);
}

}  // namespace tq
