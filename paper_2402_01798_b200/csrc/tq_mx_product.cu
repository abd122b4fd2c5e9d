// Products of microscaled 4-bit matrices on the tensor cores: C = A B^T, and both projections of a gated feed-forward block with
// its activation and the product of the two.
#include <cuda.h>

#include "tq_mx.cuh"

namespace tq {

namespace {

// ---- tcgen05 ---------------------------------------------------------------------------------------------------
// Shared-memory matrix descriptor: rows of 128 bytes, 128-byte swizzle, 8 rows every 1024 bytes (what a TMA load with
// that swizzle leaves behind).  Bits 0-13 address / 16, 32-45 byte offset of the next 8 rows / 16, 46-48 the constant 1, 61-63 swizzle.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFF) >> 4) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// 32 rows of 16 bytes, one after another: no swizzle, 8 rows every 128 bytes.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFF) >> 4) | (static_cast<uint64_t>(128 >> 4) << 32) | (1ull << 46);
}
// Instruction descriptor of kind::mxf4: both operands E2M1 (1) and K-major, E8M0 scales, M = 128, N; `id` = 0 or 2, the pair of bytes of the
// scale columns that this step of 64 elements takes.
__device__ __forceinline__ uint32_t mxf4_desc(uint32_t n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24) | (id << 29);
}
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {       // 128 x 4 scales -> 4 columns, in all four quarters
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// 32 columns of this warp's 32 lanes: thread l gets lane l
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// A tile of a tensor map into this block's shared memory; x in bytes, a multiple of 16.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

__device__ unsigned int g_product_wait_expired = 0;       // blocks whose bounded wait ran out, since load

// A bounded wait that also ends when another thread of the block has given up.
__device__ __forceinline__ bool wait_or_dead(uint32_t bar, uint32_t parity, volatile int* dead) {
    for (uint32_t it = 0; it < kWaitLimit; ++it) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((it & 255u) == 255u && *dead) return false;
    }
    *dead = 1;
    return false;
}

// ---- the kernel for many rows ------------------------------------------------------------------------------------
constexpr int kBM = 128, kBN = 256, kBK = 256;                   // rows of A, rows of B, elements of both in a stage
constexpr int kStages = 4;
constexpr uint32_t kABytes = kBM * kBK / 2, kBBytes = kBN * kBK / 2, kSABytes = kBM * kBK / 32, kSBBytes = kBN * kBK / 32;
constexpr uint32_t kStageBytes = kABytes + kBBytes + kSABytes + kSBBytes;
constexpr uint32_t kScaleColumns = 24;                           // of tensor memory, per stage: 2 x 4 for A, 2 x 8 for B
constexpr uint32_t kProductSmem = kStages * kStageBytes + 1024 + 256;
constexpr int kProductThreads = 192;

struct ProductArgs {
    const uint8_t *a_scales, *b0_scales, *b1_scales;             // in tiles
    uint64_t a_band, b0_band, b1_band;                           // bytes between 128 rows
    uint32_t m, n, k;                                            // n: columns of C, or features
    uint32_t tiles_m, tiles_n;
    void* out;                                                   // C, or the two projections (may be null)
    uint64_t out_stride;
    uint32_t out_bf16, out_wide;                                 // wide: rows start on 16-byte boundaries
    MxView h;                                                    // gated only
};

// 32 consecutive elements of one row.
__device__ __forceinline__ void store32(const ProductArgs& p, uint64_t row, uint64_t col, const float (&v)[32], uint32_t n, uint64_t offset) {
    if (p.out_bf16) {
        unsigned short* to = static_cast<unsigned short*>(p.out) + row * p.out_stride + offset + col;
        if (p.out_wide && col + 32 <= n) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                stg128(to + 8 * i, make_uint4(pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]), pack_bf16(v[8 * i + 4], v[8 * i + 5]),
                                              pack_bf16(v[8 * i + 6], v[8 * i + 7])));
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i < n) to[i] = static_cast<unsigned short>(pack_bf16(v[i], 0.0f));
        }
    } else {
        float* to = static_cast<float*>(p.out) + row * p.out_stride + offset + col;
        if (p.out_wide && col + 32 <= n) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                stg128(to + 4 * i, make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i < n) to[i] = v[i];
        }
    }
}

// GATED: 0 a plain product, 1 SiLU, 2 GELU.  One block an SM, over the tiles of the result in turn.  Warp 0 loads, warp 1 multiplies, warps 2 to 5
// take the result out of tensor memory.
template <int GATED>
__global__ void __launch_bounds__(kProductThreads, 1) mx_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b0,
                                                                        const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ ProductArgs p) {
    extern __shared__ unsigned char raw[];
    __shared__ volatile int dead;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = base + kStages * kStageBytes;
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto empty = [&](int s) { return bars + 8 * (kStages + s); };
    const uint32_t done = bars + 8 * (2 * kStages), drained = done + 8, flushed = done + 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1); mbar_init(drained, 4); mbar_init(flushed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    pdl_wait();
    const uint32_t tmem = tmem_base;
    const uint32_t tiles = p.tiles_m * p.tiles_n, chunks = (p.k + kBK - 1) / kBK;
    const uint32_t per_tile_n = GATED ? 128 : kBN;

    if (warp == 0 && lane == 0) {
        uint32_t it = 0;
        for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
            const uint32_t tm = t % p.tiles_m, tn = t / p.tiles_m;
            const uint32_t n0 = tn * per_tile_n;
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const int s = it % kStages;
                if (!wait_or_dead(empty(s), ((it / kStages) & 1) ^ 1, &dead)) goto loaded;
                const uint32_t at = base + s * kStageBytes;
                const uint32_t tiles_k = ((p.k + 127) / 128 - 2 * c) < 2 ? 1 : 2;
                const bool second = GATED || n0 + 128 < p.n;
                mbar_expect_tx(full(s), kABytes + kBBytes + tiles_k * 512 * (second ? 3 : 2));
                tma_load(at, &map_a, c * (kBK / 2), tm * kBM, full(s));
                tma_load(at + kABytes, &map_b0, c * (kBK / 2), n0, full(s));
                tma_load(at + kABytes + kBBytes / 2, GATED ? &map_b1 : &map_b0, c * (kBK / 2), GATED ? n0 : n0 + 128, full(s));
                const uint32_t sa = at + kABytes + kBBytes;
                bulk_load(sa, p.a_scales + tm * p.a_band + c * 1024, tiles_k * 512, full(s));
                bulk_load(sa + kSABytes, p.b0_scales + (n0 / 128) * p.b0_band + c * 1024, tiles_k * 512, full(s));
                if (second)
                    bulk_load(sa + kSABytes + 1024, GATED ? p.b1_scales + (n0 / 128) * p.b1_band + c * 1024 : p.b0_scales + (n0 / 128 + 1) * p.b0_band + c * 1024,
                              tiles_k * 512, full(s));
            }
        }
    loaded:
        if (dead)                                                // nothing may still be on its way into a block that ends
            for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j) mbar_wait(full(j % kStages), (j / kStages) & 1);
    } else if (warp == 1 && lane == 0) {
        uint32_t it = 0, n_tile = 0;
        for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x, ++n_tile) {
            const uint32_t n0 = t / p.tiles_m * per_tile_n;
            const uint32_t n = GATED ? 256 : p.n - n0 < 256 ? (p.n - n0 + 15) / 16 * 16 : 256;
            if (!wait_or_dead(drained, (n_tile & 1) ^ 1, &dead)) break;
            fence_after();
            bool ok = true;
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const int s = it % kStages;
                if (!wait_or_dead(full(s), (it / kStages) & 1, &dead)) { ok = false; break; }
                fence_after();
                const uint32_t at = base + s * kStageBytes, sa = at + kABytes + kBBytes;
                const uint32_t scale_a = tmem + 256 + s * kScaleColumns, scale_b = scale_a + 8;
                const uint32_t left = p.k - c * kBK, steps = left >= kBK ? 4 : (left + 63) / 64;
                for (uint32_t j = 0; 2 * j < steps; ++j) {
                    copy_scales(scale_a + 4 * j, scale_desc(sa + 512 * j));
                    copy_scales(scale_b + 8 * j, scale_desc(sa + kSABytes + 512 * j));
                    copy_scales(scale_b + 8 * j + 4, scale_desc(sa + kSABytes + 1024 + 512 * j));
                }
                for (uint32_t i = 0; i < steps; ++i)
                    mma_mxf4(tmem, operand_desc(at + 32 * i), operand_desc(at + kABytes + 32 * i), mxf4_desc(n, (i & 1) * 2), scale_a + 4 * (i >> 1), scale_b + 8 * (i >> 1),
                             (c | i) != 0);
                mma_commit(empty(s));
            }
            if (!ok) break;
            mma_commit(done);
        }
        if (dead) {                                              // let the multiplications that were issued come to an end
            mma_commit(flushed);
            mbar_wait(flushed, 0);
        }
    } else if (warp >= 2) {
        const int quarter = warp % 4;
        uint32_t n_tile = 0;
        for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x, ++n_tile) {
            const uint32_t tm = t % p.tiles_m, tn = t / p.tiles_m;
            if (!__all_sync(0xFFFFFFFFu, wait_or_dead(done, n_tile & 1, &dead))) break;
            fence_after();
            const uint32_t local = quarter * 32 + lane, row = tm * kBM + local;
            const uint32_t from = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
            if constexpr (!GATED) {
#pragma unroll 1
                for (uint32_t j = 0; j < 8; ++j) {
                    const uint32_t col = tn * kBN + 32 * j;
                    if (col >= p.n) break;
                    float v[32];
                    __syncwarp();
                    tmem_load32(from + 32 * j, v);
                    tmem_wait_loads();
                    if (row < p.m) store32(p, row, col, v, p.n, 0);
                }
            } else {
                uint32_t scales = 0;
                const uint32_t f0 = tn * 128;
#pragma unroll 1
                for (uint32_t j = 0; j < 4; ++j) {
                    float g[32], u[32];
                    __syncwarp();
                    tmem_load32(from + 32 * j, g);
                    tmem_load32(from + 128 + 32 * j, u);
                    tmem_wait_loads();
                    const uint32_t f = f0 + 32 * j;
                    if (f < p.n && row < p.m) {
                        if (p.out) {
                            store32(p, row, f, g, p.n, 0);
                            store32(p, row, f, u, p.n, p.n);
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) g[i] = gate_value<GATED == 2>(g[i]) * u[i];
                        const uint32_t byte = mx_scale_byte<false>(max_abs_32(g));
                        stg128(p.h.codes + row * p.h.code_stride + f / 2, mx_encode32<false>(g, byte, [](int, uint32_t (&)[4]) {}));
                        scales |= byte << (8 * j);
                    }
                }
                // every row of the 128, those behind the last token with zeros
                asm volatile("st.global.b32 [%0], %1;" ::"l"(p.h.scales + tm * p.h.scale_stride + tn * 512 + (local % 32) * 16 + (local / 32) * 4), "r"(scales) : "memory");
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(drained);
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && dead) atomicAdd(&g_product_wait_expired, 1u);
    fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ---- host ------------------------------------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static std::atomic<void*> known{nullptr};
    void* f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult found{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
        known.store(f, std::memory_order_relaxed);
    }
    return reinterpret_cast<EncodeTiled>(f);
}
// The codes as bytes, in boxes of `rows` rows x 128 bytes (256 elements); what lies outside reads as zero.
cudaError_t codes_map(CUtensorMap* map, const tq_mx_t& m, uint32_t rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t size[2] = {(m.cols + 31) / 32 * 16, m.rows}, stride[1] = {m.code_stride};
    const cuuint32_t box[2] = {128, rows}, step[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.codes, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int GATED>
cudaError_t launch_product_as(const CUtensorMap& a, const CUtensorMap& b0, const CUtensorMap& b1, const ProductArgs& p, cudaStream_t stream) {
    auto* kernel = mx_product_kernel<GATED>;
    if (const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem)) return e;
    const uint32_t tiles = p.tiles_m * p.tiles_n, sms = static_cast<uint32_t>(sm_count());
    return launch_kernel(kernel, dim3(tiles < sms ? tiles : sms), kProductThreads, kProductSmem, stream, a, b0, b1, p);
}

}  // namespace

cudaError_t read_product_wait_expired(unsigned int* count) { return cudaMemcpyFromSymbol(count, g_product_wait_expired, sizeof(unsigned int)); }

cudaError_t launch_mx_product(const tq_mx_t& a, const tq_mx_t& b, void* out, bool bf16, uint64_t out_stride, cudaStream_t stream) {
    CUtensorMap map_a, map_b;
    if (const cudaError_t e = codes_map(&map_a, a, kBM)) return e;
    if (const cudaError_t e = codes_map(&map_b, b, 128)) return e;
    ProductArgs p{};
    p.a_scales = a.scales; p.a_band = a.scale_stride; p.b0_scales = b.scales; p.b0_band = b.scale_stride;
    p.m = static_cast<uint32_t>(a.rows); p.n = static_cast<uint32_t>(b.rows); p.k = static_cast<uint32_t>(a.cols);
    p.tiles_m = (p.m + kBM - 1) / kBM; p.tiles_n = (p.n + kBN - 1) / kBN;
    p.out = out; p.out_stride = out_stride; p.out_bf16 = bf16;
    p.out_wide = (reinterpret_cast<uintptr_t>(out) | (p.m > 1 ? out_stride * (bf16 ? 2 : 4) : 0)) % 16 == 0;
    return launch_product_as<0>(map_a, map_b, map_b, p, stream);
}

cudaError_t launch_mx_gated(const MxGatedCall& c) {
    CUtensorMap map_x, map_g, map_u;
    if (const cudaError_t e = codes_map(&map_x, *c.x, kBM)) return e;
    if (const cudaError_t e = codes_map(&map_g, *c.w_gate, 128)) return e;
    if (const cudaError_t e = codes_map(&map_u, *c.w_up, 128)) return e;
    ProductArgs p{};
    p.a_scales = c.x->scales; p.a_band = c.x->scale_stride;
    p.b0_scales = c.w_gate->scales; p.b0_band = c.w_gate->scale_stride;
    p.b1_scales = c.w_up->scales; p.b1_band = c.w_up->scale_stride;
    p.m = static_cast<uint32_t>(c.x->rows); p.n = static_cast<uint32_t>(c.w_gate->rows); p.k = static_cast<uint32_t>(c.x->cols);
    p.tiles_m = (p.m + kBM - 1) / kBM; p.tiles_n = (p.n + 127) / 128;
    p.out = c.projections; p.out_stride = c.proj_stride; p.out_bf16 = c.proj_bf16;
    p.out_wide = (reinterpret_cast<uintptr_t>(c.projections) | (p.m > 1 ? c.proj_stride * (c.proj_bf16 ? 2 : 4) : 0)) % 16 == 0;
    p.h = mx_view(*c.h);
    return c.gelu ? launch_product_as<2>(map_x, map_g, map_u, p, c.stream) : launch_product_as<1>(map_x, map_g, map_u, p, c.stream);
}

}  // namespace tq
