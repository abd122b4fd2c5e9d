// Products of microscaled 4-bit matrices on the tensor cores: C = A B^T, and both projections of a gated feed-forward block with
// its activation and the product of the two.  Every wait inside a kernel is bounded: a block that gives up lets its copies and
// multiplications end, frees its tensor memory and counts itself.
#include <cuda.h>

#include "tq_mx.cuh"
#include "tq_wait.h"

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
// Instruction descriptor of kind::mxf4: both operands E2M1 (1) and K-major, E8M0 scales, M and N of the tile; `id` = 0 or 2, the pair of
// bytes of the scale columns that this step of 64 elements takes.
__device__ __forceinline__ uint32_t mxf4_desc(uint32_t m, uint32_t n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24) | (id << 29);
}
template <bool PAIR>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
}
// 128 x 4 scales -> 4 columns, in all four quarters of tensor memory (of both blocks of a pair, each from its own shared memory)
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// What was issued so far arrives on `bar` when it is done; of a pair, on both blocks' barriers
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(static_cast<unsigned short>(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t to, uint32_t columns) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// N columns of this warp's 32 lanes: thread l gets lane l
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[N]) {
    static_assert(N == 8 || N == 16 || N == 32, "");
    uint32_t r[N];
    if constexpr (N == 8)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
    if constexpr (N == 16)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
    if constexpr (N == 32)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(addr));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// A map itself, ahead of its first use: it is a kernel parameter.
__device__ __forceinline__ void fetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// A tile of a tensor map into this block's shared memory; x in bytes, a multiple of 16.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// The same by a block of a pair; `bar` may be the other block's.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// ---- blocks of a cluster -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t of_rank(uint32_t addr, uint32_t rank) {          // the same place in another block's shared memory
    uint32_t r; asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank)); return r;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// A word of another block's shared memory, at the place of this block's `word`.
__device__ __forceinline__ void tell_block(volatile uint32_t* word, uint32_t rank, uint32_t value) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(of_rank(smem_addr(const_cast<uint32_t*>(word)), rank)), "r"(value) : "memory");
}
// Bytes that are expected and will not come.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ unsigned int g_product_wait_expired = 0;       // blocks whose bounded wait ran out, since load

// A bounded wait that also ends when another thread of the block has given up.  `filled`: stages that the block has asked for so far.  The wait for a sum
// is renewed by them, the waits for a stage hardly ever see more than one.
__device__ __forceinline__ bool wait_or_dead(uint32_t bar, uint32_t parity, volatile int* dead, volatile uint32_t* filled) {
    const bool done = wait_with_progress(
        kWaitLimit,
        [&] {
            uint32_t done;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done) : "r"(bar), "r"(parity) : "memory");
            return done != 0;
        },
        [&] { return *dead != 0; }, [&] { return *filled; });
    if (!done) *dead = 1;
    return done;
}

// The same for all threads of a warp, with one answer.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* dead, volatile uint32_t* filled) {
    return __all_sync(0xFFFFFFFFu, wait_or_dead(bar, parity, dead, filled));
}
// One thread of the warp issues.  The others go through the same loops, so that descriptors, addresses and barriers stay uniform over the warp: computed
// by the one thread alone, they are moved to uniform registers one by one for each instruction, and a multiplication took 223 clocks where 128 are needed.
__device__ __forceinline__ bool elect() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

struct ProductArgs {
    const uint8_t *a_scales, *b0_scales, *b1_scales;             // in tiles
    uint64_t a_band, b0_band, b1_band;                           // bytes between 128 rows
    uint32_t m, n, k;                                            // n: columns of C, or features
    uint32_t tiles_m, tiles_n;
    uint32_t group;                                              // of tiles in m (pair kernel)
    uint32_t a_rows;                                             // rows of A in a box
    void* out;                                                   // C, or the two projections (may be null)
    uint64_t out_stride;
    uint32_t out_bf16, out_wide;                                 // rows start on boundaries of this many bytes: 32, 16 or 0 for fewer
    MxView h;                                                    // gated only
};

// WIDTH consecutive elements of 32 rows, one row a thread: `row0` is the warp's first.  Where rows start on 16-byte boundaries and all columns exist
// a thread stores its row; else eight columns at a time change places in `scratch` (the warp's 32 x 9 words), so that eight threads
// store neighbours (32 scattered elements a store took 47 us for 300 x 300 x 8192).
constexpr int kScratchWords = 32 * 9;
template <int WIDTH>
__device__ __forceinline__ void store_rows(const ProductArgs& p, float* scratch, uint64_t row0, uint64_t col, const float (&v)[WIDTH], uint32_t n, uint64_t offset) {
    const uint32_t lane = threadIdx.x & 31;
    if (p.out_wide >= 16 && col + WIDTH <= n) {
        const uint64_t row = row0 + lane;
        if (row >= p.m) return;
        if (p.out_bf16) {
            unsigned short* to = static_cast<unsigned short*>(p.out) + row * p.out_stride + offset + col;
            uint32_t w[WIDTH / 2];
#pragma unroll
            for (int i = 0; i < WIDTH / 2; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            if (WIDTH >= 16 && p.out_wide == 32) {
#pragma unroll
                for (int i = 0; i < WIDTH / 16; ++i) {
                    const uint32_t x[8] = {w[8 * i], w[8 * i + 1], w[8 * i + 2], w[8 * i + 3], w[8 * i + 4], w[8 * i + 5], w[8 * i + 6], w[8 * i + 7]};
                    stg256_words(to + 16 * i, x);
                }
            } else {
#pragma unroll
                for (int i = 0; i < WIDTH / 8; ++i) stg128(to + 8 * i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
            }
        } else {
            float* to = static_cast<float*>(p.out) + row * p.out_stride + offset + col;
            if (p.out_wide == 32) {
#pragma unroll
                for (int i = 0; i < WIDTH / 8; ++i) {
                    const float x[8] = {v[8 * i], v[8 * i + 1], v[8 * i + 2], v[8 * i + 3], v[8 * i + 4], v[8 * i + 5], v[8 * i + 6], v[8 * i + 7]};
                    stg256(to + 8 * i, x);
                }
            } else {
#pragma unroll
                for (int i = 0; i < WIDTH / 4; ++i)
                    stg128(to + 4 * i, make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
            }
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < WIDTH / 8; ++q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) scratch[lane * 9 + e] = v[8 * q + e];
        __syncwarp();
        const uint64_t c = col + 8 * q + lane % 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = 4 * i + lane / 8;
            const float x = scratch[r * 9 + lane % 8];
            if (row0 + r < p.m && c < n) {
                const uint64_t to = (row0 + r) * p.out_stride + offset + c;
                if (p.out_bf16) static_cast<unsigned short*>(p.out)[to] = static_cast<unsigned short>(pack_bf16(x, 0.0f));
                else static_cast<float*>(p.out)[to] = x;
            }
        }
        __syncwarp();
    }
}
// A block of h in each of 32 rows from both projections: stores what is kept of them and the codes, returns the scale byte (0 for a row that is not there).
template <bool GELU>
__device__ __forceinline__ uint32_t store_gated(const ProductArgs& p, float* scratch, uint64_t row0, uint64_t f, const float (&g)[32], const float (&u)[32]) {
    if (f >= p.n) return 0;
    if (p.out) {
        store_rows<32>(p, scratch, row0, f, g, p.n, 0);
        store_rows<32>(p, scratch, row0, f, u, p.n, p.n);
    }
    const uint64_t row = row0 + (threadIdx.x & 31);
    if (row >= p.m) return 0;
    float h[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) h[i] = gate_value<GELU>(g[i]) * u[i];
    const uint32_t byte = mx_scale_byte<false>(max_abs_32(h));
    stg128(p.h.codes + row * p.h.code_stride + f / 2, mx_encode32<false>(h, byte, [](int) { return RowBits{}; }));
    return byte;
}

// The scale tiles of the operands as rows of words (pair kernel: bulk copies without a map count on their own block's barriers alone).
struct ScaleMaps {
    CUtensorMap a, b0, b1;
};

constexpr int kBK = 256;                                         // elements of both operands in a stage: 128 bytes a row

// ---- large results ------------------------------------------------------------------------------------------------
// Two blocks on neighbouring SMs make a 256 x 256 tile with one stream of multiplications: each holds 128 rows of A, half of the 256 rows
// of B and 128 rows of the result, so that a stage of 32 KB of codes feeds 4 multiplications of 256 x 256 x 64 (512 clocks at the
// nominal rate).  GATED: the first block holds rows of w_gate and the second the same rows of w_up; the result's columns 0 .. 127
// are g and 128 .. 255 u of the same features.
// Warp 0 of each block loads, and the bytes count on the first block's barrier; its warp 1 multiplies; warps 2 to 9 of both take results out of
// tensor memory, two of them for each quarter of its lanes.  (A message from block to block for every stage, with the ordering of a release over the
// cluster, took 0.8 us a stage: 8192 x 4096 x 16384 in 375 us.)
// Tensor memory: two accumulators of 256 columns that overlap in the middle, at 0 and 112, and the scales of 6 stages from 368 on.  The
// columns that both use are taken out first, and the next tile begins when they are.  The scales have a place for each stage, so that no copy can
// meet a multiplication that still reads them: a stage is only filled again when its multiplications are done.
// 8192^3: 182 us, 6.0 PFLOP/s, the tensor pipe 75 % busy; after a second of it the 1 kW limit lowers the clock and it is 217.  Gated, 8192 tokens, 8192 x 8192, with the projections
// kept: 70 %.
constexpr int kPairStages = 6, kPairThreads = 320;
constexpr uint32_t kPairCodes = 2 * 128 * kBK / 2, kPairStage = kPairCodes + 3 * 1024;       // A, B; scales of 128 rows of A and of 256 rows of B
constexpr uint32_t kPairSmem = kPairStages * kPairStage + 1024 + 256;
constexpr uint32_t kSecond = 112, kPairScales = kSecond + 256, kPairScaleColumns = 24;
static_assert(kPairScales + kPairStages * kPairScaleColumns == 512, "tensor memory has 512 columns");

// Tile t of the result.  The tiles that are worked on at a time are a column of `group` tiles and as many to its right as there are clusters: where both operands fit
// the L2 together the whole height is taken, else 4, so that a wave of tiles reads little of either.  Whole height / 4, us: 8192 x 4096 x 16384, 107 MB of operands, 202 / 180;
// 16384 x 4096 x 8192, 89 MB, 237 / 213; 5400 x 5000 x 16384, 91 MB, 176 / 173; 8192^3, 71 MB, 183 / 188; 8192 x 8192 x 4096, 36 MB, 103 / 104; 4096 x 16384 x 8192, 8192 x 8192 x 10240
// and gated blocks of 71 to 107 MB within 2 % of one another.  It loses where A alone fits: 8192 x 8192 x 12288, 107 MB, 290 / 316.
struct PairTile {
    uint32_t m, n;
    __device__ __forceinline__ PairTile(const ProductArgs& p, uint32_t t) {
        const uint32_t per = p.group * p.tiles_n, first = t / per * p.group, in = t % per, high = p.tiles_m - first < p.group ? p.tiles_m - first : p.group;
        m = first + in % high;
        n = in / high;
    }
};

// GATED: 0 a plain product, 1 SiLU, 2 GELU.
template <int GATED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) mx_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b0,
                                                                                          const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ ScaleMaps maps,
                                                                                          const __grid_constant__ ProductArgs p) {
    extern __shared__ unsigned char raw[];
    __shared__ volatile int dead;
    __shared__ volatile uint32_t filled, ended[2];                                   // ended: of either block, its fillings, and whether it gave up (bit 0)
    __shared__ uint32_t tmem_base;
    __shared__ float scratch[8][kScratchWords];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = base + kPairStages * kPairStage;
    const auto full = [&](int s) { return bars + 8 * s; };                           // first block: the loads of both
    const auto empty = [&](int s) { return bars + 8 * (kPairStages + s); };          // the multiplications have read the stage
    const uint32_t done = bars + 8 * (2 * kPairStages), drained = done + 8, flushed = done + 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        dead = 0;
        filled = 0;
        for (int s = 0; s < kPairStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1); mbar_init(drained, 16); mbar_init(flushed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32 * 9) {
        fetch_map(&map_a); fetch_map(&map_b0); fetch_map(&maps.a); fetch_map(&maps.b0);
        if constexpr (GATED != 0) { fetch_map(&map_b1); fetch_map(&maps.b1); }
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<true>(smem_addr(&tmem_base), 512);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    pdl_wait();
    const uint32_t tmem = tmem_base;
    const uint32_t tiles = p.tiles_m * p.tiles_n, chunks = (p.k + kBK - 1) / kBK, clusters = gridDim.x / 2;
    constexpr uint32_t kWide = GATED ? 128 : 256;                // columns of C, or features, in a tile
    const bool leader = elect();
    uint32_t issued = 0;                                         // warp 0: fillings of stages

    if (warp == 0) {
        uint32_t& it = issued;
        bool ok = true;
        for (uint32_t t = blockIdx.x / 2; t < tiles && ok; t += clusters) {
            const PairTile tile(p, t);
            const uint32_t band = tile.m * 2 + rank, n0 = tile.n * kWide;
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const int s = it % kPairStages;
                if (!(ok = warp_wait(empty(s), ((it / kPairStages) & 1) ^ 1, &dead, &filled))) break;
                if (leader) {
                    const uint32_t at = base + s * kPairStage, scales = at + kPairCodes, bar = of_rank(full(s), 0);
                    if (rank == 0) mbar_expect_tx(full(s), 2 * kPairStage);       // what lies outside the matrices arrives as zeros
                    tma_load_pair(at, &map_a, c * (kBK / 2), band * 128, bar);
                    tma_load_pair(at + kPairCodes / 2, GATED && rank ? &map_b1 : &map_b0, c * (kBK / 2), GATED ? n0 : n0 + rank * 128, bar);
                    tma_load_pair(scales, &maps.a, c * 256, band, bar);
                    tma_load_pair(scales + 1024, &maps.b0, c * 256, n0 / 128, bar);
                    tma_load_pair(scales + 2048, GATED ? &maps.b1 : &maps.b0, c * 256, GATED ? n0 / 128 : n0 / 128 + 1, bar);
                    filled = it + 1;
                }
                __syncwarp();
            }
        }
    } else if (warp == 1 && rank == 0) {
        // The scales of a stage are copied behind the multiplications of the stage before, so that a tile's first are in place when it begins
        // (8192 x 8192 x 512: 36.9 us, with copies in front of their own multiplications 38.6; no difference for long k).
        const auto copy_stage = [&](uint32_t s) {
            const uint32_t scales = base + s * kPairStage + kPairCodes, to = tmem + kPairScales + s * kPairScaleColumns;
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                copy_scales<true>(to + 4 * j, scale_desc(scales + 512 * j));
                copy_scales<true>(to + 8 + 8 * j, scale_desc(scales + 1024 + 512 * j));
                copy_scales<true>(to + 12 + 8 * j, scale_desc(scales + 2048 + 512 * j));
            }
        };
        const uint32_t mine = (tiles - blockIdx.x / 2 + clusters - 1) / clusters, total = mine * chunks;
        const uint32_t last_steps = (p.k - (chunks - 1) * kBK + 63) / 64;
        bool ok = warp_wait(full(0), 0, &dead, &filled);
        if (ok) {
            fence_after();
            if (leader) copy_stage(0);
            __syncwarp();
        }
        for (uint32_t n_tile = 0, it = 0; n_tile < mine && ok; ++n_tile) {
            if (!(ok = warp_wait(drained, (n_tile & 1) ^ 1, &dead, &filled))) break;
            const uint32_t d = tmem + (n_tile & 1) * kSecond;
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const uint32_t s = it % kPairStages, next = (it + 1) % kPairStages;
                const bool more = it + 1 < total;
                if (more && !(ok = warp_wait(full(next), ((it + 1) / kPairStages) & 1, &dead, &filled))) break;
                fence_after();
                if (leader) {
                    const uint64_t a = operand_desc(base + s * kPairStage), b = operand_desc(base + s * kPairStage + kPairCodes / 2);
                    const uint32_t scale_a = tmem + kPairScales + s * kPairScaleColumns, scale_b = scale_a + 8;
                    const uint32_t steps = c + 1 < chunks ? 4 : last_steps;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)             // 64 elements, 32 bytes, are 2 in the address field
                        if (i < steps) mma_mxf4<true>(d, a + 2 * i, b + 2 * i, mxf4_desc(256, 256, (i & 1) * 2), scale_a + 4 * (i >> 1), scale_b + 8 * (i >> 1), (c | i) != 0);
                    if (more) copy_stage(next);
                    mma_commit<true>(empty(s));
                }
                __syncwarp();
            }
            if (ok && leader) mma_commit<true>(done);
            __syncwarp();
        }
    } else if (warp >= 2) {
        const uint32_t quarter = warp % 4, half = (warp - 2) / 4;
        const uint32_t tell = of_rank(drained, 0);
        uint32_t n_tile = 0;
        for (uint32_t t = blockIdx.x / 2; t < tiles; t += clusters, ++n_tile) {
            const PairTile tile(p, t);
            const uint32_t band = tile.m * 2 + rank, n0 = tile.n * kWide;
            if (!warp_wait(done, n_tile & 1, &dead, &filled)) break;
            fence_after();
            const uint32_t local = quarter * 32 + lane, row0 = band * 128 + quarter * 32;
            const uint32_t from = tmem + (n_tile & 1) * kSecond + ((quarter * 32) << 16);
            const auto release = [&] {
                fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(tell);
            };
            if constexpr (!GATED) {
                // the shared columns first: of the first accumulator its last 144, of the second its first
#pragma unroll 1
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t j = n_tile & 1 ? 2 * i + half : 7 - (2 * i + half);
                    float v[32];
                    tmem_load(from + 32 * j, v);
                    tmem_wait_loads();
                    if (i == 2 - half) release();
                    const uint32_t col = n0 + 32 * j;
                    if (col < p.n) store_rows<32>(p, scratch[warp - 2], row0, col, v, p.n, 0);
                    __syncwarp();
                }
            } else {
                uint32_t bytes = 0;
#pragma unroll 1
                for (uint32_t i = 0; i < 2; ++i) {
                    const uint32_t j = 2 * half + i, f = n0 + 32 * j;
                    float g[32], u[32];
                    tmem_load(from + 32 * j, g);
                    tmem_load(from + 128 + 32 * j, u);
                    tmem_wait_loads();
                    if (i == 1) release();
                    bytes |= store_gated<GATED == 2>(p, scratch[warp - 2], row0, f, g, u) << (8 * i);
                    __syncwarp();
                }
                // every row of the 128, those behind the last token with zeros
                if (band * 128 < p.m)
                    asm volatile("st.global.b16 [%0], %1;" ::"l"(p.h.scales + band * p.h.scale_stride + (n0 / 128) * 512 + (local % 32) * 16 + (local / 32) * 4 + 2 * half),
                                 "h"(static_cast<unsigned short>(bytes)) : "memory");
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 0 && leader)
        for (uint32_t r = 0; r < 2; ++r) tell_block(&ended[rank], r, issued << 1 | (dead != 0));
    __syncwarp();
    cluster_sync();                                              // nobody leaves before the other's multiplications and messages are through
    const uint32_t first_ended = ended[0], second_ended = ended[1];
    if ((first_ended | second_ended) & 1) {                      // nor with anything on its way into either
        if (warp == 0 && leader && rank == 0)
            for_outstanding_of_pair(first_ended >> 1, second_ended >> 1, kPairStages, [&](uint32_t s, uint32_t parity, uint32_t by) {
                if (by == 1) mbar_complete_tx(full(s), kPairStage);
                if (by == 2) mbar_expect_tx(full(s), kPairStage);
                mbar_wait(full(s), parity);
            });
        if (warp == 1 && leader) {
            if (rank == 0) mma_commit<true>(flushed);
            mbar_wait(flushed, 0);
        }
        __syncwarp();
        cluster_sync();
    }
    if (threadIdx.x == 0 && dead) atomicAdd(&g_product_wait_expired, 1u);
    fence_after();
    if (warp == 1) tmem_free<true>(tmem, 512);
}

// ---- small results ------------------------------------------------------------------------------------------------------
// Where there are too few 256 x 256 tiles for the GPU (short prompts): tiles of 128 rows of A and 128 rows of B (GATED: of each of
// the two matrices), one for a cluster of `split` blocks that share its columns k.  A slice of the tile's columns belongs to each block.  When all have
// multiplied, every block sends the others their slices of its fp32 sums (remote stores wait for nothing) and keeps its own in registers, and
// each adds up its slice in the order of the blocks.
constexpr int kSplitThreads = 320;
template <int GATED>
struct SplitShape {
    static constexpr uint32_t kN = GATED ? 256 : 128;
    static constexpr uint32_t kCodesA = 128 * kBK / 2, kCodesB = kN * kBK / 2, kScaleBytes = 1024 + (GATED ? 2048 : 1024);
    static constexpr uint32_t kStage = kCodesA + kCodesB + kScaleBytes, kStages = GATED ? 4 : 6;
    static constexpr uint32_t kScales = kN, kScaleColumns = 8 + kN / 16;          // columns of tensor memory
    static constexpr uint32_t kColumns = GATED ? 512 : 256;
    static_assert(kScales + kStages * kScaleColumns <= kColumns, "");
};

// What a block receives from another one: for either half of its slice (a gated block: of 32 features, g and then u), four columns after four columns,
// 16 bytes for each row.  A warp, which holds 32 rows, then sends 512 bytes in a piece (in pieces of 16 bytes, row after row, it took 2 us more a tile).
template <int GATED, int SPLIT>
struct SplitSums {
    static constexpr int kSlice = 128 / SPLIT;                                    // columns of C, or features
    static constexpr int kWidth = GATED ? 32 : kSlice / 2;                        // of them a thread's
    static constexpr int kHalves = kSlice / kWidth;                               // gated, four blocks: one
    static constexpr uint32_t kRowBytes = kWidth * 4 * (GATED ? 2 : 1);
};

__device__ __forceinline__ float4 load_shared4(uint32_t addr) {
    float4 v; asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory"); return v;
}

template <int GATED, int SPLIT>
__global__ void __launch_bounds__(kSplitThreads, 1) mx_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b0,
                                                                    const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ ProductArgs p, uint32_t stages) {
    using S = SplitShape<GATED>;
    extern __shared__ unsigned char raw[];
    __shared__ volatile int dead;
    __shared__ volatile uint32_t filled, failed;                  // failed: a block of the cluster gave up
    __shared__ uint32_t tmem_base;
    __shared__ __align__(8) uint64_t barriers[2 * S::kStages + 2];
    __shared__ float scratch[8][kScratchWords];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = smem_addr(barriers);
    const auto full = [&](uint32_t s) { return bars + 8 * s; };
    const auto empty = [&](uint32_t s) { return bars + 8 * (S::kStages + s); };
    const uint32_t done = bars + 8 * (2 * S::kStages), flushed = done + 8;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        dead = 0;
        filled = failed = 0;
        for (uint32_t s = 0; s < stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1); mbar_init(flushed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32 * 9) {
        fetch_map(&map_a); fetch_map(&map_b0);
        if constexpr (GATED != 0) fetch_map(&map_b1);
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<false>(smem_addr(&tmem_base), S::kColumns);
    fence_before();
    __syncthreads();
    fence_after();
    pdl_wait();
    const uint32_t tmem = tmem_base;
    const uint32_t tile = blockIdx.x / SPLIT, rank = blockIdx.x % SPLIT;
    const uint32_t tm = tile % p.tiles_m, n0 = tile / p.tiles_m * 128;
    const uint32_t chunks = (p.k + kBK - 1) / kBK;
    const uint32_t first = chunks * rank / SPLIT, last = chunks * (rank + 1) / SPLIT;       // at least one: SPLIT <= chunks
    constexpr uint32_t at_a = S::kCodesB, at_scales = S::kCodesB + S::kCodesA;              // within a stage
    const bool leader = elect();
    uint32_t issued = 0;                                         // warp 0: fillings of stages

    if (warp == 0) {
        uint32_t s = 0, round = 0;
        for (uint32_t c = first; c < last; ++c, ++issued) {
            if (!warp_wait(empty(s), (round & 1) ^ 1, &dead, &filled)) break;
            if (leader) {
                const uint32_t at = base + s * S::kStage, scales = at + at_scales;
                const uint32_t bytes = (p.k + 127) / 128 - 2 * c < 2 ? 512 : 1024;
                mbar_expect_tx(full(s), S::kCodesA + S::kCodesB + bytes * (GATED ? 3 : 2));
                tma_load(at, &map_b0, c * (kBK / 2), n0, full(s));
                if constexpr (GATED != 0) tma_load(at + S::kCodesB / 2, &map_b1, c * (kBK / 2), n0, full(s));
                tma_load(at + at_a, &map_a, c * (kBK / 2), tm * 128, full(s));
                bulk_load(scales, p.a_scales + tm * p.a_band + c * 1024ull, bytes, full(s));
                bulk_load(scales + 1024, p.b0_scales + (n0 / 128) * p.b0_band + c * 1024ull, bytes, full(s));
                if constexpr (GATED != 0) bulk_load(scales + 2048, p.b1_scales + (n0 / 128) * p.b1_band + c * 1024ull, bytes, full(s));
                filled = issued + 1;
            }
            __syncwarp();
            if (++s == stages) { s = 0; ++round; }
        }
    } else if (warp == 1) {
        const uint32_t n = GATED ? 256 : p.n - n0 < 128 ? (p.n - n0 + 15) / 16 * 16 : 128;
        const uint32_t last_steps = (p.k - (chunks - 1) * kBK + 63) / 64;
        const auto copy_stage = [&](uint32_t s) {                // of a chunk with one tile of scales the second is whatever lies there, and no step takes it
            const uint32_t scales = base + s * S::kStage + at_scales, to = tmem + S::kScales + s * S::kScaleColumns;
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                copy_scales<false>(to + 4 * j, scale_desc(scales + 512 * j));
                copy_scales<false>(to + 8 + S::kN / 32 * j, scale_desc(scales + 1024 + 512 * j));
                if constexpr (GATED != 0) copy_scales<false>(to + 12 + 8 * j, scale_desc(scales + 2048 + 512 * j));
            }
        };
        bool ok = true;
        uint32_t s = 0, round = 0;
        for (uint32_t c = first; c < last; ++c) {
            if (!(ok = warp_wait(full(s), round & 1, &dead, &filled))) break;
            fence_after();
            if (leader) {
                const uint32_t at = base + s * S::kStage;
                const uint32_t scale_a = tmem + S::kScales + s * S::kScaleColumns, scale_b = scale_a + 8;
                const uint32_t steps = c + 1 < chunks ? 4 : last_steps;
                const uint64_t a = operand_desc(at + at_a), b = operand_desc(at);
                copy_stage(s);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)                 // 64 elements, 32 bytes, are 2 in the address field
                    if (i < steps)
                        mma_mxf4<false>(tmem, a + 2 * i, b + 2 * i, mxf4_desc(128, n, (i & 1) * 2), scale_a + 4 * (i >> 1), scale_b + S::kN / 32 * (i >> 1), (c != first) | (i != 0));
                mma_commit<false>(empty(s));
            }
            __syncwarp();
            if (++s == stages) { s = 0; ++round; }
        }
        if (ok && leader) mma_commit<false>(done);
        __syncwarp();
    }
    // Where a wait ran out: lets all that was issued end, before its memory is used again or the block leaves.
    const auto settle = [&] {
        if (dead == 0) return;
        if (warp == 0 && leader) for_outstanding(issued, stages, [&](uint32_t s, uint32_t parity) { mbar_wait(full(s), parity); });
        if (warp == 1 && leader) {
            mma_commit<false>(flushed);
            mbar_wait(flushed, 0);
        }
        __syncwarp();
    };
    // Two warps for each quarter of the lanes.
    const uint32_t quarter = warp % 4, half = (warp - 2) / 4, local = quarter * 32 + lane, row0 = tm * 128 + quarter * 32;
    const uint32_t from = tmem + ((quarter * 32) << 16);
    const uint32_t rows = p.m - tm * 128 < 128 ? p.m - tm * 128 : 128;
    const bool taker = warp >= 2 && quarter * 32 < rows;        // has rows to take out of tensor memory
    bool fine = true;
    if (warp >= 2) {
        fine = warp_wait(done, 0, &dead, &filled);
        fence_after();
    }
    if constexpr (GATED != 0) {
        // the scales' tile is written for all 128 rows, those behind the last token with zeros
        uint8_t* const tail = p.h.scales + tm * p.h.scale_stride + (n0 / 128) * 512;
        for (uint32_t item = threadIdx.x; item < (128 - rows) * (4 / SPLIT); item += kSplitThreads) {
            const uint32_t r = rows + item / (4 / SPLIT);
            tail[(r % 32) * 16 + (r / 32) * 4 + rank * (4 / SPLIT) + item % (4 / SPLIT)] = 0;
        }
    }
    const auto put_scale = [&](uint32_t r, uint32_t j, uint32_t byte) {              // of row r and block j of the tile
        p.h.scales[tm * p.h.scale_stride + (n0 / 128) * 512 + (r % 32) * 16 + (r / 32) * 4 + j] = static_cast<uint8_t>(byte);
    };
    if constexpr (SPLIT == 1) {
        if (taker && fine) {
#pragma unroll 1
            for (uint32_t j = half; j < 4; j += 2) {
                const uint32_t col = n0 + 32 * j;
                float v[32];
                tmem_load(from + 32 * j, v);
                if constexpr (!GATED) {
                    tmem_wait_loads();
                    if (col < p.n) store_rows<32>(p, scratch[warp - 2], row0, col, v, p.n, 0);
                } else {
                    float u[32];
                    tmem_load(from + 128 + 32 * j, u);
                    tmem_wait_loads();
                    const uint32_t byte = store_gated<GATED == 2>(p, scratch[warp - 2], row0, col, v, u);
                    if (local < rows) put_scale(local, j, byte);
                }
                __syncwarp();
            }
        }
    } else {
        using Q = SplitSums<GATED, SPLIT>;
        const uint32_t part = rows * Q::kRowBytes, quad = rows * 16;                 // bytes from one half, or four columns, to the next
        const auto received = [&](uint32_t b, uint32_t h, uint32_t r) { return base + (b * Q::kHalves + h) * part + r * 16; };
        const auto send = [&](uint32_t owner, uint32_t h) {
            float v[Q::kWidth];
            const uint32_t to = of_rank(received(rank, h, local), owner);
#pragma unroll
            for (int w = 0; w < (GATED ? 2 : 1); ++w) {
                tmem_load(from + owner * Q::kSlice + h * Q::kWidth + 128 * w, v);
                tmem_wait_loads();
                if (local < rows)
#pragma unroll
                    for (int i = 0; i < Q::kWidth; i += 4)
                        asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(to + (w * Q::kWidth + i) / 4 * quad), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]) : "memory");
                __syncwarp();
            }
        };
        __syncthreads();
        settle();
        cluster_sync();                                          // all blocks have multiplied: the stages are free
        if (dead != 0 && threadIdx.x < SPLIT) tell_block(&failed, threadIdx.x, 1);
        if (taker && fine) {
#pragma unroll 1
            for (uint32_t i = 0; i < SPLIT; ++i) {
                const uint32_t owner = (rank + 1 + i) % SPLIT;
                if (owner == rank) continue;
                if (Q::kHalves == 2) send(owner, half);
                else if ((i & 1) == half) send(owner, 0);
            }
        }
        __syncthreads();
        cluster_sync();
        if (taker && !failed && half < Q::kHalves) {
            const uint32_t col = n0 + rank * Q::kSlice + half * Q::kWidth;
            float v[Q::kWidth];
            const auto add_up = [&](float (&x)[Q::kWidth], uint32_t first_quad) {        // what the own block has in x with the others', in their order
#pragma unroll
                for (int i = 0; i < Q::kWidth; i += 4) {
                    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (uint32_t b = 0; b < SPLIT; ++b) {
                        float4 y = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                        if (b != rank && local < rows) y = load_shared4(received(b, half, local) + (first_quad + i / 4) * quad);
                        sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
                    }
                    x[i] = sum.x; x[i + 1] = sum.y; x[i + 2] = sum.z; x[i + 3] = sum.w;
                }
            };
            tmem_load(from + rank * Q::kSlice + half * Q::kWidth, v);
            tmem_wait_loads();
            add_up(v, 0);
            if constexpr (!GATED) {
                if (col < p.n) store_rows<Q::kWidth>(p, scratch[warp - 2], row0, col, v, p.n, 0);
            } else {
                float u[32];
                tmem_load(from + 128 + rank * Q::kSlice + half * Q::kWidth, u);
                tmem_wait_loads();
                add_up(u, 8);
                const uint32_t byte = store_gated<GATED == 2>(p, scratch[warp - 2], row0, col, v, u);
                if (local < rows) put_scale(local, rank * Q::kHalves + half, byte);
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if constexpr (SPLIT == 1) settle();
    if (threadIdx.x == 0 && dead) atomicAdd(&g_product_wait_expired, 1u);
    fence_after();
    if (warp == 1) tmem_free<false>(tmem, S::kColumns);
}

// ---- few rows of A: single tokens ------------------------------------------------------------------------------------------
// 1 x 8192 x 4096: 4.9 us, of which an empty one takes 2.4; gated 1 x 4096 x 8192 6.7.
// Up to 64 rows of A are the narrow operand here: a multiplication of 128 rows of B by 8 to 64 rows of A, k shared by a cluster of SPLIT blocks.  What counts is
// that every SM reads B as fast as it can: with A's rows on the wide side, four multiplications of 128 x 128 x 64 and their scales took 540 clocks for
// 16 KB of B (1 x 8192 x 8192 read 2.5 TB/s).  Two blocks an SM, so that one loads while the other starts or ends.
// A thread of the epilogue has one column of C, or feature, for all rows; 32 features of a row are a warp's, and so is their block of h.
constexpr uint32_t kMostTokens = 64;
// Beyond, the activation of one row after another takes too long.  This kernel / split blocks, us: 8 x 1024 x 2048 5.0 / 6.2, 16 6.3 / 6.2, 24 7.0 / 5.8, 64 12 / 5.6; 16 x 4096 x 8192
// 8.1 / 10, 24 9.0 / 10, 32 10 / 10, 64 14 / 8.8; 16 x 2048 x 16384 8.9 / 9.6, 24 9.9 / 9.6, 64 16 / 8.9; 16 x 8192 x 8192 11 / 16, 32 13 / 11.  Without a gate: 48 x 1000 x 4000 4.8 / 5.5, 64 5.2 / 5.7;
// 48 x 8192 x 4096 6.8 / 7.4, 64 7.5 / 6.6; 32 x 4096 x 8192 6.5 / 6.6, 64 8.0 / 7.0; 16 x 16384 x 2048 5.4 / 6.5, 64 7.6 / 5.9.
constexpr uint32_t kMostGatedTokens = 16;
template <int GATED>
struct TokenShape {
    static constexpr uint32_t kCodesB = (GATED ? 256 : 128) * kBK / 2, kScaleBytes = (GATED ? 3 : 2) * 1024;
    static constexpr uint32_t kMostStages = GATED ? 5 : 8, kMostSmem = 108 * 1024;
    static constexpr uint32_t kScales = 128, kScaleColumns = GATED ? 24 : 16, kColumns = 256;       // of tensor memory; sums in the first 128
    static_assert(kScales + kMostStages * kScaleColumns <= kColumns, "");
    __host__ __device__ static uint32_t stage(uint32_t a_rows) { return kCodesB + a_rows * 128 + kScaleBytes; }
};

// The bytes of 8 codes are in lanes 0, 8, 16 and 24: one element a thread.
__device__ __forceinline__ uint32_t e2m1_of_warp(float y) {
    const float v[8] = {y, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t lane = threadIdx.x & 31;
    return __reduce_or_sync(0xFFu << (lane & 24), e2m1_nearest8(v) << (4 * (lane & 7)));
}
__device__ __forceinline__ float load_shared(uint32_t addr) { float v; asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory"); return v; }
__device__ __forceinline__ void store_one(const ProductArgs& p, uint64_t at, float x) {
    if (p.out_bf16) static_cast<unsigned short*>(p.out)[at] = static_cast<unsigned short>(pack_bf16(x, 0.0f));
    else static_cast<float*>(p.out)[at] = x;
}
// Row r, 32 features from f on, one a thread.
template <bool GELU>
__device__ __forceinline__ void store_gated_warp(const ProductArgs& p, uint32_t r, uint32_t f, float g, float u) {
    const uint32_t lane = threadIdx.x & 31;
    if (f >= p.n) return;
    if (p.out) {
        store_one(p, r * p.out_stride + f + lane, g);
        store_one(p, r * p.out_stride + p.n + f + lane, u);
    }
    const float x = gate_value<GELU>(g) * u;
    // a NaN's pattern without its sign is above infinity's, and that above all others
    const uint32_t byte = mx_scale_byte<false>(__uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x) & 0x7FFFFFFFu)));
    const uint32_t codes = e2m1_of_warp(x * mx_inv_scale(byte));
    if ((lane & 7) == 0)
        asm volatile("st.global.b32 [%0], %1;" ::"l"(p.h.codes + r * p.h.code_stride + f / 2 + lane / 2), "r"(byte == 255u ? 0u : codes) : "memory");
    if (lane == 0) p.h.scales[mx_scale_at(p.h, r, f / 32)] = static_cast<uint8_t>(byte);
}

template <int GATED, int SPLIT>
__global__ void __launch_bounds__(kSplitThreads, 2) mx_token_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b0,
                                                                    const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ ProductArgs p, uint32_t stages) {
    using S = TokenShape<GATED>;
    constexpr int kSums = GATED ? 2 : 1;
    extern __shared__ unsigned char raw[];
    __shared__ volatile int dead;
    __shared__ volatile uint32_t filled, failed;                  // failed: a block of the cluster gave up
    __shared__ uint32_t tmem_base;
    __shared__ __align__(8) uint64_t barriers[2 * S::kMostStages + 2];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = smem_addr(barriers);
    const auto full = [&](uint32_t s) { return bars + 8 * s; };
    const auto empty = [&](uint32_t s) { return bars + 8 * (S::kMostStages + s); };
    const uint32_t done = bars + 8 * (2 * S::kMostStages), flushed = done + 8;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        dead = 0;
        filled = failed = 0;
        for (uint32_t s = 0; s < stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1); mbar_init(flushed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32 * 9) {
        fetch_map(&map_a); fetch_map(&map_b0);
        if constexpr (GATED != 0) fetch_map(&map_b1);
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<false>(smem_addr(&tmem_base), S::kColumns);
    fence_before();
    __syncthreads();
    fence_after();
    pdl_wait();
    const uint32_t tmem = tmem_base;
    const uint32_t rank = blockIdx.x % SPLIT, n0 = blockIdx.x / SPLIT * 128;
    const uint32_t chunks = (p.k + kBK - 1) / kBK;
    const uint32_t first = chunks * rank / SPLIT, last = chunks * (rank + 1) / SPLIT;       // at least one: SPLIT <= chunks
    const uint32_t stage_bytes = S::stage(p.a_rows), at_scales = S::kCodesB + p.a_rows * 128;     // scales of A, B and B's second matrix
    const bool leader = elect();
    uint32_t issued = 0;                                         // warp 0: fillings of stages

    if (warp == 0) {
        uint32_t s = 0, round = 0;
        for (uint32_t c = first; c < last; ++c, ++issued) {
            if (!warp_wait(empty(s), (round & 1) ^ 1, &dead, &filled)) break;
            if (leader) {
                const uint32_t at = base + s * stage_bytes, scales = at + at_scales;
                const uint32_t bytes = (p.k + 127) / 128 - 2 * c < 2 ? 512 : 1024;
                mbar_expect_tx(full(s), S::kCodesB + p.a_rows * 128 + bytes * (1 + kSums));
                tma_load(at, &map_b0, c * (kBK / 2), n0, full(s));
                if constexpr (GATED != 0) tma_load(at + S::kCodesB / 2, &map_b1, c * (kBK / 2), n0, full(s));
                bulk_load(scales + 1024, p.b0_scales + (n0 / 128) * p.b0_band + c * 1024ull, bytes, full(s));
                if constexpr (GATED != 0) bulk_load(scales + 2048, p.b1_scales + (n0 / 128) * p.b1_band + c * 1024ull, bytes, full(s));
                tma_load(at + S::kCodesB, &map_a, c * (kBK / 2), 0, full(s));
                bulk_load(scales, p.a_scales + c * 1024ull, bytes, full(s));
                filled = issued + 1;
            }
            __syncwarp();
            if (++s == stages) { s = 0; ++round; }
        }
    } else if (warp == 1) {
        const uint32_t last_steps = (p.k - (chunks - 1) * kBK + 63) / 64;
        uint32_t s = 0, round = 0;
        bool ok = true;
        for (uint32_t c = first; c < last; ++c) {
            if (!(ok = warp_wait(full(s), round & 1, &dead, &filled))) break;
            fence_after();
            if (leader) {
                const uint32_t at = base + s * stage_bytes, scales = at + at_scales;
                const uint32_t columns = tmem + S::kScales + s * S::kScaleColumns;           // 2 x 4 of A, 2 x 4 of B, 2 x 4 of B's second matrix
                const uint32_t steps = c + 1 < chunks ? 4 : last_steps;
                const uint64_t a = operand_desc(at + S::kCodesB), b = operand_desc(at), b1 = operand_desc(at + S::kCodesB / 2);
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j)                 // of a chunk with one tile of scales the second is whatever lies there, and no step takes it
#pragma unroll
                    for (uint32_t w = 0; w < 1 + kSums; ++w) copy_scales<false>(columns + 8 * w + 4 * j, scale_desc(scales + 1024 * w + 512 * j));
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)                 // 64 elements, 32 bytes, are 2 in the address field
                    if (i < steps) {
                        const uint32_t idesc = mxf4_desc(128, p.a_rows, (i & 1) * 2), more = (c != first) | (i != 0);
                        mma_mxf4<false>(tmem, b + 2 * i, a + 2 * i, idesc, columns + 8 + 4 * (i >> 1), columns + 4 * (i >> 1), more);
                        if constexpr (GATED != 0) mma_mxf4<false>(tmem + kMostTokens, b1 + 2 * i, a + 2 * i, idesc, columns + 16 + 4 * (i >> 1), columns + 4 * (i >> 1), more);
                    }
                mma_commit<false>(empty(s));
            }
            __syncwarp();
            if (++s == stages) { s = 0; ++round; }
        }
        if (ok && leader) mma_commit<false>(done);
        __syncwarp();
    }
    // Where a wait ran out: lets all that was issued end, before its memory is used again or the block leaves.
    const auto settle = [&] {
        if (dead == 0) return;
        if (warp == 0 && leader) for_outstanding(issued, stages, [&](uint32_t s, uint32_t parity) { mbar_wait(full(s), parity); });
        if (warp == 1 && leader) {
            mma_commit<false>(flushed);
            mbar_wait(flushed, 0);
        }
        __syncwarp();
    };
    // Two warps for each quarter of the lanes, 32 columns or features: they take eight rows in turn.
    const uint32_t quarter = warp % 4, half = (warp - 2) / 4;
    const uint32_t from = tmem + ((quarter * 32) << 16);
    bool fine = true;
    if (warp >= 2) {
        fine = warp_wait(done, 0, &dead, &filled);
        fence_after();
    }
    if constexpr (GATED != 0) {
        // the scales' tile is written for all 128 rows, those behind the last token with zeros
        for (uint32_t item = threadIdx.x; item < (128 - p.m) * (4 / SPLIT); item += kSplitThreads) {
            const uint32_t r = p.m + item / (4 / SPLIT), j = rank * (4 / SPLIT) + item % (4 / SPLIT);
            p.h.scales[(n0 / 128) * 512 + (r % 32) * 16 + (r / 32) * 4 + j] = 0;
        }
        // and where the features end inside it, the blocks behind them as well
        for (uint32_t item = threadIdx.x; item < p.m * (4 / SPLIT); item += kSplitThreads) {
            const uint32_t r = item / (4 / SPLIT), j = rank * (4 / SPLIT) + item % (4 / SPLIT);
            if (n0 + 32 * j >= p.n) p.h.scales[(n0 / 128) * 512 + (r % 32) * 16 + (r / 32) * 4 + j] = 0;
        }
    }
    if constexpr (SPLIT == 1) {
        if (warp >= 2 && fine) {
#pragma unroll 1
            for (uint32_t r0 = 8 * half; r0 < p.m; r0 += 16) {
                float v[8], u[8];
                tmem_load(from + r0, v);
                if constexpr (GATED != 0) tmem_load(from + kMostTokens + r0, u);
                tmem_wait_loads();
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    if (r0 + i >= p.m) break;
                    if constexpr (GATED != 0) store_gated_warp<GATED == 2>(p, r0 + i, n0 + 32 * quarter, v[i], u[i]);
                    else if (n0 + 32 * quarter + lane < p.n) store_one(p, (r0 + i) * p.out_stride + n0 + 32 * quarter + lane, v[i]);
                }
                __syncwarp();
            }
        }
    } else {
        constexpr uint32_t kSlice = 128 / SPLIT;                 // columns or features of a block
        // what a block receives: from each block, for each row, its slice of g (or C) and of u
        const auto place = [&](uint32_t b, uint32_t r, uint32_t w, uint32_t col) { return base + (((b * p.m + r) * kSums + w) * kSlice + col) * 4; };
        __syncthreads();
        settle();
        cluster_sync();                                          // all blocks have multiplied: the stages are free
        if (dead != 0 && threadIdx.x < SPLIT) tell_block(&failed, threadIdx.x, 1);
        if (warp >= 2 && fine) {
            const uint32_t col = quarter * 32 + lane, owner = col / kSlice;
#pragma unroll 1
            for (uint32_t r0 = 8 * half; r0 < p.m; r0 += 16) {
#pragma unroll
                for (uint32_t w = 0; w < kSums; ++w) {
                    float v[8];
                    tmem_load(from + kMostTokens * w + r0, v);
                    tmem_wait_loads();
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i)
                        if (r0 + i < p.m) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(of_rank(place(rank, r0 + i, w, col % kSlice), owner)), "f"(v[i]) : "memory");
                    __syncwarp();
                }
            }
        }
        __syncthreads();
        cluster_sync();
        if constexpr (GATED != 0) {
            constexpr uint32_t kBlocks = kSlice / 32;            // SPLIT is 2 or 4
            for (uint32_t item = warp; item < p.m * kBlocks && !failed; item += kSplitThreads / 32) {
                const uint32_t r = item / kBlocks, j = item % kBlocks;
                float g = 0.0f, u = 0.0f;
#pragma unroll
                for (uint32_t b = 0; b < SPLIT; ++b) { g += load_shared(place(b, r, 0, 32 * j + lane)); u += load_shared(place(b, r, 1, 32 * j + lane)); }
                store_gated_warp<GATED == 2>(p, r, n0 + rank * kSlice + 32 * j, g, u);
            }
        } else {
            for (uint32_t item = threadIdx.x; item < p.m * kSlice && !failed; item += kSplitThreads) {
                const uint32_t r = item / kSlice, col = n0 + rank * kSlice + item % kSlice;
                float x = 0.0f;
#pragma unroll
                for (uint32_t b = 0; b < SPLIT; ++b) x += load_shared(place(b, r, 0, item % kSlice));
                if (col < p.n) store_one(p, r * p.out_stride + col, x);
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if constexpr (SPLIT == 1) settle();
    if (threadIdx.x == 0 && dead) atomicAdd(&g_product_wait_expired, 1u);
    fence_after();
    if (warp == 1) tmem_free<false>(tmem, S::kColumns);
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

// Shared memory of a block that waits in the tensor core's allocator while its cluster waits for it: no more of them on an SM than its tensor memory serves at once,
// or two clusters that hold each other's columns would wait for ever.  Blocks with 256 columns ask for more than a third of an SM's memory, so that two
// fit; those with 512 for so much that nothing of the kind fits beside them.
constexpr size_t kLeastHalf = 77 * 1024, kLeastWhole = 160 * 1024;
struct BlockMemory {
    uint32_t stages;
    size_t bytes;
};
inline size_t at_least(size_t need, size_t least) { return need > least ? need : least; }
template <int GATED>
BlockMemory split_memory(uint32_t rows, uint64_t chunks, uint32_t split) {
    using S = SplitShape<GATED>;
    const uint64_t most = (chunks + split - 1) / split;
    const uint32_t stages = most < S::kStages ? static_cast<uint32_t>(most) : S::kStages, sums = split > 1 ? rows * 128 * 4 * (GATED ? 2 : 1) : 0;
    const uint32_t staged = stages * S::kStage;
    return BlockMemory{stages, at_least((staged > sums ? staged : sums) + 1024, GATED ? kLeastWhole : kLeastHalf)};
}
template <int GATED>
BlockMemory token_memory(uint32_t rows, uint32_t a_rows, uint64_t chunks, uint32_t split) {
    using S = TokenShape<GATED>;
    const uint64_t most = (chunks + split - 1) / split;
    uint32_t stages = S::kMostSmem / S::stage(a_rows);
    if (stages > S::kMostStages) stages = S::kMostStages;
    if (stages > most) stages = static_cast<uint32_t>(most);
    const uint32_t staged = stages * S::stage(a_rows), sums = split > 1 ? rows * 128 * 4 * (GATED ? 2 : 1) : 0;
    return BlockMemory{stages, at_least((staged > sums ? staged : sums) + 1024, kLeastHalf)};
}
constexpr size_t kMostSplitSmem = 212 * 1024, kMostTokenSmem = 109 * 1024;        // of any call, beside a few KB of fixed arrays

// Which kernel, and how many blocks share a tile: by an estimate of the time in ns, fitted to graphs of 20 launches.  A pair takes 430 a stage and 1300 a
// tile at least; a split block 310 (two B matrices: 365) and up to 70 more as the SMs fill.  Adding up costs 1 us and 4 ns for each row and block.
// Measured (pair / split 1 / 2 / 4 / 8, us; a graph of 20): 65 x 1024 x 1024 5.4 / 3.6 / 4.5 / 4.3, 128 x 4096 x 4096 9.8 / 7.7 / 7.2 / 6.7 / 9.3, 128 x 16384 x 2048 8.5 / 5.8 / 12 / 16 / 32,
// 128 x 4096 x 16384 24 / 22 / 15 / 11 / 22, 250 x 1024 x 4096 9.3 / 7.4 / 6.9 / 6.2 / 8.1, 777 x 1000 x 4000 10.4 / 8.6 / 7.7 / 13 / 17, 512 x 8192 x 2048 8.6 / 11 / 24 / 31 / 61,
// 1024 x 2048 x 4096 10 / 8.5 / 15 / 26 / 35, 2048 x 2048 x 512 6.6 / 7.6 / 14, 2048^3 8.6 / 11 / 24 / 31 / 61, gated 65 x 4096 x 8192 11 / 9.6 / 8.9 / 17, gated 512 x 4096 x 8192 18 / 20 / 38 / 73.
// Of 35 such shapes it takes the fastest, or one within 5 %, in 33; eight blocks would be better for 256 x 256 x 8192 (7.2, 6.2) and 300 x 300 x 8192 (7.7, 6.8).
struct ProductPlan {
    bool pair;
    uint32_t split;
};
template <int GATED>
ProductPlan plan_product(uint32_t m, uint32_t n, uint32_t k) {
    const uint64_t sms = static_cast<uint64_t>(sm_count()), chunks = (static_cast<uint64_t>(k) + kBK - 1) / kBK;
    const uint64_t wide = (static_cast<uint64_t>(m) + 255) / 256 * ((static_cast<uint64_t>(n) + (GATED ? 127 : 255)) / (GATED ? 128 : 256)), pairs = sms / 2;
    const uint64_t tile = chunks * 430 > 1300 ? chunks * 430 : 1300;
    uint64_t best = 3500 + (wide + pairs - 1) / pairs * tile;
    ProductPlan plan{true, 1};
    const uint64_t narrow = (static_cast<uint64_t>(m) + 127) / 128 * ((static_cast<uint64_t>(n) + 127) / 128);
    const uint32_t rows = m < 128 ? m : 128;
    for (uint32_t split = 1; split <= (GATED ? 4u : 8u) && split <= chunks; split *= 2) {
        const uint64_t room = split == 8 ? sms * 7 / 8 : sms, blocks = narrow * split;
        const uint64_t waves = (blocks + room - 1) / room, stage = (GATED ? 365 : 310) + 70 * (blocks < sms ? blocks : sms) / sms;
        const uint64_t sums = split == 1 ? 500 : 800 + 100 * split + 4 * rows * split;
        const uint64_t cost = 2600 + waves * ((chunks + split - 1) / split * stage + sums) + (waves - 1) * 1500;
        if (cost < best) { best = cost; plan = ProductPlan{false, split}; }
    }
    return plan;
}
// Blocks a tile for few rows: as many as fit on the GPU at once, two on an SM, while each has two stages at least.
template <int GATED>
uint32_t plan_tokens(uint32_t n, uint32_t k) {
    const uint64_t tiles = (static_cast<uint64_t>(n) + 127) / 128, chunks = (static_cast<uint64_t>(k) + kBK - 1) / kBK, room = 2 * static_cast<uint64_t>(sm_count());
    uint32_t split = 1;
    while (split < (GATED ? 4u : 8u) && tiles * split * 2 <= room && chunks >= split * 4) split *= 2;
    return split;
}

// `most`: of shared memory, for any call
template <auto KERNEL>
cudaError_t launch_clustered(unsigned blocks, unsigned cluster, unsigned threads, size_t smem, size_t most, cudaStream_t stream, void** args) {
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared_memory(KERNEL, most, allowed)) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream; cfg.attrs = attr; cfg.numAttrs = cluster ? 2 : 1;
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(KERNEL), args);
}

// Scale tiles, two at a time.
cudaError_t scales_map(CUtensorMap* map, const tq_mx_t& m) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t size[2] = {(m.cols + 127) / 128 * 128, (m.rows + 127) / 128}, stride[1] = {m.scale_stride};
    const cuuint32_t box[2] = {256, 1}, step[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, m.scales, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int GATED, int SPLIT, bool TOKENS>
cudaError_t launch_split_as(const CUtensorMap& map_a, const CUtensorMap& map_b0, const CUtensorMap& map_b1, const ProductArgs& p, cudaStream_t stream) {
    const uint64_t chunks = (static_cast<uint64_t>(p.k) + kBK - 1) / kBK;
    BlockMemory mem = TOKENS ? token_memory<GATED>(p.m, p.a_rows, chunks, SPLIT) : split_memory<GATED>(p.m < 128 ? p.m : 128, chunks, SPLIT);
    void* args[] = {const_cast<CUtensorMap*>(&map_a), const_cast<CUtensorMap*>(&map_b0), const_cast<CUtensorMap*>(&map_b1), const_cast<ProductArgs*>(&p), &mem.stages};
    const unsigned blocks = p.tiles_m * p.tiles_n * SPLIT;
    if constexpr (TOKENS) return launch_clustered<mx_token_kernel<GATED, SPLIT>>(blocks, SPLIT, kSplitThreads, mem.bytes, kMostTokenSmem, stream, args);
    else return launch_clustered<mx_split_kernel<GATED, SPLIT>>(blocks, SPLIT, kSplitThreads, mem.bytes, kMostSplitSmem, stream, args);
}
template <int GATED, bool TOKENS>
cudaError_t launch_split(uint32_t split, const CUtensorMap& map_a, const CUtensorMap& map_b0, const CUtensorMap& map_b1, const ProductArgs& p, cudaStream_t stream) {
    if (split == 2) return launch_split_as<GATED, 2, TOKENS>(map_a, map_b0, map_b1, p, stream);
    if (split == 4) return launch_split_as<GATED, 4, TOKENS>(map_a, map_b0, map_b1, p, stream);
    if constexpr (!GATED) if (split == 8) return launch_split_as<0, 8, TOKENS>(map_a, map_b0, map_b1, p, stream);
    return launch_split_as<GATED, 1, TOKENS>(map_a, map_b0, map_b1, p, stream);
}

template <int GATED>
cudaError_t launch_product_as(const tq_mx_t& a, const tq_mx_t& b0, const tq_mx_t& b1, ProductArgs p, cudaStream_t stream) {
    p.a_scales = a.scales; p.a_band = a.scale_stride;
    p.b0_scales = b0.scales; p.b0_band = b0.scale_stride;
    p.b1_scales = b1.scales; p.b1_band = b1.scale_stride;
    p.m = static_cast<uint32_t>(a.rows); p.n = static_cast<uint32_t>(b0.rows); p.k = static_cast<uint32_t>(a.cols);
    const uint64_t at = reinterpret_cast<uintptr_t>(p.out) | (p.m > 1 ? p.out_stride * (p.out_bf16 ? 2 : 4) : 0) | (GATED ? p.n * (p.out_bf16 ? 2 : 4) : 0);
    p.out_wide = at % 32 == 0 ? 32 : at % 16 == 0 ? 16 : 0;
    const bool tokens = p.m <= (GATED ? kMostGatedTokens : kMostTokens);
    const ProductPlan plan = tokens ? ProductPlan{false, plan_tokens<GATED>(p.n, p.k)} : plan_product<GATED>(p.m, p.n, p.k);
    p.a_rows = tokens ? (p.m + 7) / 8 * 8 : 128;
    CUtensorMap map_a, map_b0, map_b1;
    if (const cudaError_t e = codes_map(&map_a, a, p.a_rows)) return e;
    if (const cudaError_t e = codes_map(&map_b0, b0, 128)) return e;
    if (GATED) {
        if (const cudaError_t e = codes_map(&map_b1, b1, 128)) return e;
    } else {
        map_b1 = map_b0;
    }
    if (plan.pair) {
        p.tiles_m = (p.m + 255) / 256; p.tiles_n = (p.n + (GATED ? 127 : 255)) / (GATED ? 128 : 256);
        const uint64_t operands = (static_cast<uint64_t>(p.m) + static_cast<uint64_t>(p.n) * (GATED ? 2 : 1)) * p.k * 17 / 32;
        p.group = operands > 80'000'000 && p.tiles_m > 4 ? 4 : p.tiles_m;
        const uint32_t tiles = p.tiles_m * p.tiles_n, pairs = static_cast<uint32_t>(sm_count()) / 2;
        ScaleMaps maps;
        if (const cudaError_t e = scales_map(&maps.a, a)) return e;
        if (const cudaError_t e = scales_map(&maps.b0, b0)) return e;
        maps.b1 = maps.b0;
        if (GATED)
            if (const cudaError_t e = scales_map(&maps.b1, b1)) return e;
        void* args[] = {&map_a, &map_b0, &map_b1, &maps, &p};
        return launch_clustered<mx_pair_kernel<GATED>>(2 * (tiles < pairs ? tiles : pairs), 0, kPairThreads, kPairSmem, kPairSmem, stream, args);
    }
    p.tiles_m = (p.m + 127) / 128; p.tiles_n = (p.n + 127) / 128;
    return tokens ? launch_split<GATED, true>(plan.split, map_a, map_b0, map_b1, p, stream) : launch_split<GATED, false>(plan.split, map_a, map_b0, map_b1, p, stream);
}

}  // namespace

cudaError_t read_product_wait_expired(unsigned int* count) { return cudaMemcpyFromSymbol(count, g_product_wait_expired, sizeof(unsigned int)); }

cudaError_t launch_mx_product(const tq_mx_t& a, const tq_mx_t& b, void* out, bool bf16, uint64_t out_stride, cudaStream_t stream) {
    ProductArgs p{};
    p.out = out; p.out_stride = out_stride; p.out_bf16 = bf16;
    return launch_product_as<0>(a, b, b, p, stream);
}

cudaError_t launch_mx_gated(const MxGatedCall& c) {
    ProductArgs p{};
    p.out = c.projections; p.out_stride = c.proj_stride; p.out_bf16 = c.proj_bf16;
    p.h = mx_view(*c.h);
    return c.gelu ? launch_product_as<2>(*c.x, *c.w_gate, *c.w_up, p, c.stream) : launch_product_as<1>(*c.x, *c.w_gate, *c.w_up, p, c.stream);
}

}  // namespace tq
