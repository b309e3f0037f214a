// omc_mx_matmul / omc_mx_linear: products of two matrices in the 4-bit microscaled format on the tensor cores.
//
//     Y[m][n] = sum_k  2^(sx[m][k/32] - 127) X[m][k]  *  2^(sw[n][k/32] - 127) W[n][k]
// with E2M1 codes and E8M0 scales as operands of tcgen05.mma (kind::mxf4, one scale per 32) and FP32
// accumulation.  W's rows are the M side of the instruction (the 128 lanes of tensor memory) and X's the
// N side, so that a product with few rows of X wastes no tensor work on a side that is 128 at least, and the
// accumulator's lanes run along Y's contiguous dimension: a warp's store is 32 neighbouring values.
//
// A CTA computes 128 x NT of Y.  Warp 0 (one thread) runs the copies over K (256 values, 128 bytes of codes
// and 8 scales a row, per stage), warp 1 (one thread) moves each stage's scales into tensor memory
// (tcgen05.cp) and issues the products, warps 2-5 store the result.  Two CTAs share an SM, so that one's
// epilogue runs under the other's products.  With fewer tiles than SMs the K steps of a tile are
// divided among the CTAs of a cluster: each sends its part of every splits-th row of X to that row's CTA (stores to distributed
// shared memory, which nobody waits for), which adds the parts up in a fixed order.
#include <cuda.h>
#include <cuda_runtime.h>

#include "element.cuh"
#include "mx_format.cuh"
#include "omc_internal.h"
#include "tensor_core.cuh"

namespace omc {
bool mx_shape_ok(uint64_t rows, uint64_t cols);
}

namespace {

using namespace omc;
using namespace omc::tc;

constexpr int BM = 128, BK = 256;                     // W rows per CTA; K per stage (128 bytes of codes)
constexpr int INSTR_K = 64;                           // K of one tcgen05.mma with 4-bit inputs
constexpr int TILE_W_BYTES = BM * BK / 2;
constexpr int SCALE_BYTES = 1024;                     // scales of 128 rows x 256 columns
constexpr int TMEM_COLS = 256;                        // half of an SM's: two CTAs fit
constexpr int SCALE_COLS = 8;                         // tensor-memory columns of 128 rows x 256 columns' scales
constexpr int THREADS = 192;
// Every instantiation asks for this much, so that never more than two CTAs (2 x 256 columns of tensor
// memory) share an SM: a third would wait for tensor memory while its cluster's other CTAs hold some.
constexpr int SMEM = 112 * 1024;

// Instruction descriptor: A and B are E2M1 (type 1 at bits 7 and 10), both K-major, N/8 at bit 17, E8M0 scales (bit 23),
// M/128 at bit 27; which bytes of a scale column apply (0: the first two, 2: the last two) at bits 4 (B) and 29 (A).
__host__ __device__ constexpr uint32_t instr_desc(int m, int n, int half)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27) |
           ((uint32_t)(2 * half) << 4) | ((uint32_t)(2 * half) << 29);
}
__device__ __forceinline__ void mma_mx(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t scale_a, uint32_t scale_b,
                                       uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
}
// 512 bytes of scales (32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart) into four columns
// of tensor memory, the same for each quarter of its lanes.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem)
{
    const uint64_t desc = (uint64_t)((smem >> 4) & 0x3FFFu) | (1ull << 16) | (8ull << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// Eight columns of tensor memory of this warp's quarter of the lanes, a word each from every lane's registers.
__device__ __forceinline__ void tmem_store8(uint32_t taddr, uint4 a, uint4 b)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load16_async(uint32_t taddr, uint32_t *v)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// After the wait: nothing computed from these registers may move above it.
__device__ __forceinline__ void loaded16(uint32_t *v)
{
    asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]));
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t *v)
{
    tmem_load16_async(taddr, v);
    tmem_load_wait();
    loaded16(v);
}
__device__ __forceinline__ void store_remote(uint32_t cluster_addr, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
// Four neighbouring values of a row of Y, as many of them as the row has.
template <typename T>
__device__ __forceinline__ void put4(T *p, uint32_t left, float4 v)
{
    if (left > 0) p[0] = el::from_float<T>(v.x);
    if (left > 1) p[1] = el::from_float<T>(v.y);
    if (left > 2) p[2] = el::from_float<T>(v.z);
    if (left > 3) p[3] = el::from_float<T>(v.w);
}

template <int NT>
struct Cfg {
    static constexpr int TILE_X_BYTES = NT * BK / 2;
    static constexpr int STAGE = TILE_W_BYTES + TILE_X_BYTES + 2 * SCALE_BYTES;
    static constexpr int FIT = (SMEM - 1024 - 256) / STAGE;
    static constexpr int NSTAGES = FIT < 6 ? FIT : 6;
    static constexpr int D_COLS = NT < 32 ? 32 : NT;      // accumulator columns; the scales' follow
    static_assert(STAGE % 1024 == 0 && D_COLS + NSTAGES * 2 * SCALE_COLS <= TMEM_COLS, "");
    static_assert(BM * NT * 4 <= NSTAGES * STAGE, "a partial result fits where the stages were");
};

// blockIdx.x: tile of W's rows x cluster size + rank in the cluster; blockIdx.y: tile of X's rows.
template <int NT, typename T>
__global__ void __launch_bounds__(THREADS)
mx_matmul_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                 const uint8_t *__restrict__ w_scales, const uint8_t *__restrict__ x_scales, T *__restrict__ y, uint64_t ldy,
                 uint32_t M, uint32_t N, uint32_t K, uint32_t splits, uint32_t *status)
{
    using C = Cfg<NT>;
    constexpr int NS = C::NSTAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - saddr(smem_raw));
    const uint32_t bars = base + NS * C::STAGE;           // full[NS], empty[NS], done, tmem slot
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    const uint32_t done = bars + 8u * (2 * NS), tmem_slot = done + 8u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = splits > 1 ? cluster_cta_rank() : 0u;
    const uint32_t tile_n = blockIdx.x / splits, tile_m = blockIdx.y;
    const uint32_t ksteps = (K + BK - 1) / BK;
    const uint32_t k_begin = (uint32_t)((uint64_t)ksteps * rank / splits), k_end = (uint32_t)((uint64_t)ksteps * (rank + 1) / splits);

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));
    el::enter_stream_order();

    bool ok = true;
    if (tid == 0) {
        // ---- producer
        const uint8_t *ws = w_scales + (uint64_t)tile_n * ksteps * SCALE_BYTES;
        const uint8_t *xs = x_scales + (uint64_t)(tile_m * NT / 128) * ksteps * SCALE_BYTES;
        for (uint32_t k = k_begin, it = 0; k < k_end; ++k, ++it) {
            const int s = it % NS;
            if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, WAIT_LIMIT);
            if (!ok) break;
            const uint32_t a = base + s * C::STAGE;
            mbar_expect_tx(full(s), C::STAGE);
            tma_load_2d(a, &map_w, (int)(k * (BK / 2)), (int)(tile_n * BM), full(s));
            tma_load_2d(a + TILE_W_BYTES, &map_x, (int)(k * (BK / 2)), (int)(tile_m * NT), full(s));
            bulk_load(a + TILE_W_BYTES + C::TILE_X_BYTES, ws + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
            bulk_load(a + TILE_W_BYTES + C::TILE_X_BYTES + SCALE_BYTES, xs + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
        }
    } else if (tid == 32) {
        // ---- products; a stage's scales have columns of their own, free again when the stage is
        for (uint32_t k = k_begin, it = 0; k < k_end; ++k, ++it) {
            const int s = it % NS;
            ok = mbar_wait(full(s), (it / NS) & 1u, WAIT_LIMIT);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t a = base + s * C::STAGE, b = a + TILE_W_BYTES, sc = b + C::TILE_X_BYTES;
            const uint32_t ta = tmem_base + C::D_COLS + s * 2 * SCALE_COLS, tb = ta + SCALE_COLS;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                copy_scales(ta + 4 * h, sc + 512 * h);
                copy_scales(tb + 4 * h, sc + SCALE_BYTES + 512 * h);
            }
#pragma unroll
            for (int i = 0; i < BK / INSTR_K; ++i)
                mma_mx(tmem_base, umma_desc(a + i * INSTR_K / 2), umma_desc(b + i * INSTR_K / 2), instr_desc(BM, NT, i & 1),
                       ta + 4 * (i >> 1), tb + 4 * (i >> 1), (it | (uint32_t)i) != 0);
            umma_commit(empty(s));
        }
        if (ok) umma_commit(done);
    }
    __syncwarp();
    const int q = warp & 3;                               // quarter of the lanes a warp may read
    const uint32_t n = tile_n * BM + q * 32 + lane, m0 = tile_m * NT;
    if (warp >= 2) {
        ok = mbar_wait(done, 0u, WAIT_LIMIT);
        ok = __all_sync(0xFFFFFFFFu, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    // every CTA of the cluster is through with its stages: parts may be put there
    if (splits > 1) cluster_barrier();
    if (warp >= 2) {
        if (ok) {
#pragma unroll 1
            for (int c = 0; c < NT; c += 16) {
                if (m0 + c >= M) break;
                uint32_t v[16];
                tmem_load16(tmem_base + ((uint32_t)(q * 32) << 16) + c, v);
                if (splits > 1) {
                    // row c + j of the tile belongs to CTA (c + j) mod splits, there place (c + j) / splits of part `rank`
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t r = c + j, place = rank * (NT / splits) + r / splits;
                        store_remote(map_to_cta(base + (place * BM + q * 32 + lane) * 4, r % splits), __uint_as_float(v[j]));
                    }
                } else if (n < N) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (m0 + c + j < M) y[(uint64_t)(m0 + c + j) * ldy + n] = el::from_float<T>(__uint_as_float(v[j]));
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    if (!ok) atomicExch(status, 1u);
    __syncthreads();
    if (splits > 1) {
        cluster_barrier();                                 // the parts of this CTA's rows have arrived
        const float4 *parts = reinterpret_cast<const float4 *>(base_ptr) + lane;
        const uint32_t mine = NT / splits, nn = tile_n * BM + lane * 4;
        for (uint32_t i = warp; i < mine && m0 + i * splits + rank < M; i += THREADS / 32) {
            float4 sum = parts[i * 32];
            for (uint32_t r = 1; r < splits; ++r) {         // in the order of their K ranges
                const float4 v = parts[(r * mine + i) * 32];
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
            if (nn < N) put4(y + (uint64_t)(m0 + i * splits + rank) * ldy + nn, N - nn, sum);
        }
    }
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
}

// ---- large products: one persistent CTA per SM, tiles of 128 x 256 -----------------------------------
// 48 KB of codes per K step for twice the products of a 128 x 128 tile's 32 KB: what bounds the smaller tile is the
// traffic from L2 to shared memory.
//   warp 0   copies (one thread); warp 1   scales to tensor memory and products (one thread)
//   warps 4-11   epilogue: a quarter of the lanes and half of the columns each
//   warps 12-15  scales from shared to tensor memory, a copy in each quarter of the lanes.  (tcgen05.cp does the same in
//   one instruction per 512 bytes, but in the tensor pipe, between the products: measured 30 us of 142 at 16384 x 2048 x 8192.)
// Tensor memory (512 columns): the two accumulators would fill it, and the scales need 3 x 24 columns, so
// accumulator 1 starts 80 columns early, inside accumulator 0.  The epilogue reads the shared columns
// first and releases them; the products of the next tile start then, under the rest of the epilogue.
// The scales of three K steps have columns of their own; those of step it - 3 are free once its products are through,
// which the stage's own barrier tells.
// The kernel does not let its successor start early: it would only take room on SMs that are busy to the end.
struct Wide {
    static constexpr int NT = 256;
    static constexpr int TILE_X_BYTES = NT * BK / 2;
    static constexpr int STAGE = TILE_W_BYTES + TILE_X_BYTES + 3 * SCALE_BYTES;
    static constexpr int NSTAGES = 4;
    static constexpr int SMEM = NSTAGES * STAGE + 1024 + 256;
    static constexpr int THREADS = 512, EPILOGUE_THREADS = 256, SCALE_THREADS = 128;
    static constexpr int SLOTS = 3, SLOT_COLS = 3 * SCALE_COLS, SHARED_COLS = 80;      // (3 x 24, in whole loads of 16)
    static constexpr int ACC1 = 256 - SHARED_COLS, SCALES = 512 - SHARED_COLS;
    static_assert(STAGE % 1024 == 0 && SMEM <= 227 * 1024 && 8 * (2 * NSTAGES + 7 + SLOTS) <= 256, "");
};

// Tiles in the order in which the CTAs take them: bands of sixteen tiles of W's rows, so that the tiles in work
// at a time form a block of about sixteen by nine and share their operands in L2.
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tiles_n, uint32_t tiles_m, uint32_t &tn, uint32_t &tm)
{
    const uint32_t per_band = 16 * tiles_m, band = t / per_band, in_band = t - band * per_band;
    const uint32_t width = min(16u, tiles_n - band * 16);
    tm = in_band / width;
    tn = band * 16 + in_band - tm * width;
}

template <typename T>
__global__ void __launch_bounds__(Wide::THREADS, 1)
mx_matmul_wide_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                      const uint8_t *__restrict__ w_scales, const uint8_t *__restrict__ x_scales, T *__restrict__ y, uint64_t ldy,
                      uint32_t M, uint32_t N, uint32_t K, uint32_t *status)
{
    using C = Wide;
    constexpr int NS = C::NSTAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = base + NS * C::STAGE;      // full[NS], empty[NS], acc_full[2], acc_shared[2], acc_empty[2], scaled[SLOTS], tmem slot
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * NS + b); };
    auto acc_shared = [&](int b) { return bars + 8u * (2 * NS + 2 + b); };      // the shared columns have been read
    auto acc_empty = [&](int b) { return bars + 8u * (2 * NS + 4 + b); };       // all have
    auto scaled = [&](int s) { return bars + 8u * (2 * NS + 6 + s); };          // a step's scales are in tensor memory
    const uint32_t tmem_slot = bars + 8u * (2 * NS + 6 + C::SLOTS);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ksteps = (K + BK - 1) / BK;
    const uint32_t tiles_n = (N + BM - 1) / BM, tiles_m = (M + C::NT - 1) / C::NT, ntiles = tiles_n * tiles_m;

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int s = 0; s < C::SLOTS; ++s) mbar_init(scaled(s), C::SCALE_THREADS);
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_shared(b), C::EPILOGUE_THREADS);
            mbar_init(acc_empty(b), C::EPILOGUE_THREADS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));

    bool ok = true;
    if (tid == 0) {
        const uint32_t x_blocks = (M + 127) / 128;
        uint32_t it = 0;
        for (uint32_t t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            const uint8_t *ws = w_scales + (uint64_t)tn * ksteps * SCALE_BYTES;
            const uint8_t *xs0 = x_scales + (uint64_t)(2 * tm) * ksteps * SCALE_BYTES;
            const uint8_t *xs1 = x_scales + (uint64_t)min(2 * tm + 1, x_blocks - 1) * ksteps * SCALE_BYTES;      // (no such rows: any scales)
            for (uint32_t k = 0; k < ksteps; ++k, ++it) {
                const int s = it % NS;
                if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, WAIT_LIMIT);
                if (!ok) break;
                const uint32_t a = base + s * C::STAGE, sc = a + TILE_W_BYTES + C::TILE_X_BYTES;
                mbar_expect_tx(full(s), C::STAGE);
                tma_load_2d(a, &map_w, (int)(k * (BK / 2)), (int)(tn * BM), full(s));
                tma_load_2d(a + TILE_W_BYTES, &map_x, (int)(k * (BK / 2)), (int)(tm * C::NT), full(s));
                bulk_load(sc, ws + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
                bulk_load(sc + SCALE_BYTES, xs0 + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
                bulk_load(sc + 2 * SCALE_BYTES, xs1 + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
            }
        }
    } else if (tid == 32) {
        uint32_t it = 0, lt = 0;
        for (uint32_t t = blockIdx.x; t < ntiles && ok; t += gridDim.x, ++lt) {
            const uint32_t buf = lt & 1u;
            if (lt >= 1) ok = mbar_wait(acc_shared(buf ^ 1u), ((lt - 1) >> 1) & 1u, WAIT_LIMIT);     // of the tile before
            if (ok && lt >= 2) ok = mbar_wait(acc_empty(buf), ((lt >> 1) - 1) & 1u, WAIT_LIMIT);     // of the one before that
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t d = tmem_base + buf * C::ACC1;
            for (uint32_t k = 0; k < ksteps; ++k, ++it) {
                const int s = it % NS;
                ok = mbar_wait(full(s), (it / NS) & 1u, WAIT_LIMIT);
                if (ok) ok = mbar_wait(scaled(it % C::SLOTS), (it / C::SLOTS) & 1u, WAIT_LIMIT);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t a = base + s * C::STAGE, b = a + TILE_W_BYTES;
                const uint32_t ta = tmem_base + C::SCALES + it % C::SLOTS * C::SLOT_COLS, tb = ta + SCALE_COLS;
#pragma unroll
                for (int i = 0; i < BK / INSTR_K; ++i)
                    mma_mx(d, umma_desc(a + i * INSTR_K / 2), umma_desc(b + i * INSTR_K / 2), instr_desc(BM, C::NT, i & 1),
                           ta + 4 * (i >> 1), tb + 8 * (i >> 1), (k | (uint32_t)i) != 0);
                umma_commit(empty(s));
            }
            if (ok) umma_commit(acc_full(buf));
        }
    } else if (warp >= 12) {
        const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t steps = (ntiles - blockIdx.x + gridDim.x - 1) / gridDim.x * ksteps;
        for (uint32_t it = 0; it < steps; ++it) {
            const int s = it % NS;
            if (it >= (uint32_t)C::SLOTS) ok = mbar_wait(empty((it - C::SLOTS) % NS), ((it - C::SLOTS) / NS) & 1u, WAIT_LIMIT);      // columns are free
            ok = ok && mbar_wait(full(s), (it / NS) & 1u, WAIT_LIMIT);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sc = base + s * C::STAGE + TILE_W_BYTES + C::TILE_X_BYTES + lane * 16;
            const uint32_t ta = tmem_base + C::SCALES + it % C::SLOTS * C::SLOT_COLS + quarter, tb = ta + SCALE_COLS;
            tmem_store8(ta, shared16(sc), shared16(sc + 512));
            tmem_store8(tb, shared16(sc + SCALE_BYTES), shared16(sc + 2 * SCALE_BYTES));                    // columns 0 .. 127: X's rows 0 .. 127, 128 .. 255
            tmem_store8(tb + 8, shared16(sc + SCALE_BYTES + 512), shared16(sc + 2 * SCALE_BYTES + 512));    // columns 128 .. 255
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(scaled(it % C::SLOTS));
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2;
        uint32_t lt = 0;
        for (uint32_t t = blockIdx.x; t < ntiles; t += gridDim.x, ++lt) {
            const uint32_t buf = lt & 1u;
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            ok = mbar_wait(acc_full(buf), (lt >> 1) & 1u, WAIT_LIMIT);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t n = tn * BM + q * 32 + lane, m0 = tm * C::NT;
            const uint32_t acc = tmem_base + buf * C::ACC1 + ((uint32_t)(q * 32) << 16);
            T *out = y + (uint64_t)m0 * ldy + n;
            // shared columns: the last 80 of accumulator 0 (upper half), the first 80 of accumulator 1 (lower half)
            const bool mine = (half == 1) == (buf == 0);
            auto put = [&](int c, const uint32_t *v) {           // sixteen columns from c on
                if (n >= N) return;
                T *p = out + (uint64_t)c * ldy;
#pragma unroll
                for (int j = 0; j < 16; ++j, p += ldy)
                    if (m0 + c + j < M) *p = el::from_float<T>(__uint_as_float(v[j]));
            };
            int c = half * 128, c_end = c + 128;
            if (mine) {
                const int first = buf == 0 ? 256 - C::SHARED_COLS : 0;
                uint32_t v[C::SHARED_COLS];
#pragma unroll
                for (int i = 0; i < C::SHARED_COLS; i += 16) tmem_load16_async(acc + first + i, v + i);
                tmem_load_wait();
#pragma unroll
                for (int i = 0; i < C::SHARED_COLS; i += 16) loaded16(v + i);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                mbar_arrive(acc_shared(buf));
#pragma unroll
                for (int i = 0; i < C::SHARED_COLS; i += 16) put(first + i, v + i);
                if (buf == 0) c_end = first;
                else c = C::SHARED_COLS;
            } else {
                mbar_arrive(acc_shared(buf));
            }
#pragma unroll 1
            for (; c < c_end; c += 16) {
                uint32_t v[16];
                tmem_load16(acc + c, v);
                put(c, v);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(acc_empty(buf));
        }
    }
    if (!ok) atomicExch(status, 1u);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    __syncthreads();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
}

// The codes as bytes: boxes of box_rows rows x 128 bytes, 128-byte swizzle, zeros outside.
bool make_codes_map(CUtensorMap *m, const void *ptr, uint64_t rows, uint64_t cols, uint32_t box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {mx::row_bytes(cols), rows};
    const cuuint64_t strides[1] = {mx::row_bytes(cols)};
    const cuuint32_t box[2] = {BK / 2, box_rows};
    const cuuint32_t elem[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Product {
    const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
    uint32_t M, N, K;
    void *y;
    uint64_t ldy;
    uint32_t *status;
    void *stream;
};

template <int NT, typename T>
int launch(const Product &p)
{
    CUtensorMap map_w, map_x;
    if (!make_codes_map(&map_w, p.w_codes, p.N, p.K, BM) || !make_codes_map(&map_x, p.x_codes, p.M, p.K, NT)) return OMC_ERR_CUDA;
    const int rc = el::allow_smem<mx_matmul_kernel<NT, T>>(SMEM);
    if (rc) return rc;
    const uint32_t tiles_n = (p.N + BM - 1) / BM, tiles_m = (p.M + NT - 1) / NT, ksteps = (p.K + BK - 1) / BK;
    // divide K while the CTAs still fit on the device at once
    uint32_t splits = 1;
    while (splits < 8 && (uint64_t)tiles_n * tiles_m * splits <= el::sm_count() && ksteps >= splits * 2) splits *= 2;
    return note_cuda(el::launch(mx_matmul_kernel<NT, T>, dim3(tiles_n * splits, tiles_m), THREADS, SMEM, splits, p.stream, map_w, map_x,
                                p.w_scales, p.x_scales, static_cast<T *>(p.y), p.ldy, p.M, p.N, p.K, splits, p.status));
}

template <typename T>
int launch_wide(const Product &p)
{
    CUtensorMap map_w, map_x;
    if (!make_codes_map(&map_w, p.w_codes, p.N, p.K, BM) || !make_codes_map(&map_x, p.x_codes, p.M, p.K, Wide::NT)) return OMC_ERR_CUDA;
    const int rc = el::allow_smem<mx_matmul_wide_kernel<T>>(Wide::SMEM);
    if (rc) return rc;
    const uint64_t ntiles = (uint64_t)((p.N + BM - 1) / BM) * ((p.M + Wide::NT - 1) / Wide::NT);
    const uint32_t sms = el::sm_count();
    return note_cuda(el::launch(mx_matmul_wide_kernel<T>, dim3(ntiles < sms ? (uint32_t)ntiles : sms), Wide::THREADS, Wide::SMEM, 1, p.stream,
                                map_w, map_x, p.w_scales, p.x_scales, static_cast<T *>(p.y), p.ldy, p.M, p.N, p.K, p.status));
}

// Few rows of X: the narrowest tile that holds them all (their scales start at a multiple of 128 rows).
template <typename T>
int launch_any(const Product &p)
{
    if (p.M <= 16) return launch<16, T>(p);
    if (p.M <= 32) return launch<32, T>(p);
    if (p.M <= 64) return launch<64, T>(p);
    if ((uint64_t)((p.N + 127) / 128) * ((p.M + 255) / 256) >= 96) return launch_wide<T>(p);
    return launch<128, T>(p);
}

int product(const Product &p, int type)
{
    return type == OMC_TYPE_F32 ? launch_any<float>(p) : type == OMC_TYPE_F16 ? launch_any<__half>(p) : launch_any<__nv_bfloat16>(p);
}

bool product_shape_ok(uint64_t M, uint64_t N, uint64_t K)
{
    return mx_shape_ok(M, K) && mx_shape_ok(N, K) && M <= 128ull * 65535;
}

}  // namespace

extern "C" int omc_mx_matmul(const uint8_t *x_codes, const uint8_t *x_scales, uint64_t M, const uint8_t *w_codes,
                             const uint8_t *w_scales, uint64_t N, uint64_t K, void *y, int type, uint64_t ldy, uint32_t *status,
                             void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !y || !status) return OMC_ERR_NULL_PTR;
    if (!product_shape_ok(M, N, K) || ldy < N) return OMC_ERR_INVALID_ARG;
    if (!el::aligned16(x_codes) || !el::aligned16(x_scales) || !el::aligned16(w_codes) || !el::aligned16(w_scales) ||
        reinterpret_cast<uintptr_t>(y) % el::size_of(type) || reinterpret_cast<uintptr_t>(status) % 4)
        return OMC_ERR_MISALIGNED;
    return product({x_codes, x_scales, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, y, ldy, status, stream}, type);
}

extern "C" int omc_mx_linear(const void *x, int type, uint64_t M, uint64_t K, uint64_t ldx, const uint8_t *w_codes,
                             const uint8_t *w_scales, uint64_t N, void *y, int y_type, uint64_t ldy, uint8_t *workspace,
                             uint32_t *status, void *stream)
{
    if (!el::type_ok(type) || !el::type_ok(y_type)) return OMC_ERR_INVALID_ARG;
    if (!x || !w_codes || !w_scales || !y || !workspace || !status) return OMC_ERR_NULL_PTR;
    if (!product_shape_ok(M, N, K) || ldx < K || ldy < N) return OMC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x) % el::size_of(type) || !el::aligned16(w_codes) || !el::aligned16(w_scales) ||
        !el::aligned16(workspace) || reinterpret_cast<uintptr_t>(y) % el::size_of(y_type) || reinterpret_cast<uintptr_t>(status) % 4)
        return OMC_ERR_MISALIGNED;
    uint8_t *scales = workspace + mx::codes_bytes(M, K);
    const int rc = omc_mx_quantise(x, type, M, K, ldx, workspace, scales, nullptr, nullptr, stream);
    if (rc) return rc;
    return product({workspace, scales, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, y, ldy, status, stream}, y_type);
}
