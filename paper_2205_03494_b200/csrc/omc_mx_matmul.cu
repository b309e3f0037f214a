// omc_mx_matmul / omc_mx_linear: products of two matrices in the 4-bit microscaled format on the tensor cores.
//
//     Y[m][n] = sum_k  2^(sx[m][k/32] - 127) X[m][k]  *  2^(sw[n][k/32] - 127) W[n][k]
// with E2M1 codes and E8M0 scales as operands of tcgen05.mma (kind::mxf4, one scale per 32) and FP32
// accumulation.  W's rows are the M side of the instruction (the 128 lanes of tensor memory) and X's the
// N side, so that a product with few rows of X wastes no tensor work on a side that is 128 at least, and the
// accumulator's lanes run along Y's contiguous dimension: a warp's store is 32 neighbouring values.
//
// One persistent CTA per SM walks over tiles of 128 x NT of Y.
//   warp 0       (one thread) copies: per K step of 256 values 128 bytes of codes and 8 scales of each row
//   warp 1       (one thread) products, tcgen05.mma of 128 x NT x 64
//   warps 4-11   results: a quarter of tensor memory's lanes and half of the columns each
//   warps 12-15  scales from shared to tensor memory, a copy in each quarter of the lanes.  (tcgen05.cp does the same in
//                one instruction per 512 bytes, but in the tensor pipe, between the products: measured 30 us of 142 at
//                M = 16384, N = 2048, K = 8192.)
// Tensor memory (512 columns) holds two accumulators, so that the results of one tile are stored under the products of
// the next, and the scales of three or four K steps; a step's columns are free again when its products are through,
// which the barrier of its stage tells.  With NT = 256 the accumulators alone would fill it: accumulator 1 starts 80
// columns early, inside accumulator 0; the shared columns are read first and released, then the next products start.
// The widest tile needs the fewest bytes per product (a 128 x 128 tile was bound by the traffic from L2 to shared memory);
// narrower ones spread a small product over more SMs.  With fewer tiles than SMs the K steps of a tile are divided
// among the CTAs of a cluster: each owns a share of X's rows and gets the others' parts of these (stores to distributed
// shared memory, which nobody waits for), which it adds up in a fixed order.
// The waits for copies, products and results are bounded, those of a cluster's CTAs for one another end because these do; tensor memory is
// released on every path, after the products.  It is taken only after the kernel before on the stream has finished: nothing
// waits for another kernel while it holds what others need.
// Measured: M = 16384, N = 2048, K = 8192 107 us (5.1 PFLOP/s, twenty in a row; 125 us, 4.4 PFLOP/s, held at 1.48 GHz by the power cap
// when repeated for seconds), M = N = 8192, K = 2048 67 us.  The instructions alone, without copies, scales and results, take
// 98 us at the first of these; most of the rest is the way from a freed step to the next scales in tensor memory, which the
// products wait for (one more exchange between lanes there cost 3 to 5 %).
#include <cuda.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "element.cuh"
#include "mx_encode.cuh"
#include "mx_format.cuh"
#include "mx_schedule.h"
#include "omc_internal.h"
#include "tensor_core.cuh"

namespace omc {
bool mx_shape_ok(uint64_t rows, uint64_t cols);
}

namespace {

using namespace omc;
using namespace omc::tc;

constexpr int BM = mx::TILE_W, BK = mx::STEP_K;       // W rows per CTA; K per stage (128 bytes of codes)
static_assert(mx::LAID_OUT_SMS == DEFAULT_SMS, "");
constexpr int INSTR_K = 64;                           // K of one tcgen05.mma with 4-bit inputs
constexpr int TILE_W_BYTES = BM * BK / 2;
constexpr int SCALE_BYTES = 1024;                     // scales of 128 rows x 256 columns
constexpr int SCALE_COLS = 8;                         // ... in tensor-memory columns
constexpr int THREADS = 512, EPILOGUE_THREADS = 256, SCALE_THREADS = 128;
constexpr int TMEM_COLS = 512;

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
// Before a CTA ends, also after a wait that ran out: its copies have landed (`issued` stages were filled, in turn) ...
template <typename F>
__device__ __forceinline__ void copies_landed(uint32_t issued, uint32_t stages, uint32_t limit, F full)
{
    for (uint32_t it = issued > stages ? issued - stages : 0u; it < issued; ++it) mbar_wait_held(full(it % stages), (it / stages) & 1u, limit);
}
// ... and what was issued to the tensor cores has finished, whichever thread's wait it was (a barrier for this alone).
__device__ __forceinline__ void products_finished(uint32_t bar)
{
    umma_commit(bar);
    mbar_wait_held(bar, 0u, HELD_LIMIT);
}
// A thread whose wait ran out says so to the caller and, through a word of shared memory, to the CTA's issuing thread, which asks
// behind a barrier.  (A barrier that joins the threads' answers costs 1024 x 2048 x 2048 1.5 %.)
__device__ __forceinline__ void shared_word(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t shared_word(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void give_up(uint32_t *status, uint32_t gave_up)
{
    atomicExch(status, 1u);
    shared_word(gave_up, 1u);
}
// The waits' limits: constants, and for omc_mx_inject_wait_timeout, in kernels of their own (limits that are variables cost
// 1024 x 2048 x 2048 5 %, 16384 x 2048 x 8192 0.8 %), the given number of polls; the first CTA then announces its copies without issuing them, or gives up the waits
// for results at once, with the products on their way.
struct Usual {
    static constexpr uint32_t polls = WAIT_LIMIT, held = HELD_LIMIT;
    static __device__ __forceinline__ bool missing() { return false; }
    static __device__ __forceinline__ uint32_t results() { return held; }
};
struct Trial {
    uint32_t polls, held, what;
    __device__ __forceinline__ bool missing() const { return what == OMC_MX_COPIES_MISSING && blockIdx.x == 0; }
    __device__ __forceinline__ uint32_t results() const { return what == OMC_MX_RESULTS_LATE && blockIdx.x == 0 ? 0u : held; }
};
// Four neighbouring values of a row of Y, as many of them as the row has.
template <typename T>
__device__ __forceinline__ void put4(T *p, uint32_t left, float4 v)
{
    if (left > 0) p[0] = el::from_float<T>(v.x);
    if (left > 1) p[1] = el::from_float<T>(v.y);
    if (left > 2) p[2] = el::from_float<T>(v.z);
    if (left > 3) p[3] = el::from_float<T>(v.w);
}

// The sums of the parts of `mine` rows of Y from row m on, in the order of the parts' K ranges; part r, row i at [r][i][128].
template <typename T>
__device__ __forceinline__ void add_parts(const float4 *parts, uint32_t warp, uint32_t warps, uint32_t splits, uint32_t mine, uint32_t m, uint32_t M,
                                          uint32_t n, uint32_t N, T *y, uint64_t ldy)
{
    for (uint32_t i = warp; i < mine && m + i < M; i += warps) {
        float4 sum = parts[i * 32];
        for (uint32_t r = 1; r < splits; ++r) {
            const float4 v = parts[(r * mine + i) * 32];
            sum.x += v.x;
            sum.y += v.y;
            sum.z += v.z;
            sum.w += v.w;
        }
        if (n < N) put4(y + (uint64_t)(m + i) * ldy + n, N - n, sum);
    }
}

template <int NT_>
struct Cfg {
    static constexpr int NT = NT_;
    static constexpr int TILE_X_BYTES = NT * BK / 2;
    static constexpr int X_BLOCKS = NT > 128 ? 2 : 1;                     // blocks of 128 rows that X's scales come in
    static constexpr int STAGE = TILE_W_BYTES + TILE_X_BYTES + (1 + X_BLOCKS) * SCALE_BYTES;
    static constexpr int NSTAGES = 208 * 1024 / STAGE;
    static constexpr int SLOTS = NT == 256 ? 3 : 4, SLOT_COLS = (1 + X_BLOCKS) * SCALE_COLS;
    static constexpr int D_COLS = NT;
    static constexpr bool DIVIDES = NT == 128;                            // K may be divided among a cluster's CTAs (few tiles: never of 256 rows)
    static constexpr int SHARED_COLS = NT == 256 ? 80 : 0;                // (3 x 24, in whole loads of 16)
    static constexpr int ACC1 = D_COLS - SHARED_COLS, SCALES = ACC1 + D_COLS;
    static constexpr int BARRIERS = 2 * NSTAGES + 7 + SLOTS;
    static constexpr int SMEM = NSTAGES * STAGE + 1024 + 256;
    static_assert(STAGE % 1024 == 0 && SMEM <= 227 * 1024 && 8 * BARRIERS + 8 <= 256, "");
    static_assert(SCALES + SLOTS * SLOT_COLS <= 512 && (!DIVIDES || BM * NT * 4 <= NSTAGES * STAGE), "");
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

template <int NT, typename T, typename WAITS>
__global__ void __launch_bounds__(THREADS, 1)
mx_matmul_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                 const uint8_t *w_scales, const uint8_t *x_scales, T *__restrict__ y, uint64_t ldy,
                 uint32_t M, uint32_t N, uint32_t K, uint32_t splits, uint32_t *status, WAITS waits)
{
    using C = Cfg<NT>;
    constexpr int NS = C::NSTAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - saddr(smem_raw));
    const uint32_t bars = base + NS * C::STAGE;      // full[NS], empty[NS], acc_full[2], acc_shared[2], acc_empty[2], scaled[SLOTS], drained; tmem slot, gave_up
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * NS + b); };
    auto acc_shared = [&](int b) { return bars + 8u * (2 * NS + 2 + b); };      // the shared columns have been read
    auto acc_empty = [&](int b) { return bars + 8u * (2 * NS + 4 + b); };       // all have
    auto scaled = [&](int s) { return bars + 8u * (2 * NS + 6 + s); };          // a step's scales are in tensor memory
    const uint32_t drained = bars + 8u * (C::BARRIERS - 1), tmem_slot = bars + 8u * C::BARRIERS, gave_up = tmem_slot + 4u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // with divided K a cluster has one tile, and a CTA of it a range of its K steps
    const uint32_t rank = splits > 1 ? cluster_cta_rank() : 0u;
    const uint32_t ksteps = (K + BK - 1) / BK;
    const uint32_t k_begin = (uint32_t)((uint64_t)ksteps * rank / splits), k_end = (uint32_t)((uint64_t)ksteps * (rank + 1) / splits);
    const uint32_t tiles_n = (N + BM - 1) / BM, tiles_m = (M + NT - 1) / NT, ntiles = tiles_n * tiles_m;
    const uint32_t first = blockIdx.x / splits, step = gridDim.x / splits;
    const uint32_t steps = (ntiles - first + step - 1) / step * (k_end - k_begin);      // of this CTA

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int s = 0; s < C::SLOTS; ++s) mbar_init(scaled(s), SCALE_THREADS);
        mbar_init(drained, 1);
        shared_word(gave_up, 0u);
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_shared(b), EPILOGUE_THREADS);
            mbar_init(acc_empty(b), EPILOGUE_THREADS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)TMEM_COLS) : "memory");
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
        for (uint32_t t = first; t < ntiles && ok; t += step) {
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            const uint32_t xb = tm * NT / 128;
            const uint8_t *ws = w_scales + (uint64_t)tn * ksteps * SCALE_BYTES;
            const uint8_t *xs0 = x_scales + (uint64_t)xb * ksteps * SCALE_BYTES;
            const uint8_t *xs1 = x_scales + (uint64_t)min(xb + 1, x_blocks - 1) * ksteps * SCALE_BYTES;      // (no such rows: any scales)
            for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
                const int s = it % NS;
                if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, waits.polls);
                if (!ok) break;
                const uint32_t a = base + s * C::STAGE, sc = a + TILE_W_BYTES + C::TILE_X_BYTES;
                mbar_expect_tx(full(s), C::STAGE);
                if (waits.missing()) continue;
                tma_load_2d(a, &map_w, (int)(k * (BK / 2)), (int)(tn * BM), full(s));
                tma_load_2d(a + TILE_W_BYTES, &map_x, (int)(k * (BK / 2)), (int)(tm * NT), full(s));
                bulk_load(sc, ws + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
                bulk_load(sc + SCALE_BYTES, xs0 + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
                if (C::X_BLOCKS == 2) bulk_load(sc + 2 * SCALE_BYTES, xs1 + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
            }
        }
        copies_landed(it, NS, waits.held, full);
    } else if (tid == 32) {
        uint32_t it = 0, lt = 0;
        for (uint32_t t = first; t < ntiles && ok; t += step, ++lt) {
            const uint32_t buf = lt & 1u;
            if (C::SHARED_COLS && lt >= 1) ok = mbar_wait(acc_shared(buf ^ 1u), ((lt - 1) >> 1) & 1u, waits.polls);     // of the tile before
            if (ok && lt >= 2) ok = mbar_wait(acc_empty(buf), ((lt >> 1) - 1) & 1u, waits.polls);                       // of the one before that
            if (!ok) break;
            const uint32_t d = tmem_base + buf * C::ACC1;
            for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
                const int s = it % NS;
                ok = mbar_wait_held(full(s), (it / NS) & 1u, waits.held);
                ok = ok && mbar_wait_held(scaled(it % C::SLOTS), (it / C::SLOTS) & 1u, waits.held);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t a = base + s * C::STAGE, b = a + TILE_W_BYTES;
                const uint32_t ta = tmem_base + C::SCALES + it % C::SLOTS * C::SLOT_COLS, tb = ta + SCALE_COLS;
#pragma unroll
                for (int i = 0; i < BK / INSTR_K; ++i)
                    mma_mx(d, umma_desc(a + i * INSTR_K / 2), umma_desc(b + i * INSTR_K / 2), instr_desc(BM, NT, i & 1),
                           ta + 4 * (i >> 1), tb + 4 * C::X_BLOCKS * (i >> 1), k != k_begin || i != 0);
                umma_commit(empty(s));
            }
            if (ok) umma_commit(acc_full(buf));
        }
    } else if (warp >= 12) {
        const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
        for (uint32_t it = 0; it < steps; ++it) {
            const int s = it % NS;
            if (it >= (uint32_t)C::SLOTS) ok = mbar_wait(empty((it - C::SLOTS) % NS), ((it - C::SLOTS) / NS) & 1u, waits.polls);      // columns are free
            ok = ok && mbar_wait_held(full(s), (it / NS) & 1u, waits.held);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sc = base + s * C::STAGE + TILE_W_BYTES + C::TILE_X_BYTES + lane * 16;
            const uint32_t ta = tmem_base + C::SCALES + it % C::SLOTS * C::SLOT_COLS + quarter, tb = ta + SCALE_COLS;
            tmem_store8(ta, shared16(sc), shared16(sc + 512));
            if constexpr (C::X_BLOCKS == 2) {
                tmem_store8(tb, shared16(sc + SCALE_BYTES), shared16(sc + 2 * SCALE_BYTES));                    // K's first half: X's rows 0 .. 127, 128 .. 255
                tmem_store8(tb + 8, shared16(sc + SCALE_BYTES + 512), shared16(sc + 2 * SCALE_BYTES + 512));    // its second
            } else {
                tmem_store8(tb, shared16(sc + SCALE_BYTES), shared16(sc + SCALE_BYTES + 512));
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(scaled(it % C::SLOTS));
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2;
        uint32_t lt = 0;
        for (uint32_t t = first; t < ntiles; t += step, ++lt) {
            const uint32_t buf = lt & 1u;
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            ok = mbar_wait_held(acc_full(buf), (lt >> 1) & 1u, waits.results());
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (t + step >= ntiles) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            if (!ok || (C::DIVIDES && splits > 1)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t n = tn * BM + q * 32 + lane, m0 = tm * NT;
            const uint32_t acc = tmem_base + buf * C::ACC1 + ((uint32_t)(q * 32) << 16);
            T *out = y + (uint64_t)m0 * ldy + n;
            const bool whole = m0 + NT <= M;                     // no column needs a check
            auto put = [&](int c, const uint32_t *v) {           // sixteen columns from c on
                if (n >= N) return;
                T *p = out + (uint64_t)c * ldy;
                if (whole) {
#pragma unroll
                    for (int j = 0; j < 16; ++j, p += ldy) *p = el::from_float<T>(__uint_as_float(v[j]));
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j, p += ldy)
                        if (m0 + c + j < M) *p = el::from_float<T>(__uint_as_float(v[j]));
                }
            };
            int c = half * (NT / 2), c_end = c + NT / 2;
            if constexpr (C::SHARED_COLS != 0) {
                // the last 80 columns of accumulator 0 (upper half), the first 80 of accumulator 1 (lower half)
                if ((half == 1) == (buf == 0)) {
                    const int from = buf == 0 ? 256 - C::SHARED_COLS : 0;
                    uint32_t v[C::SHARED_COLS];
#pragma unroll
                    for (int i = 0; i < C::SHARED_COLS; i += 16) tmem_load16_async(acc + from + i, v + i);
                    tmem_load_wait();
#pragma unroll
                    for (int i = 0; i < C::SHARED_COLS; i += 16) loaded16(v + i);
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    mbar_arrive(acc_shared(buf));
#pragma unroll
                    for (int i = 0; i < C::SHARED_COLS; i += 16) put(from + i, v + i);
                    if (buf == 0) c_end = from;
                    else c = C::SHARED_COLS;
                } else {
                    mbar_arrive(acc_shared(buf));
                }
            }
#pragma unroll 1
            for (; c < c_end && m0 + c < M; c += 16) {
                uint32_t v[16];
                tmem_load16(acc + c, v);
                put(c, v);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(acc_empty(buf));
        }
    }
    if (C::DIVIDES && splits > 1) {
        uint32_t tn, tm;
        tile_of(first, tiles_n, tiles_m, tn, tm);
        const uint32_t m0 = tm * NT, mine = NT / splits;
        __syncwarp();
        cluster_barrier();                                 // every CTA of the cluster is through with its stages: parts may be put there
        if (warp >= 4 && warp < 12 && ok) {
            const int q = warp & 3, half = (warp - 4) >> 2;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
            for (int c = half * (NT / 2); c < (half + 1) * (NT / 2) && m0 + c < M; c += 16) {
                uint32_t v[16];
                tmem_load16(tmem_base + ((uint32_t)(q * 32) << 16) + c, v);
                // row r of the tile belongs to CTA r / mine, there place r mod mine of part `rank`
                const uint32_t here = base + (rank * mine * BM + q * 32 + lane) * 4;
                const uint32_t to = map_to_cta(here + (c & (mine - 1)) * BM * 4, c >> (31 - __clz(mine)));      // (mine >= 32)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (m0 + c + j < M) store_remote(to + j * BM * 4, __uint_as_float(v[j]));
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
        __syncwarp();
        cluster_barrier();                                 // the parts of this CTA's rows have arrived
        add_parts(reinterpret_cast<const float4 *>(base_ptr) + lane, warp, THREADS / 32, splits, mine, m0 + rank * mine, M, tn * BM + lane * 4, N, y, ldy);
    }
    // The first tile's number keeps a register to the end, as the join would make it: if the loops over the tiles may count in that
    // register, the compiler's code for them is 2 % slower (16384 x 2048 x 8192 109.1 instead of 107.0 us).
    if constexpr (!C::DIVIDES) asm volatile("" ::"r"(first));
    if (!ok) give_up(status, gave_up);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    __syncthreads();
    if (tid == 32 && shared_word(gave_up)) products_finished(drained);
    __syncwarp();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
}

// ---- few rows of X (at most 64): the time is that of W's way from memory and of the start-up --------------
// Two CTAs of six warps share an SM, one tile each; the issuing thread copies the scales itself (tcgen05.cp; a step's before
// the products of the step before it, so that these do not wait for the copy), each stage with columns of its own.
template <int NT>
struct Narrow {
    static constexpr int TILE_X_BYTES = NT * BK / 2;
    static constexpr int STAGE = TILE_W_BYTES + TILE_X_BYTES + 2 * SCALE_BYTES;
    // Every instantiation asks for this much, so that never more than two CTAs (2 x 256 columns of tensor memory) share an
    // SM: a third would wait for tensor memory while its cluster's other CTAs hold some.
    static constexpr int SMEM = 112 * 1024;
    static constexpr int NSTAGES = (SMEM - 1024 - 256) / STAGE;
    static constexpr int D_COLS = NT < 32 ? 32 : NT, TMEM_COLS = 256;
    static constexpr int THREADS = 192;
    static_assert(STAGE % 1024 == 0 && D_COLS + NSTAGES * 2 * SCALE_COLS <= TMEM_COLS && 8 * (2 * NSTAGES + 3) <= 256, "");
    static_assert(BM * NT * 4 <= NSTAGES * STAGE, "a partial result fits where the stages were");
};

// Rows of X that are not quantised yet.
template <typename TX>
struct Values {
    const TX *x;
    uint64_t ld;
    uint32_t rows;        // M rounded up to a power of two
    uint32_t vector;      // rows start on 16-byte boundaries
    using Type = TX;
    static constexpr int N = el::Word<TX>::N;
};
struct Nothing {};

// X quantised already (SOURCE = Nothing: map_x, x_scales), or at most 16 rows of values of type TX (SOURCE = Values<TX>), which warps 2-5 of
// every CTA quantise for themselves on the way into the operand tile: a thread a block, 8 `rows` threads a K step, the other threads
// the steps after it.  Tile rows behind `rows` stay as they are: they only enter columns that nobody reads.
template <int NT, typename T, typename SOURCE, typename WAITS>
__global__ void __launch_bounds__(Narrow<NT>::THREADS)
mx_matmul_narrow_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                        const uint8_t *w_scales, const uint8_t *x_scales, SOURCE source, T *__restrict__ y, uint64_t ldy,
                        uint32_t M, uint32_t N, uint32_t K, uint32_t splits, uint32_t *status, WAITS waits)
{
    constexpr bool VALUES = !std::is_same<SOURCE, Nothing>::value;
    static_assert(!VALUES || NT == 16, "sixteen rows of eight blocks are a thread each");
    using C = Narrow<NT>;
    constexpr int NS = C::NSTAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - saddr(smem_raw));
    const uint32_t bars = base + NS * C::STAGE;           // full[NS], empty[NS], done, drained; tmem slot, gave_up
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    const uint32_t done = bars + 8u * (2 * NS), drained = done + 8u, tmem_slot = drained + 8u, gave_up = tmem_slot + 4u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = splits > 1 ? cluster_cta_rank() : 0u;
    const uint32_t tile_n = blockIdx.x / splits;
    const uint32_t ksteps = (K + BK - 1) / BK;
    const uint32_t k_begin = (uint32_t)((uint64_t)ksteps * rank / splits), k_end = (uint32_t)((uint64_t)ksteps * (rank + 1) / splits);

    if (tid == 0) {
        uint32_t arrivals = 1;
        if constexpr (VALUES) arrivals += 8 * source.rows;
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), arrivals); mbar_init(empty(s), 1); }
        mbar_init(done, 1);
        mbar_init(drained, 1);
        shared_word(gave_up, 0u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    el::enter_stream_order();
    // tensor memory is taken while the first copies are on their way; warps 2-5 learn where it is at barrier 1
    uint32_t tmem_base = 0;
    auto read_slot = [&]() {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot) : "memory");
    };
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        asm volatile("bar.arrive 1, 160;" ::: "memory");
        read_slot();
    }

    bool ok = true;
    if (tid == 0) {
        const uint8_t *ws = w_scales + (uint64_t)tile_n * ksteps * SCALE_BYTES;
        uint32_t it = 0;
        for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
            const int s = it % NS;
            if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, waits.polls);
            if (!ok) break;
            const uint32_t a = base + s * C::STAGE;
            mbar_expect_tx(full(s), VALUES ? TILE_W_BYTES + SCALE_BYTES : C::STAGE);
            if (waits.missing()) continue;
            tma_load_2d(a, &map_w, (int)(k * (BK / 2)), (int)(tile_n * BM), full(s));
            bulk_load(a + TILE_W_BYTES + C::TILE_X_BYTES, ws + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
            if constexpr (!VALUES) {
                tma_load_2d(a + TILE_W_BYTES, &map_x, (int)(k * (BK / 2)), 0, full(s));
                bulk_load(a + TILE_W_BYTES + C::TILE_X_BYTES + SCALE_BYTES, x_scales + (uint64_t)k * SCALE_BYTES, SCALE_BYTES, full(s));
            }
        }
        copies_landed(it, NS, waits.held, full);
    } else if (tid == 32) {
        const uint32_t steps = k_end - k_begin;
        auto bring_scales = [&](uint32_t it) {            // its columns were last read NS steps ago, before the stage was refilled
            const int s = it % NS;
            if (!mbar_wait_held(full(s), (it / NS) & 1u, waits.held)) return false;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sc = base + s * C::STAGE + TILE_W_BYTES + C::TILE_X_BYTES;
            const uint32_t ta = tmem_base + C::D_COLS + s * 2 * SCALE_COLS, tb = ta + SCALE_COLS;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                copy_scales(ta + 4 * h, sc + 512 * h);
                copy_scales(tb + 4 * h, sc + SCALE_BYTES + 512 * h);
            }
            return true;
        };
        ok = bring_scales(0);
        for (uint32_t it = 0; it < steps && ok; ++it) {
            const int s = it % NS;
            if (it + 1 < steps) ok = bring_scales(it + 1);
            if (!ok) break;
            const uint32_t a = base + s * C::STAGE, b = a + TILE_W_BYTES;
            const uint32_t ta = tmem_base + C::D_COLS + s * 2 * SCALE_COLS, tb = ta + SCALE_COLS;
#pragma unroll
            for (int i = 0; i < BK / INSTR_K; ++i)
                mma_mx(tmem_base, umma_desc(a + i * INSTR_K / 2), umma_desc(b + i * INSTR_K / 2), instr_desc(BM, NT, i & 1),
                       ta + 4 * (i >> 1), tb + 4 * (i >> 1), (it | (uint32_t)i) != 0);
            umma_commit(empty(s));
        }
        if (ok) umma_commit(done);
    } else if (VALUES && warp >= 2) {
        if constexpr (VALUES) {
            const uint32_t t = tid - 64, team = 8 * source.rows, r = t % team / 8, block = t % 8;
            for (uint32_t it = t / team; it < k_end - k_begin; it += 128 / team) {
                const int s = it % NS;
                const uint32_t col = (k_begin + it) * BK + block * 32;
                uint32_t w[32 / SOURCE::N], codes[4], scale;
                if (r >= M || col >= K) {
#pragma unroll
                    for (int i = 0; i < 32 / SOURCE::N; ++i) w[i] = 0u;
                } else if (source.vector) {
                    mx::load<typename SOURCE::Type, true, 32>(source.x + r * source.ld, col, K, w);
                } else {
                    mx::load<typename SOURCE::Type, false, 32>(source.x + r * source.ld, col, K, w);
                }
                mx::encode_block<typename SOURCE::Type, 32>(w, codes, scale);
                if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, waits.polls);
                if (!ok) break;
                uint8_t *tile = base_ptr + s * C::STAGE + TILE_W_BYTES;
                // 128-byte swizzle: 16-byte chunk c of row r sits at chunk c ^ (r mod 8)
                *reinterpret_cast<uint4 *>(tile + r * 128 + ((block ^ (r & 7)) << 4)) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
                tile[C::TILE_X_BYTES + SCALE_BYTES + (block >> 2) * 512 + r * 16 + (block & 3)] = (uint8_t)scale;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // visible to the tensor cores
                mbar_arrive(full(s));
            }
        }
    }
    __syncwarp();
    const int q = warp & 3;                               // quarter of the lanes a warp may read
    const uint32_t n = tile_n * BM + q * 32 + lane, mine = NT / splits;
    if (warp >= 2) {
        asm volatile("bar.sync 1, 160;" ::: "memory");
        read_slot();
        ok = mbar_wait_held(done, 0u, waits.results()) && ok;
        ok = __all_sync(0xFFFFFFFFu, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    // every CTA of the cluster is through with its stages: parts may be put there
    if (splits > 1) cluster_barrier();
    if (warp >= 2) {
        if (ok) {
#pragma unroll 1
            for (int c = 0; c < NT && c < (int)M; c += 16) {
                uint32_t v[16];
                tmem_load16(tmem_base + ((uint32_t)(q * 32) << 16) + c, v);
                if (splits > 1) {
                    // row r of the tile belongs to CTA r / mine, there place r mod mine of part `rank`
                    const uint32_t here = base + (rank * mine * BM + q * 32 + lane) * 4, shift = 31 - __clz(mine);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < M) store_remote(map_to_cta(here + ((c + j) & (mine - 1)) * BM * 4, (c + j) >> shift), __uint_as_float(v[j]));
                } else if (n < N) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < M) y[(uint64_t)(c + j) * ldy + n] = el::from_float<T>(__uint_as_float(v[j]));
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    if (!ok) give_up(status, gave_up);
    __syncwarp();
    __syncthreads();
    if (tid == 32 && shared_word(gave_up)) products_finished(drained);
    __syncwarp();
    if (splits > 1) {
        cluster_barrier();                                 // the parts of this CTA's rows have arrived
        add_parts(reinterpret_cast<const float4 *>(base_ptr) + lane, warp, C::THREADS / 32, splits, mine, rank * mine, M, tile_n * BM + lane * 4, N, y, ldy);
    }
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::TMEM_COLS) : "memory");
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

// What omc_mx_inject_wait_timeout asked for, for the calling thread's next product with FP32 results (what = 0: nothing).
thread_local Trial next_trial = {0u, 0u, 0u};
Trial take_trial()
{
    const Trial t = next_trial;
    next_trial = {0u, 0u, 0u};
    return t;
}

struct Product {
    const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
    uint32_t M, N, K;
    void *y;
    uint64_t ldy;
    uint32_t *status;
    void *stream;
};

template <int NT, typename T, typename WAITS>
int launch(const Product &p, uint32_t splits, WAITS waits)
{
    using C = Cfg<NT>;
    CUtensorMap map_w, map_x;
    if (!make_codes_map(&map_w, p.w_codes, p.N, p.K, BM) || !make_codes_map(&map_x, p.x_codes, p.M, p.K, NT)) return OMC_ERR_CUDA;
    if (const int rc = el::allow_smem<mx_matmul_kernel<NT, T, WAITS>>(C::SMEM)) return rc;
    const uint64_t tiles = mx::tiles_of(p.M, p.N, NT), sms = el::sm_count();
    if (tiles >= (1ull << 31)) return OMC_ERR_INVALID_ARG;
    const uint32_t grid = (uint32_t)(splits > 1 ? tiles * splits : tiles < sms ? tiles : sms);
    return note_cuda(el::launch(mx_matmul_kernel<NT, T, WAITS>, dim3(grid), THREADS, C::SMEM, splits, p.stream, map_w, map_x, p.w_scales, p.x_scales,
                                static_cast<T *>(p.y), p.ldy, p.M, p.N, p.K, splits, p.status, waits));
}

template <int NT, typename T, typename SOURCE, typename WAITS>
int launch_narrow(const Product &p, uint32_t splits, SOURCE source, WAITS waits)
{
    using C = Narrow<NT>;
    CUtensorMap map_w, map_x;
    if (!make_codes_map(&map_w, p.w_codes, p.N, p.K, BM)) return OMC_ERR_CUDA;
    if (std::is_same<SOURCE, Nothing>::value) {
        if (!make_codes_map(&map_x, p.x_codes, p.M, p.K, NT)) return OMC_ERR_CUDA;
    } else {
        map_x = map_w;      // not used
    }
    if (const int rc = el::allow_smem<mx_matmul_narrow_kernel<NT, T, SOURCE, WAITS>>(C::SMEM)) return rc;
    return note_cuda(el::launch(mx_matmul_narrow_kernel<NT, T, SOURCE, WAITS>, dim3((uint32_t)mx::tiles_of(p.M, p.N, NT) * splits), C::THREADS, C::SMEM, splits, p.stream, map_w, map_x,
                                p.w_scales, p.x_scales, source, static_cast<T *>(p.y), p.ldy, p.M, p.N, p.K, splits, p.status, waits));
}

template <typename T, typename WAITS>
int launch_any(const Product &p, WAITS waits)
{
    const mx::Schedule s = mx::schedule_of(p.M, p.N, p.K);
    switch (s.tile) {
    case 16: return launch_narrow<16, T>(p, s.splits, Nothing(), waits);
    case 32: return launch_narrow<32, T>(p, s.splits, Nothing(), waits);
    case 64: return launch_narrow<64, T>(p, s.splits, Nothing(), waits);
    case 128: return launch<128, T>(p, s.splits, waits);
    default: return launch<256, T>(p, s.splits, waits);
    }
}

// At most this many rows of values are quantised inside the product.
constexpr uint64_t VALUE_ROWS = 16;

template <typename TX>
int product_of_values(const Product &p, const void *x, uint64_t ld, int type)
{
    uint32_t rows = 1;
    while (rows < p.M) rows *= 2;
    const Values<TX> v = {static_cast<const TX *>(x), ld, rows, el::aligned16(x) && ld * sizeof(TX) % 16 == 0};
    const uint32_t splits = mx::schedule_of(p.M, p.N, p.K).splits;
    if (type == OMC_TYPE_F16) return launch_narrow<16, __half>(p, splits, v, Usual());
    if (type == OMC_TYPE_BF16) return launch_narrow<16, __nv_bfloat16>(p, splits, v, Usual());
    const Trial trial = take_trial();
    return trial.what ? launch_narrow<16, float>(p, splits, v, trial) : launch_narrow<16, float>(p, splits, v, Usual());
}

int product(const Product &p, int type)
{
    if (type == OMC_TYPE_F16) return launch_any<__half>(p, Usual());
    if (type == OMC_TYPE_BF16) return launch_any<__nv_bfloat16>(p, Usual());
    const Trial trial = take_trial();
    return trial.what ? launch_any<float>(p, trial) : launch_any<float>(p, Usual());
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
    if (M <= VALUE_ROWS) {
        const Product p = {nullptr, nullptr, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, y, ldy, status, stream};
        return type == OMC_TYPE_F32 ? product_of_values<float>(p, x, ldx, y_type)
               : type == OMC_TYPE_F16 ? product_of_values<__half>(p, x, ldx, y_type) : product_of_values<__nv_bfloat16>(p, x, ldx, y_type);
    }
    uint8_t *scales = workspace + mx::codes_bytes(M, K);
    const int rc = omc_mx_quantise(x, type, M, K, ldx, workspace, scales, nullptr, nullptr, stream);
    if (rc) return rc;
    return product({workspace, scales, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, y, ldy, status, stream}, y_type);
}

extern "C" int omc_mx_inject_wait_timeout(uint32_t polls, int what)
{
    if (polls < 1 || polls > (1u << 16) || (what != OMC_MX_COPIES_MISSING && what != OMC_MX_RESULTS_LATE)) return OMC_ERR_INVALID_ARG;
    next_trial = {polls, polls, (uint32_t)what};
    return OMC_OK;
}
