// omc_byte_matmul / omc_byte_linear / omc_byte_gated / omc_byte_gated_linear: products of two matrices of 8-bit integers under one scale a row
// (i8_format.cuh) on the tensor cores, tcgen05.mma kind::i8 with 32-bit integer sums.
//
//     Y[m][n] = (sum_k X[m][k] W[n][k]) * sx[m] * sw[n]
// The sum is exact, so that tiles, divisions of K and kernels are free to follow the shape: the bits are the same.  The gated layer takes
// two rows of W for a column of its result, one of each half of W, as two columns of the same accumulator.
//
// Three kernels:
//   tile    tiles of 128 rows of X on an SM or 256 on a pair of SMs; X's rows are the lanes of tensor memory.
//   small   few rows, or few tiles and long sums: W's rows are the 128 lanes, 16 .. 64 rows of X the columns, so that few rows of X
//           waste nothing; K divided among the CTAs of a cluster where there are few tiles.
//   rows    up to four rows of X: no tensor cores, a warp multiplies four rows of W as they come from memory (dp4a); values that are
//           not quantised yet are quantised by every CTA for itself.
#include <cuda.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "element.cuh"
#include "gate.cuh"
#include "i8_format.cuh"
#include "i8_quantise.cuh"
#include "i8_schedule.h"
#include "omc_internal.h"
#include "tensor_core.cuh"

namespace omc {
bool i8_shape_ok(uint64_t rows, uint64_t cols);
}

namespace {

using namespace omc;
using namespace omc::tc;
using el::Word;

constexpr int BK = 128;                                // K of a step: 128 bytes of codes, one swizzled row
constexpr int INSTR_K = 32;                            // K of one tcgen05.mma with 8-bit inputs
constexpr int TILE_BYTES = 128 * BK;                   // 128 rows of a step

// Instruction descriptor: 32-bit integer sums (2 at bit 4), A and B signed (1 at bits 7 and 10), both K-major, N / 8 at bit 17, M / 16 at bit 24.
__host__ __device__ constexpr uint32_t instr_desc(int m, int n)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_i8(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_i8_pair(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// Sixteen columns of this warp's quarter of tensor memory; complete after tmem_wait.
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t *v)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// After the wait: nothing computed from these registers may move above it.
__device__ __forceinline__ void loaded16(uint32_t *v)
{
    asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void shared_word(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t shared_word(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory"); }
__device__ __forceinline__ void store_remote(uint32_t cluster_addr, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
// A thread whose wait ran out says so to the caller and, through a word of shared memory, to its CTA.
__device__ __forceinline__ void give_up(uint32_t *status, uint32_t gave_up)
{
    atomicExch(status, 1u);
    shared_word(gave_up, 1u);
}
// Before a CTA ends, also after a wait that ran out: the copies of the last `stages` of `issued` steps have landed, by the barriers that tell.
template <typename F>
__device__ __forceinline__ void copies_landed(uint32_t issued, uint32_t stages, uint32_t limit, F barrier)
{
    for (uint32_t it = issued > stages ? issued - stages : 0u; it < issued; ++it) mbar_wait_held(barrier(it % stages), (it / stages) & 1u, limit);
}
// The waits' limits: constants; for omc_byte_inject_wait_timeout, in kernels of their own, the given number of polls, and in the first CTA (or
// pair) copies that are announced without being issued, or results that are given up at once with the products on their way.
struct Usual {
    static constexpr uint32_t polls = WAIT_LIMIT, held = HELD_LIMIT;
    static __device__ __forceinline__ bool missing(uint32_t) { return false; }
    static __device__ __forceinline__ uint32_t results(uint32_t) { return held; }
};
struct Trial {
    uint32_t polls, held, what;
    __device__ __forceinline__ bool missing(uint32_t unit) const { return what == OMC_BYTE_COPIES_MISSING && unit == 0; }
    __device__ __forceinline__ uint32_t results(uint32_t unit) const { return what == OMC_BYTE_RESULTS_LATE && unit == 0 ? 0u : held; }
};

// What every kernel is given.  N: columns of Y (gated: F, and W has 2 F rows).
template <typename T>
struct Result {
    const float *x_scales, *w_scales;
    T *y, *pre;
    uint64_t ldy, ld_pre;
    uint32_t M, N, K;
    int act;
    uint32_t *status;
};

template <int ACT, bool FINE>
__device__ __forceinline__ void gate16(const float *a, const float *b, float *y)
{
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
        const float2 v = el::mul2(gate::act2<ACT, FINE>(make_float2(a[j], a[j + 1])), make_float2(b[j], b[j + 1]));
        y[j] = v.x, y[j + 1] = v.y;
    }
}
// FINE: results are FP32 numbers.
template <bool FINE>
__device__ __forceinline__ void gate16(int act, const float *a, const float *b, float *y)
{
    if (act == OMC_GATE_SILU) gate16<OMC_GATE_SILU, FINE>(a, b, y);
    else if (act == OMC_GATE_SIGMOID) gate16<OMC_GATE_SIGMOID, FINE>(a, b, y);
    else gate16<OMC_GATE_GELU, FINE>(a, b, y);
}
template <bool FINE>
__device__ __forceinline__ float gate1(int act, float a, float b)
{
    const float2 aa = el::twice(a);
    return (act == OMC_GATE_SILU ? gate::act2<OMC_GATE_SILU, FINE>(aa)
            : act == OMC_GATE_SIGMOID ? gate::act2<OMC_GATE_SIGMOID, FINE>(aa) : gate::act2<OMC_GATE_GELU, FINE>(aa)).x * b;
}
// Sixteen sums of a row as values; ws: the columns' scales, in shared memory.
__device__ __forceinline__ void values16(const uint32_t *v, const i8::RowScale &x, bool any_big, const float4 *ws, float *f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 w = ws[j];
        f[4 * j] = i8::value((int)v[4 * j], x, w.x);
        f[4 * j + 1] = i8::value((int)v[4 * j + 1], x, w.y);
        f[4 * j + 2] = i8::value((int)v[4 * j + 2], x, w.z);
        f[4 * j + 3] = i8::value((int)v[4 * j + 3], x, w.w);
    }
    if (any_big) {            // rare: of a warp's rows one has a scale of 2^64 or more
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] *= x.g;
    }
}

// ---- tiles of 128 or 256 rows of X ---------------------------------------------------------------------
// CG CTAs, a cluster, share a tile of 128 CG rows of X by BN rows of W (gated: BN / 2 of either half).  With two, each holds 128 rows of X and
// BN / 2 rows of W for a K step (32 KB for the largest tile, five steps on their way), the leader issues products of 256 x BN x 32 whose upper half
// accumulates in its own tensor memory and whose lower half in its peer's, and each CTA stores its 128 rows.  In the gated layer the accumulator's
// first BN / 2 columns are a, the others b: with two CTAs the leader holds the gate's rows and its peer the same rows of the other half.
// Barriers as their waiters need them: full (in the leader, the bytes of both CTAs' copies), empty and acc_full (in each CTA, a commit
// reaches both), acc_empty (in the leader, an arrival of each of the warps that store results).
// Every wait is bounded, and a role whose wait ran out leaves its loop, so that both CTAs reach the closing barrier on every path.
// Tensor memory is taken after the kernel before on the stream has finished and let go after the products.
// The tensor cores bound long sums: 16384 x 2048 x 8192 BF16 162 us in bursts, 3.4 POP/s (twice the rate measured of BF16 products is 3.2), 8192 x 2048 x 8192 92 us;
// for seconds the board's power does (about 1 kW).  Short sums are bound by results: 8192 x 8192 x 256 BF16 40 us, of which 128 MB of results take
// 20 at the copy rate and the sums 11; gated 8192 x 8192 x 2048 BF16 with what is kept 209 us (188 without), products alone 171.
// A tile's results leave tensor memory while the next tile's products are made: two accumulators, 512 columns for the largest tile.
template <int CG, int BN, bool GATED>
struct Tile {
    static constexpr int W_ROWS = BN / CG;                           // of a CTA
    static constexpr int STAGE = TILE_BYTES + W_ROWS * BK;
    static constexpr int STORE_WARPS = 8, STORE_THREADS = 32 * STORE_WARPS, THREADS = 64 + STORE_THREADS;
    static constexpr int SCALES = 2 * BN * 4;                        // of W's rows, of two tiles
    // results on their way from a warp to memory, in boxes of 32 rows (or 16 or 32 columns of rows off the 16-byte boundaries)
    static constexpr int ROOM_EACH = 6 * 1024, ROOM = STORE_WARPS * ROOM_EACH;
    static constexpr int FIT = (220 * 1024 - SCALES - ROOM - 1024 - 256) / STAGE, NSTAGES = FIT < 8 ? FIT : 8;
    static constexpr int BARRIERS = 2 * NSTAGES + 5;
    static constexpr int SMEM = NSTAGES * STAGE + SCALES + ROOM + 1024 + 256;
    static constexpr int TMEM_COLS = 2 * BN;
    static constexpr int COLS = GATED ? BN / 2 : BN;                 // of Y
    static constexpr int W_BOX = GATED ? BN / 2 : W_ROWS;            // rows of a copy
    static_assert(STAGE % 1024 == 0 && NSTAGES >= 4 && 8 * BARRIERS + 8 <= 256, "");
};

// Barrier of the threads that store results, and whether all of them say yes: they leave their loop together or not at all.
template <int THREADS>
__device__ __forceinline__ bool together(bool ok)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all) : "r"((uint32_t)ok), "n"(THREADS) : "memory");
    return all != 0u;
}
// Tiles in the order in which they are taken: bands of eight tiles of W's rows, so that the tiles in work at a time form a
// block of about eight by nine and share their operands in L2.
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tiles_n, uint32_t tiles_m, uint32_t &tn, uint32_t &tm)
{
    const uint32_t per_band = 8 * tiles_m, band = t / per_band, in_band = t - band * per_band;
    const uint32_t width = min(8u, tiles_n - band * 8);
    tm = in_band / width;
    tn = band * 8 + in_band - tm * width;
}

// COLS neighbouring values of each lane's row, from column `col` on, to a matrix of `cols` columns whose rows start anywhere: through shared memory,
// so that neighbouring lanes store neighbouring words.  Of 16-bit types a row may start in the upper half of a word: its words are then made with
// the neighbour lane's, and its first and last values go out alone.
template <typename T, int COLS>
__device__ __forceinline__ void store_any(const float *f, T *to, uint64_t ld, uint32_t row0, uint32_t rows, uint32_t col, uint32_t cols, int lane, uint32_t *room)
{
    constexpr int N = Word<T>::N, WORDS = COLS / N, PITCH = WORDS + 4, TOGETHER = 32 / WORDS;      // (an odd number of sixteens from row to row: no bank twice)
    static_assert(WORDS <= 32 && 32 * PITCH * 4 <= 6 * 1024, "");
    __syncwarp();
#pragma unroll
    for (int j = 0; j < WORDS; j += 4)
        *reinterpret_cast<uint4 *>(room + lane * PITCH + j) =
            make_uint4(Word<T>::pack(f + j * N), Word<T>::pack(f + (j + 1) * N), Word<T>::pack(f + (j + 2) * N), Word<T>::pack(f + (j + 3) * N));
    __syncwarp();
    const int n = row0 < rows ? (int)min(32u, rows - row0) : 0, j = lane % WORDS, first = lane / WORDS;
    T *p = to + (uint64_t)(row0 + first) * ld + col;
    if (col + COLS <= cols) {
#pragma unroll 4
        for (int r = first; r < 32; r += TOGETHER, p += TOGETHER * ld) {
            const uint32_t w = room[r * PITCH + j];
            if constexpr (N == 1) {
                if (r < n) reinterpret_cast<uint32_t *>(p)[j] = w;
            } else {
                const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, w, 1, WORDS);
                const bool odd = (reinterpret_cast<uintptr_t>(p) & 2) != 0;
                uint16_t *const h = reinterpret_cast<uint16_t *>(p) + 2 * j;
                if (r < n) {
                    if (!odd) *reinterpret_cast<uint32_t *>(h) = w;
                    else if (j > 0) *reinterpret_cast<uint32_t *>(h - 1) = __byte_perm(before, w, 0x5432);
                    else h[0] = (uint16_t)w;
                    if (odd && j == WORDS - 1) h[1] = (uint16_t)(w >> 16);
                }
            }
        }
    } else {
        for (int r = first; r < n; r += TOGETHER, p += TOGETHER * ld) {
            const uint32_t w = room[r * PITCH + j];
            if constexpr (N == 1) {
                if (col + j < cols) reinterpret_cast<uint32_t *>(p)[j] = w;
            } else {
                uint16_t *const h = reinterpret_cast<uint16_t *>(p) + 2 * j;
                if (col + 2 * j < cols) h[0] = (uint16_t)w;
                if (col + 2 * j + 1 < cols) h[1] = (uint16_t)(w >> 16);
            }
        }
    }
}

// The same of 32 columns of a 16-bit type, in aligned pieces of 16 bytes, put together from words in the middle of which a piece may start, and what lies before a
// row's first and behind its last such piece value by value.  (8000 x 8001 x 512 BF16 95 us, with store_any 128.  With sixteen columns, of which half lie at such
// ends, it is store_any that is faster: gated 8000 x 8001 x 512 382 and 428 us; of 32 columns of FP32 values too, 4000 x 3001 x 300 19.5 and 25.6.)
template <typename T>
__device__ __forceinline__ void store_pieces(const float *f, T *to, uint64_t ld, uint32_t row0, uint32_t rows, uint32_t col, uint32_t cols, int lane, uint32_t *room)
{
    constexpr int COLS = 32, N = Word<T>::N, WORDS = COLS / N, PITCH = WORDS + 1, BYTES = 4 * WORDS, PIECES = BYTES / 16, E = 16 / (int)sizeof(T);
    constexpr int ROWS = 32 / PIECES, EDGE_ROWS = 32 / E;          // of a turn of the warp
    static_assert(N == 2 && 32 * PITCH * 4 <= 6 * 1024, "");
    __syncwarp();
#pragma unroll
    for (int j = 0; j < WORDS; ++j) room[lane * PITCH + j] = Word<T>::pack(f + j * N);
    __syncwarp();
    const int n = row0 < rows ? (int)min(32u, rows - row0) : 0, bytes = (int)min((uint32_t)COLS, cols - col) * (int)sizeof(T);
    const uint64_t pitch = ld * sizeof(T);
    uint8_t *const start = reinterpret_cast<uint8_t *>(to + (uint64_t)row0 * ld + col);
    // piece p of a row holds its bytes from 16 p - shift on
    {
        const int first = lane / PIECES, p = lane % PIECES;
        uint8_t *at = start + first * pitch;
#pragma unroll
        for (int r = first; r < 32; r += ROWS, at += ROWS * pitch) {
            const int shift = (int)(reinterpret_cast<uintptr_t>(at) & 15), o = 16 * p - shift, w = max(o, 0) / 4;
            const uint32_t *const from = room + r * PITCH + w;
            uint32_t v[4];
            const uint32_t by = (shift & 2) * 8;
            uint32_t here = from[0];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t next = from[i + 1];         // (behind the row's last word a pad, of which nothing is taken)
                v[i] = __funnelshift_r(here, next, by);
                here = next;
            }
            if (r < n && o >= 0 && o + 16 <= bytes) *reinterpret_cast<uint4 *>(at + o) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
    {
        const int first = lane / E, e = lane % E * (int)sizeof(T);
        uint8_t *at = start + first * pitch;
#pragma unroll
        for (int r = first; r < 32; r += EDGE_ROWS, at += EDGE_ROWS * pitch) {
            const uint8_t *const from = reinterpret_cast<const uint8_t *>(room + r * PITCH);
            const int before = -(int)reinterpret_cast<uintptr_t>(at) & 15, behind = ((bytes - before) & ~15) + before;       // (behind < 0: the row ends before a piece starts)
            // of whole rows of pieces as many values lie before the first as are missing behind the last
            const int o = bytes == BYTES && e >= before ? BYTES - 16 + e : e;
            if (r < n && o < bytes && (o < before || (bytes == BYTES && before > 0))) *reinterpret_cast<T *>(at + o) = *reinterpret_cast<const T *>(from + o);
            if (bytes < BYTES && r < n && behind >= before && behind + e < bytes) *reinterpret_cast<T *>(at + behind + e) = *reinterpret_cast<const T *>(from + behind + e);
        }
    }
}

// Rows on 16-byte boundaries: a warp's boxes of 32 rows go out as bulk tensor stores, which write whole sectors and clip at the matrix's ends.
// (They clip whole pieces of 16 bytes: a matrix 257 FP32 values wide got 260 written.)
// (With each lane storing its own row, 32 bytes at a time, the stores took the load/store unit's time: 8192 x 8192 x 256 BF16 46.7 us.)
// A box is 64 bytes wide, three a warp in turn; in the gated layer of 16-bit types 32 bytes, sixteen columns, so that there are two sets of three (y, a, b).
// (Sixteen warps instead of eight for the largest tiles: 8192 x 8192 x 256 BF16 37 instead of 40 us, but a stage less, 16384 x 2048 x 8192 174 instead of 165 us.)
template <typename T, bool GATED>
struct Box {
    static constexpr int BYTES = GATED && sizeof(T) == 2 ? 32 : 64, COLS = BYTES / (int)sizeof(T), SIZE = 32 * BYTES;
};
// Sixteen values of a lane's row into a box, from its 16-byte piece `piece` on.  64-byte swizzle: piece p of row r sits at piece p ^ (r / 2 mod 4); 32-byte:
// at p ^ (r / 4 mod 2).  Either way eight lanes' pieces fall into different banks.
template <typename T, int BYTES>
__device__ __forceinline__ void box16(uint32_t box, int piece, const float *f, int lane)
{
    constexpr int N = Word<T>::N;
    const uint32_t turn = BYTES == 64 ? (lane >> 1) & 3 : (lane >> 2) & 1;
#pragma unroll
    for (int i = 0; i < 16 / (4 * N); ++i) {
        const uint32_t at = box + lane * BYTES + (((piece + i) ^ turn) << 4);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(Word<T>::pack(f + (4 * i) * N)), "r"(Word<T>::pack(f + (4 * i + 1) * N)),
                     "r"(Word<T>::pack(f + (4 * i + 2) * N)), "r"(Word<T>::pack(f + (4 * i + 3) * N)) : "memory");
    }
}
// Waits until at most PENDING of this warp's stores still read their boxes.
template <int PENDING>
__device__ __forceinline__ void boxes_free(int lane)
{
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
}
__device__ __forceinline__ void boxes_written() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); __syncwarp(); }
__device__ __forceinline__ void send_box(uint32_t box, const CUtensorMap *map, uint32_t col, uint32_t row, int lane)
{
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(col), "r"(row), "r"(box) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}

// Where Y, a and b go, as tensor maps (rows on 16-byte boundaries).
struct Targets {
    CUtensorMap y, a, b;
};

template <int CG, int BN, typename T, bool GATED, typename WAITS>
__global__ void __launch_bounds__(Tile<CG, BN, GATED>::THREADS, 1)
i8_tile_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ Targets to, Result<T> o, uint32_t whole,
               WAITS waits)
{
    using C = Tile<CG, BN, GATED>;
    constexpr int NS = C::NSTAGES, TN = C::COLS, TM = 128 * CG;
    constexpr uint32_t IDESC = instr_desc(TM, BN);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - saddr(smem_raw));
    float *const scales = reinterpret_cast<float *>(base_ptr + NS * C::STAGE);
    const uint32_t bars = base + NS * C::STAGE + C::SCALES + C::ROOM;      // full[NS], empty[NS], acc_full[2], acc_empty[2], drained; tmem slot, gave_up
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * NS + b); };
    auto acc_empty = [&](int b) { return bars + 8u * (2 * NS + 2 + b); };
    const uint32_t drained = bars + 8u * (C::BARRIERS - 1), tmem_slot = bars + 8u * C::BARRIERS, gave_up = tmem_slot + 4u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_cta_rank() : 0u;         // 0: the leader
    const uint32_t ksteps = (o.K + BK - 1) / BK;
    const uint32_t tiles_m = (o.M + TM - 1) / TM, tiles_n = (o.N + TN - 1) / TN, ntiles = tiles_m * tiles_n;
    const uint32_t unit = blockIdx.x / CG, units = gridDim.x / CG;
    auto commit = [&](uint32_t bar) {
        if constexpr (CG == 2) umma_commit_pair(bar);
        else umma_commit(bar);
    };

    if (tid == 64) {
        prefetch_map(&map_x);
        prefetch_map(&map_w);
        if (whole) prefetch_map(&to.y);
    }
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), CG * C::STORE_WARPS); }
        mbar_init(drained, 1);
        shared_word(gave_up, 0u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // with a tile each the next kernel may take the SMs that are left at once, else when the last tile's sums are there
    if (ntiles <= units) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 1) {          // with two CTAs the same warp of both takes the pair's tensor memory
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    fence_after();
    const uint32_t tmem_base = shared_word(tmem_slot);

    bool ok = true;
    if (tid == 0) {
        uint32_t it = 0;
        for (uint32_t t = unit; t < ntiles && ok; t += units) {
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            const int xr = (int)(tm * TM + rank * 128), wr = (int)(tn * TN + (CG == 2 ? rank * (GATED ? o.N : (uint32_t)C::W_ROWS) : 0u));
            for (uint32_t k = 0; k < ksteps; ++k, ++it) {
                const int s = it % NS;
                if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, waits.polls);
                if (!ok) break;
                if (rank == 0) mbar_expect_tx(full(s), CG * C::STAGE);          // the bytes of both CTAs
                if (waits.missing(unit)) continue;
                const uint32_t a = base + s * C::STAGE;
                if constexpr (CG == 2) {
                    const uint32_t lead_full = map_to_cta(full(s), 0u);
                    tma_load_2d_pair(a, &map_x, (int)(k * BK), xr, lead_full);
                    tma_load_2d_pair(a + TILE_BYTES, &map_w, (int)(k * BK), wr, lead_full);
                } else {
                    tma_load_2d(a, &map_x, (int)(k * BK), xr, full(s));
                    tma_load_2d(a + TILE_BYTES, &map_w, (int)(k * BK), wr, full(s));
                    if constexpr (GATED) tma_load_2d(a + TILE_BYTES + C::W_BOX * BK, &map_w, (int)(k * BK), wr + (int)o.N, full(s));
                }
            }
        }
        // (the peer's copies tell the leader; the products that read them tell both: without this a peer that had issued its last copies could end before they
        // landed, if the leader gave up meanwhile)
        if (rank == 0) copies_landed(it, NS, waits.held, full);
        else copies_landed(it, NS, waits.held, empty);
    } else if (tid == 32 && rank == 0) {
        uint32_t it = 0, lt = 0;
        for (uint32_t t = unit; t < ntiles && ok; t += units, ++lt) {
            const uint32_t buf = lt & 1u;
            if (lt >= 2) ok = mbar_wait(acc_empty(buf), ((lt >> 1) - 1) & 1u, waits.polls);
            if (!ok) break;
            fence_after();
            const uint32_t d = tmem_base + buf * BN;
            for (uint32_t k = 0; k < ksteps; ++k, ++it) {
                const int s = it % NS;
                ok = mbar_wait_held(full(s), (it / NS) & 1u, waits.held);
                if (!ok) break;
                fence_after();
                const uint32_t a = base + s * C::STAGE, b = a + TILE_BYTES;
#pragma unroll
                for (int i = 0; i < BK / INSTR_K; ++i) {
                    if constexpr (CG == 2) mma_i8_pair(d, umma_desc(a + i * INSTR_K), umma_desc(b + i * INSTR_K), IDESC, (k | (uint32_t)i) != 0);
                    else mma_i8(d, umma_desc(a + i * INSTR_K), umma_desc(b + i * INSTR_K), IDESC, (k | (uint32_t)i) != 0);
                }
                commit(empty(s));          // the stage goes back to both producers
            }
            if (ok) commit(acc_full(buf));
        }
    } else if (warp >= 2) {
        const int q = warp & 3, part_of_row = (warp - 2) >> 2, mine = tid - 64;
        using B = Box<T, GATED>;
        constexpr int PER_BOX = B::COLS, BOXES = C::ROOM_EACH / B::SIZE, SETS = BOXES / 3, SHARE = TN / (C::STORE_WARPS / 4);      // columns of a warp
        const uint32_t boxes = base + NS * C::STAGE + C::SCALES + (warp - 2) * C::ROOM_EACH;
        uint32_t *const room = reinterpret_cast<uint32_t *>(base_ptr + NS * C::STAGE + C::SCALES + (warp - 2) * C::ROOM_EACH);
        uint32_t lt = 0, box = 0;                          // the next box, in turn
        // the store of a box clips at multiples of 16 bytes only: the last columns of other widths go out one by one
        const bool ends_whole = o.N * sizeof(T) % 16 == 0;
        auto boxed = [&](uint32_t col) { return whole && (ends_whole || col + PER_BOX <= o.N); };
        for (uint32_t t = unit; t < ntiles; t += units, ++lt) {
            const uint32_t buf = lt & 1u;
            uint32_t tn, tm;
            tile_of(t, tiles_n, tiles_m, tn, tm);
            // the scales of the tile's rows of W, one a thread (a buffer is written again two tiles later: a barrier lies between)
            if (mine < BN) {
                const uint32_t w_row = tn * TN + (GATED ? mine % TN : mine);
                scales[buf * BN + mine] = w_row < o.N ? o.w_scales[w_row + (GATED && mine >= TN ? o.N : 0u)] : 0.f;
            }
            const uint32_t row0 = tm * TM + rank * 128 + q * 32;
            const i8::RowScale xs(row0 + lane < o.M ? o.x_scales[row0 + lane] : 0.f);
            const bool any_big = __any_sync(0xFFFFFFFFu, xs.big());
            ok = together<C::STORE_THREADS>(mbar_wait_held(acc_full(buf), (lt >> 1) & 1u, waits.results(unit)));
            if (t + units >= ntiles) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            if (!ok) break;
            fence_after();
            const uint32_t acc = tmem_base + buf * BN + ((uint32_t)(q * 32) << 16);
            const float4 *ws = reinterpret_cast<const float4 *>(scales + buf * BN);
            const uint32_t col0 = tn * TN;
            const bool rows_here = row0 < o.M;             // of this warp
            // sums of the next columns leave tensor memory while those before are worked on
            const int c_end = min((part_of_row + 1) * SHARE, (int)(o.N - col0));
            if constexpr (GATED) {
                uint32_t v[16], u[16];
                int c = part_of_row * SHARE;
                if (c < c_end) {
                    tmem_load16(acc + c, v);
                    tmem_load16(acc + TN + c, u);
                }
#pragma unroll 1
                for (; c < c_end; c += 16) {
                    tmem_wait();
                    loaded16(v);
                    loaded16(u);
                    float a[16], b[16], y[16];
                    values16(v, xs, any_big, ws + c / 4, a);
                    values16(u, xs, any_big, ws + TN / 4 + c / 4, b);
                    if (c + 16 < c_end) {
                        tmem_load16(acc + c + 16, v);
                        tmem_load16(acc + TN + c + 16, u);
                    }
                    gate16<sizeof(T) == 4>(o.act, a, b, y);
                    const uint32_t col = col0 + c;
                    static_assert(PER_BOX == 16, "");
                    if (boxed(col)) {
                        // a set of three boxes with what is kept, else one
                        if (o.pre) {
                            boxes_free<3 * (SETS - 1)>(lane);
                        } else {
                            boxes_free<BOXES - 1>(lane);
                        }
                        const uint32_t here = boxes + box * B::SIZE;
                        box16<T, B::BYTES>(here, 0, y, lane);
                        if (o.pre) {
                            box16<T, B::BYTES>(here + B::SIZE, 0, a, lane);
                            box16<T, B::BYTES>(here + 2 * B::SIZE, 0, b, lane);
                        }
                        boxes_written();
                        if (rows_here) {
                            send_box(here, &to.y, col, row0, lane);
                            if (o.pre) {
                                send_box(here + B::SIZE, &to.a, col, row0, lane);
                                send_box(here + 2 * B::SIZE, &to.b, col, row0, lane);
                            }
                        }
                        box += o.pre ? 3 : 1;
                        if (box >= (uint32_t)(o.pre ? 3 * SETS : BOXES)) box = 0;
                    } else {
                        boxes_free<0>(lane);
                        if (o.pre) {
                            store_any<T, 16>(a, o.pre, o.ld_pre, row0, o.M, col, o.N, lane, room);
                            store_any<T, 16>(b, o.pre + o.N, o.ld_pre, row0, o.M, col, o.N, lane, room);
                        }
                        store_any<T, 16>(y, o.y, o.ldy, row0, o.M, col, o.N, lane, room);
                    }
                }
            } else {
                uint32_t v[32];
                int c = part_of_row * SHARE;
                if (c < c_end) {
                    tmem_load16(acc + c, v);
                    tmem_load16(acc + c + 16, v + 16);
                }
#pragma unroll 1
                for (; c < c_end; c += 32) {
                    tmem_wait();
                    loaded16(v);
                    loaded16(v + 16);
                    float f[32];
                    values16(v, xs, any_big, ws + c / 4, f);
                    values16(v + 16, xs, any_big, ws + c / 4 + 4, f + 16);
                    if (c + 32 < c_end) {
                        tmem_load16(acc + c + 32, v);
                        tmem_load16(acc + c + 48, v + 16);
                    }
                    if (!whole) {
                        if constexpr (sizeof(T) == 2) store_pieces<T>(f, o.y, o.ldy, row0, o.M, col0 + c, o.N, lane, room);
                        else store_any<T, 32>(f, o.y, o.ldy, row0, o.M, col0 + c, o.N, lane, room);
                        continue;
                    }
#pragma unroll
                    for (int part = 0; part < 32 / PER_BOX; ++part) {
                        const uint32_t col = col0 + c + part * PER_BOX, here = boxes + box * B::SIZE;
                        if (col >= o.N) break;
                        if (boxed(col)) {
                            boxes_free<BOXES - 1>(lane);
#pragma unroll
                            for (int i = 0; i < PER_BOX; i += 16) box16<T, B::BYTES>(here, i * (int)sizeof(T) / 16, f + part * PER_BOX + i, lane);
                            boxes_written();
                            if (rows_here) send_box(here, &to.y, col, row0, lane);
                            box = box == BOXES - 1 ? 0 : box + 1;
                        } else {
                            boxes_free<0>(lane);
                            if constexpr (sizeof(T) == 2) store_pieces<T>(f, o.y, o.ldy, row0, o.M, col, o.N, lane, room);
                            else store_any<T, PER_BOX>(f + part * PER_BOX, o.y, o.ldy, row0, o.M, col, o.N, lane, room);
                        }
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2) arrive_at(map_to_cta(acc_empty(buf), 0u));
                else mbar_arrive(acc_empty(buf));
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    if (!ok) give_up(o.status, gave_up);
    fence_before();
    __syncthreads();
    // what was issued has finished, whichever thread's wait ran out (if none of the leader's did, its results were all waited for)
    if (tid == 32 && rank == 0 && shared_word(gave_up)) {
        commit(drained);
        mbar_wait_held(drained, 0u, HELD_LIMIT);
    }
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();          // neither CTA ends or lets go of tensor memory while the other may still signal it
    if (warp == 1) {
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::TMEM_COLS) : "memory");
    }
}

// ---- few rows of X or few tiles ------------------------------------------------------------------------
// A CTA has one tile of 128 rows of W (gated: of either half of W, with an accumulator each) by NT rows of X, or a range of its K steps.
// With a divided K each CTA of the cluster owns a share of the tile's rows of X and gets the others' sums of these (stores to distributed
// shared memory).  Lanes of tensor memory run along Y's contiguous dimension: a warp's store is 32 neighbouring values.
// Bound by latency: without steps a CTA takes 2.5 us (gated 3.5), a step 0.25 (0.39), as copies, products and results follow one another.  16 x 8192 x 2048 BF16 5.9 us (W's 16.8 MB take 2.6 at the copy
// rate), 64 x 2048 x 8192 8.0 us, 77 x 777 x 1000 5.3 us (8-fold divided K).  (With all of an SM's shared memory for one gated CTA of 16 or 32 rows
// 16 x 8192 x 2048 takes 11.4 us, with two CTAs an SM 7.2.)
template <int NT, bool GATED>
struct Small {
    static constexpr int W_TILES = GATED ? 2 : 1, TILE_X = NT * BK;
    static constexpr int STAGE = W_TILES * TILE_BYTES + TILE_X;
    static constexpr int BUDGET = (GATED && NT > 32 ? 212 : 112) * 1024;           // the latter: two CTAs share an SM
    static constexpr int PARTS = 128 * NT * 4 * W_TILES;                            // sums of the cluster's CTAs for this one's rows
    static constexpr int NSTAGES = (BUDGET - 1024 - 256 - NT * 4 - PARTS) / STAGE;
    static constexpr int SMEM = NSTAGES * STAGE + PARTS + NT * 4 + 1024 + 256;
    static constexpr int COLS = NT < 32 ? 32 : NT, ALL_COLS = W_TILES * COLS;       // of tensor memory
    static constexpr int THREADS = 192;
    static_assert(NSTAGES >= 2 && STAGE % 1024 == 0 && 8 * (2 * NSTAGES + 2) + 8 <= 256, "");
};

template <int NT, typename T, bool GATED, typename WAITS>
__global__ void __launch_bounds__(Small<NT, GATED>::THREADS)
i8_small_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, Result<T> o, uint32_t splits, WAITS waits)
{
    using C = Small<NT, GATED>;
    constexpr int NS = C::NSTAGES;
    constexpr uint32_t IDESC = instr_desc(128, NT);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (saddr(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - saddr(smem_raw));
    float *const scales = reinterpret_cast<float *>(base_ptr + NS * C::STAGE + C::PARTS);      // of the tile's rows of X
    const uint32_t bars = base + NS * C::STAGE + C::PARTS + NT * 4;      // full[NS], empty[NS], done, drained; tmem slot, gave_up
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    const uint32_t done = bars + 8u * (2 * NS), drained = done + 8u, tmem_slot = drained + 8u, gave_up = tmem_slot + 4u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = splits > 1 ? cluster_cta_rank() : 0u;
    const uint32_t tiles_n = (o.N + 127) / 128, tile = blockIdx.x / splits, tm = tile / tiles_n, tn = tile - tm * tiles_n, m0 = tm * NT;
    const uint32_t ksteps = (o.K + BK - 1) / BK;
    const uint32_t k_begin = (uint32_t)((uint64_t)ksteps * rank / splits), k_end = (uint32_t)((uint64_t)ksteps * (rank + 1) / splits);

    if (tid == 64) {
        prefetch_map(&map_x);
        prefetch_map(&map_w);
    }
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1);
        mbar_init(drained, 1);
        shared_word(gave_up, 0u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (splits > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this CTA runs: sums may be put into its shared memory
    el::enter_stream_order();
    // tensor memory is taken while the first copies are on their way; warps 2 .. 5 learn where it is at barrier 1
    uint32_t tmem_base = 0;
    auto read_slot = [&]() {
        fence_after();
        tmem_base = shared_word(tmem_slot);
    };
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::ALL_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
        asm volatile("bar.arrive 1, 160;" ::: "memory");
        read_slot();
    }
    bool ok = true;
    if (tid == 0) {
        uint32_t it = 0;
        for (uint32_t k = k_begin; k < k_end; ++k, ++it) {
            const int s = it % NS;
            if (it >= (uint32_t)NS) ok = mbar_wait(empty(s), ((it / NS) - 1) & 1u, waits.polls);
            if (!ok) break;
            const uint32_t a = base + s * C::STAGE;
            mbar_expect_tx(full(s), C::STAGE);
            if (waits.missing(blockIdx.x)) continue;
            tma_load_2d(a, &map_w, (int)(k * BK), (int)(tn * 128), full(s));
            if constexpr (GATED) tma_load_2d(a + TILE_BYTES, &map_w, (int)(k * BK), (int)(o.N + tn * 128), full(s));
            tma_load_2d(a + C::W_TILES * TILE_BYTES, &map_x, (int)(k * BK), (int)m0, full(s));
        }
        copies_landed(it, NS, waits.held, full);
    } else if (tid == 32) {
        for (uint32_t it = 0; it < k_end - k_begin; ++it) {
            const int s = it % NS;
            ok = mbar_wait_held(full(s), (it / NS) & 1u, waits.held);
            if (!ok) break;
            fence_after();
            const uint32_t a = base + s * C::STAGE, b = a + C::W_TILES * TILE_BYTES;
#pragma unroll
            for (int i = 0; i < BK / INSTR_K; ++i)
#pragma unroll
                for (int w = 0; w < C::W_TILES; ++w)
                    mma_i8(tmem_base + w * C::COLS, umma_desc(a + w * TILE_BYTES + i * INSTR_K), umma_desc(b + i * INSTR_K), IDESC, (it | (uint32_t)i) != 0);
            umma_commit(empty(s));
        }
        if (ok) umma_commit(done);
    }
    __syncwarp();
    const int q = warp & 3;                               // quarter of the lanes a warp may read
    const uint32_t n = tn * 128 + q * 32 + lane, mine = NT / splits;
    float wa = 0.f, wb = 0.f, was[4], wbs[4];             // scales of W's rows: with divided K this lane's four columns of the rows that its warp adds up
    if (splits > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t col = tn * 128 + i * 32 + lane;
            was[i] = col < o.N ? o.w_scales[col] : 0.f;
            wbs[i] = GATED && col < o.N ? o.w_scales[o.N + col] : 0.f;
        }
    } else if (warp >= 2 && n < o.N) {
        wa = o.w_scales[n];
        if constexpr (GATED) wb = o.w_scales[o.N + n];
    }
    if (warp >= 2) {
        for (uint32_t i = tid - 64; i < (uint32_t)NT; i += 128) scales[i] = m0 + i < o.M ? o.x_scales[m0 + i] : 0.f;
        asm volatile("bar.sync 1, 160;" ::: "memory");
        read_slot();
        ok = mbar_wait_held(done, 0u, waits.results(blockIdx.x)) && ok;
        ok = __all_sync(0xFFFFFFFFu, ok);
        fence_after();
    }
    if (splits > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // every CTA of the cluster runs
    if (warp >= 2) {
        if (ok) {
            const uint32_t at = tmem_base + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < NT && m0 + c < o.M; c += 16) {
                uint32_t v[16], u[GATED ? 16 : 1];
                tmem_load16(at + c, v);
                if constexpr (GATED) tmem_load16(at + C::COLS + c, u);
                tmem_wait();
                loaded16(v);
                if constexpr (GATED) loaded16(u);
                if (splits > 1) {
                    // row r of the tile belongs to CTA r / mine, there place r mod mine of part `rank`: [part][row][half of W][128]
                    const uint32_t here = base + NS * C::STAGE + (rank * mine * C::W_TILES * 128 + q * 32 + lane) * 4, shift = 31 - __clz(mine);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (m0 + c + j < o.M) {
                            const uint32_t to = map_to_cta(here + ((c + j) & (mine - 1)) * C::W_TILES * 512, (c + j) >> shift);
                            store_remote(to, v[j]);
                            if constexpr (GATED) store_remote(to + 512, u[j]);
                        }
                } else if (n < o.N) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t m = m0 + c + j;
                        if (m < o.M) {
                            const i8::RowScale xs(scales[c + j]);
                            const float a = i8::value_in_two((int)v[j], xs, wa);
                            if constexpr (GATED) {
                                const float b = i8::value_in_two((int)u[j], xs, wb);
                                if (o.pre) {
                                    o.pre[m * o.ld_pre + n] = el::from_float<T>(a);
                                    o.pre[m * o.ld_pre + o.N + n] = el::from_float<T>(b);
                                }
                                o.y[m * o.ldy + n] = el::from_float<T>(gate1<sizeof(T) == 4>(o.act, a, b));
                            } else {
                                o.y[m * o.ldy + n] = el::from_float<T>(a);
                            }
                        }
                    }
                }
            }
        }
        fence_before();
    }
    if (!ok) give_up(o.status, gave_up);
    __syncwarp();
    __syncthreads();
    if (tid == 32 && shared_word(gave_up)) {               // what was issued has finished, whichever thread's wait ran out
        umma_commit(drained);
        mbar_wait_held(drained, 0u, HELD_LIMIT);
    }
    __syncwarp();
    if (splits > 1) {
        cluster_barrier();                                 // the sums of this CTA's rows have arrived
        const int32_t *parts = reinterpret_cast<const int32_t *>(base_ptr + NS * C::STAGE);
        for (uint32_t r = warp; r < mine; r += C::THREADS / 32) {
            const uint32_t in_tile = rank * mine + r, m = m0 + in_tile;
            if (m >= o.M) break;
            const i8::RowScale xs(scales[in_tile]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t l = i * 32 + lane, col = tn * 128 + l;
                int32_t a = 0, b = 0;
                for (uint32_t p = 0; p < splits; ++p) {
                    const int32_t *part = parts + (p * mine + r) * C::W_TILES * 128 + l;
                    a += part[0];
                    if constexpr (GATED) b += part[128];
                }
                if (col < o.N) {
                    const float fa = i8::value_in_two(a, xs, was[i]);
                    if constexpr (GATED) {
                        const float fb = i8::value_in_two(b, xs, wbs[i]);
                        if (o.pre) {
                            o.pre[m * o.ld_pre + col] = el::from_float<T>(fa);
                            o.pre[m * o.ld_pre + o.N + col] = el::from_float<T>(fb);
                        }
                        o.y[m * o.ldy + col] = el::from_float<T>(gate1<sizeof(T) == 4>(o.act, fa, fb));
                    } else {
                        o.y[m * o.ldy + col] = el::from_float<T>(fa);
                    }
                }
            }
        }
    }
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::ALL_COLS) : "memory");
}

// ---- up to four rows of X --------------------------------------------------------------------------------
// W is read once, sixteen bytes a lane, and multiplied with dp4a against X's codes in shared memory; a chunk's registers take the next one as soon as they are free, and
// a warp adds up its lanes' sums at the end of its four rows.  Bound by W's bytes: 1 x 8192 x 2048 with quantisation 3.4 us (4.9 TB/s; 2.6 at the copy rate),
// 1 x 32768 x 4096 23.3 us (5.8 TB/s), four rows against 8192 x 2048 5.7 us, gated 1 x 2048 x 512 2.3 us.  (Neighbouring rows of W in the warps of a CTA, so that
// some SMs have twice the others': 1 x 2048 x 8192 6.3 us, now 5.7.)
constexpr int ROWS_THREADS = 256, ROWS_WARPS = 8, W_ROWS = 4, CHUNKS = 4;      // W rows of a warp at a time; 512-byte chunks on their way

// Rows of X in memory, quantised already or not.
struct Codes {
    const int8_t *codes;
    const float *scales;
};
template <typename TX, bool VECTOR>
struct Values {
    const TX *x;
    uint64_t ld;
};

// Codes of rows m < M to shared memory ([MT][pitch], zeros behind), their scales too.  All threads of the CTA.
template <int MT>
__device__ __forceinline__ void bring_rows(const Codes &s, uint32_t M, uint32_t K, uint32_t pitch, int8_t *codes, float *scales, uint32_t *)
{
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        for (uint32_t c = threadIdx.x * 16; c < pitch; c += ROWS_THREADS * 16) {
            uint4 q = make_uint4(0u, 0u, 0u, 0u);
            if (m < (int)M) q = *reinterpret_cast<const uint4 *>(s.codes + (uint64_t)m * pitch + c);
            *reinterpret_cast<uint4 *>(codes + m * pitch + c) = q;
        }
        if (threadIdx.x == 0) scales[m] = m < (int)M ? s.scales[m] : 0.f;
    }
    __syncthreads();
}
template <int MT, typename TX, bool VECTOR>
__device__ __forceinline__ void bring_rows(const Values<TX, VECTOR> &s, uint32_t M, uint32_t K, uint32_t pitch, int8_t *codes, float *scales, uint32_t *slots)
{
    constexpr int E = i8::PIECE<TX>;
    const uint32_t col = threadIdx.x * E;
    uint32_t first[MT][4], top[MT];                        // a thread's first piece of each row stays in registers
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int i = 0; i < 4; ++i) first[m][i] = 0u;
        if (m < (int)M && col < K) mx::load<TX, VECTOR, E>(s.x + m * s.ld, col, K, first[m]);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        uint32_t t = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = mx::max_magnitude<TX>(t, first[m][i] & i8::MAGNITUDE<TX>);
        if (m < (int)M)
            for (uint32_t c = col + ROWS_THREADS * E; c < K; c += ROWS_THREADS * E) {
                uint32_t w[4];
                mx::load<TX, VECTOR, E>(s.x + m * s.ld, c, K, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) t = mx::max_magnitude<TX>(t, w[i] & i8::MAGNITUDE<TX>);
            }
        top[m] = __reduce_max_sync(0xFFFFFFFFu, i8::top_bits<TX>(t));
    }
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int m = 0; m < MT; ++m) slots[m * ROWS_WARPS + (threadIdx.x >> 5)] = top[m];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        uint32_t t = 0u;
#pragma unroll
        for (int i = 0; i < ROWS_WARPS; ++i) t = max(t, slots[m * ROWS_WARPS + i]);
        const i8::Scale sc = i8::scale_of(t);
        if (threadIdx.x == 0) scales[m] = m < (int)M ? sc.s : 0.f;
        for (uint32_t c = col; c < pitch; c += ROWS_THREADS * E) {
            uint32_t w[4] = {0u, 0u, 0u, 0u}, q[E / 4];
            if (c == col) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = first[m][i];
            } else if (m < (int)M && c < K) {
                mx::load<TX, VECTOR, E>(s.x + m * s.ld, c, K, w);
            }
            i8::encode_piece<TX>(w, sc.r, sc.nan(), q);
            i8::store_codes<E>(codes + m * pitch, c, E, q);
        }
    }
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ void put(void *p, uint64_t at, float v) { static_cast<T *>(p)[at] = el::from_float<T>(v); }
__device__ __forceinline__ void put(int type, void *p, uint64_t at, float v)
{
    if (type == OMC_TYPE_F32) put<float>(p, at, v);
    else if (type == OMC_TYPE_F16) put<__half>(p, at, v);
    else put<__nv_bfloat16>(p, at, v);
}

template <int MT, bool GATED, typename SOURCE>
__global__ void __launch_bounds__(ROWS_THREADS, 2)
i8_rows_kernel(SOURCE source, const int8_t *w_codes, const float *w_scales, void *y, int type, uint64_t ldy, void *pre, uint64_t ld_pre, uint32_t M,
               uint32_t N, uint32_t K, int act)
{
    constexpr int OUTS = GATED ? W_ROWS / 2 : W_ROWS;     // columns of Y of a warp at a time
    extern __shared__ __align__(16) uint8_t smem_raw[];
    int8_t *const codes = reinterpret_cast<int8_t *>(smem_raw);
    __shared__ float scales[MT];
    __shared__ uint32_t slots[MT * ROWS_WARPS];
    const uint32_t pitch = (uint32_t)i8::row_bytes(K), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t tasks = (N + OUTS - 1) / OUTS, step = gridDim.x * ROWS_WARPS;
    uint32_t task = blockIdx.x + warp * gridDim.x;        // every SM the same number of them, within one a CTA
    el::enter_stream_order();
    uint4 w[CHUNKS][W_ROWS];
    // row r of W of a task: gated, the gate's rows first; rows that do not exist are the last one again
    auto row_of = [&](uint32_t t, int r) -> const int8_t * {
        const uint32_t n = min(t * OUTS + r % OUTS, N - 1) + (GATED && r >= OUTS ? N : 0u);
        return w_codes + (uint64_t)n * pitch;
    };
    auto fetch = [&](uint32_t t, uint32_t k0, int c) {
#pragma unroll
        for (int r = 0; r < W_ROWS; ++r) {
            const uint32_t k = k0 + c * 512 + lane * 16;
            w[c][r] = k < pitch ? *reinterpret_cast<const uint4 *>(row_of(t, r) + k) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    if (task < tasks) {                                    // on its way while X is quantised
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) fetch(task, 0, c);
    }
    bring_rows<MT>(source, M, K, pitch, codes, scales, slots);
    for (; task < tasks; task += step) {
        const uint32_t n = task * OUTS + lane / MT, m = lane % MT;
        const bool mine = lane < OUTS * MT && n < N && m < M;
        const float wa = mine ? w_scales[n] : 0.f, wb = GATED && mine ? w_scales[N + n] : 0.f;
        int32_t acc[W_ROWS][MT];
#pragma unroll
        for (int i = 0; i < W_ROWS * MT; ++i) acc[i / MT][i % MT] = 0;
        for (uint32_t k0 = 0; k0 < pitch; k0 += CHUNKS * 512) {
            const bool more = k0 + CHUNKS * 512 < pitch;   // of these rows of W
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t k = k0 + c * 512 + lane * 16;
                if (k < pitch)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(codes + m * pitch + k);
#pragma unroll
                        for (int r = 0; r < W_ROWS; ++r) {
                            acc[r][m] = __dp4a((int)w[c][r].x, (int)x.x, acc[r][m]);
                            acc[r][m] = __dp4a((int)w[c][r].y, (int)x.y, acc[r][m]);
                            acc[r][m] = __dp4a((int)w[c][r].z, (int)x.z, acc[r][m]);
                            acc[r][m] = __dp4a((int)w[c][r].w, (int)x.w, acc[r][m]);
                        }
                    }
                if (more || task + step < tasks) fetch(more ? task : task + step, more ? k0 + CHUNKS * 512 : 0u, c);
            }
        }
        int32_t a = 0, b = 0;                              // lane i < OUTS MT has the sums of column i / MT, row i mod MT
#pragma unroll
        for (int i = 0; i < W_ROWS * MT; ++i) {
            const int32_t sum = __reduce_add_sync(0xFFFFFFFFu, acc[i / MT][i % MT]);
            if (i < OUTS * MT) a = lane == (uint32_t)i ? sum : a;
            else b = lane == (uint32_t)(i - OUTS * MT) ? sum : b;
        }
        if (mine) {
            const i8::RowScale xs(scales[m]);
            const float fa = i8::value_in_two(a, xs, wa);
            if constexpr (GATED) {
                const float fb = i8::value_in_two(b, xs, wb);
                if (pre) {
                    put(type, pre, m * ld_pre + n, fa);
                    put(type, pre, m * ld_pre + N + n, fb);
                }
                put(type, y, m * ldy + n, type == OMC_TYPE_F32 ? gate1<true>(act, fa, fb) : gate1<false>(act, fa, fb));
            } else {
                put(type, y, m * ldy + n, fa);
            }
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------------------
// Codes as bytes, the zeros that pad the rows included: boxes of box_rows rows x 128 bytes, 128-byte swizzle, zeros outside.
bool make_codes_map(CUtensorMap *m, const void *ptr, uint64_t rows, uint64_t cols, uint32_t box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {i8::row_bytes(cols), rows};
    const cuuint64_t strides[1] = {i8::row_bytes(cols)};
    const cuuint32_t box[2] = {BK, box_rows};
    const cuuint32_t elem[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Product {
    const int8_t *x_codes;
    const float *x_scales;
    const int8_t *w_codes;
    const float *w_scales;
    uint32_t M, N, K;         // N: columns of Y
    bool gated;
    int act;
    void *y;
    uint64_t ldy;
    void *pre;
    uint64_t ld_pre;
    int type;
    uint32_t *status;
    void *stream;
    uint64_t w_rows() const { return gated ? 2ull * N : N; }
};

// What omc_byte_inject_wait_timeout asked for, for the calling thread's next product of more than four rows with FP32 results (what = 0: nothing).
thread_local Trial next_trial = {0u, 0u, 0u};
Trial take_trial()
{
    const Trial t = next_trial;
    next_trial = {0u, 0u, 0u};
    return t;
}

template <typename T>
Result<T> result_of(const Product &p)
{
    return {p.x_scales, p.w_scales, static_cast<T *>(p.y), static_cast<T *>(p.pre), p.ldy, p.ld_pre, p.M, p.N, p.K, p.act, p.status};
}

// A result matrix in boxes of 32 rows.
template <typename T, bool GATED>
bool make_result_map(CUtensorMap *m, T *p, uint64_t rows, uint64_t cols, uint64_t ld)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {ld * sizeof(T)};
    const cuuint32_t box[2] = {(cuuint32_t)Box<T, GATED>::COLS, 32};
    const cuuint32_t elem[2] = {1, 1};
    const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    return fn(m, type, 2, p, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
              Box<T, GATED>::BYTES == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Whether rows start on 16-byte boundaries, and `second` values on from there.
template <typename T>
bool whole_rows(const T *p, uint64_t ld, uint64_t second)
{
    return ((uint64_t)reinterpret_cast<uintptr_t>(p) | ld * sizeof(T) | second * sizeof(T)) % 16 == 0;
}

// Whether every row of the results can go out in boxes (a tensor map's pitch is below 2^40 bytes).
template <typename T>
bool whole_results(const Product &p)
{
    return whole_rows(static_cast<const T *>(p.y), p.ldy, 0) && p.ldy < (1ull << 37) &&
           (!p.pre || (whole_rows(static_cast<const T *>(p.pre), p.ld_pre, p.N) && p.ld_pre < (1ull << 37)));
}

template <int CG, int BN, typename T, bool GATED, typename WAITS>
int launch_tiles(const Product &p, WAITS waits)
{
    using C = Tile<CG, BN, GATED>;
    CUtensorMap map_x, map_w;
    if (!make_codes_map(&map_x, p.x_codes, p.M, p.K, 128) || !make_codes_map(&map_w, p.w_codes, p.w_rows(), p.K, C::W_BOX)) return OMC_ERR_CUDA;
    if (const int rc = el::allow_smem<i8_tile_kernel<CG, BN, T, GATED, WAITS>>(C::SMEM)) return rc;
    const uint64_t tiles = (uint64_t)((p.M + 128 * CG - 1) / (128 * CG)) * ((p.N + C::COLS - 1) / C::COLS), units = el::sm_count() > CG ? el::sm_count() / CG : 1;
    if (tiles >= (1ull << 31)) return OMC_ERR_INVALID_ARG;
    const Result<T> r = result_of<T>(p);
    Targets to = {};
    const bool whole = whole_results<T>(p);
    if (whole && !make_result_map<T, GATED>(&to.y, r.y, p.M, p.N, r.ldy)) return OMC_ERR_CUDA;
    if (whole && r.pre && (!make_result_map<T, GATED>(&to.a, r.pre, p.M, p.N, r.ld_pre) || !make_result_map<T, GATED>(&to.b, r.pre + p.N, p.M, p.N, r.ld_pre))) return OMC_ERR_CUDA;
    return note_cuda(el::launch(i8_tile_kernel<CG, BN, T, GATED, WAITS>, dim3(CG * (uint32_t)(tiles < units ? tiles : units)), C::THREADS, C::SMEM, CG, p.stream,
                                map_x, map_w, to, r, (uint32_t)whole, waits));
}

template <int NT, typename T, bool GATED, typename WAITS>
int launch_small(const Product &p, uint32_t splits, WAITS waits)
{
    using C = Small<NT, GATED>;
    CUtensorMap map_x, map_w;
    if (!make_codes_map(&map_x, p.x_codes, p.M, p.K, NT) || !make_codes_map(&map_w, p.w_codes, p.w_rows(), p.K, 128)) return OMC_ERR_CUDA;
    if (const int rc = el::allow_smem<i8_small_kernel<NT, T, GATED, WAITS>>(C::SMEM)) return rc;
    const uint64_t tiles = (uint64_t)((p.M + NT - 1) / NT) * ((p.N + 127) / 128);
    if (tiles * splits >= (1ull << 31)) return OMC_ERR_INVALID_ARG;
    return note_cuda(el::launch(i8_small_kernel<NT, T, GATED, WAITS>, dim3((uint32_t)tiles * splits), C::THREADS, C::SMEM, splits, p.stream, map_x, map_w,
                                result_of<T>(p), splits, waits));
}

template <typename T, bool GATED, typename WAITS>
int launch_any(const Product &p, WAITS waits)
{
    const i8::Schedule s = i8::schedule_of(p.M, p.N, p.K, GATED, whole_results<T>(p));
    switch (s.kernel) {
    case i8::PAIR_256: return launch_tiles<2, 256, T, GATED>(p, waits);
    case i8::ONE_128: return launch_tiles<1, 128, T, GATED>(p, waits);
    case i8::SMALL_16: return launch_small<16, T, GATED>(p, s.splits, waits);
    case i8::SMALL_32: return launch_small<32, T, GATED>(p, s.splits, waits);
    default: return launch_small<64, T, GATED>(p, s.splits, waits);
    }
}

template <int MT, bool GATED, typename SOURCE>
int launch_rows(const Product &p, const SOURCE &source)
{
    const uint32_t smem = MT * (uint32_t)i8::row_bytes(p.K);
    if (const int rc = el::allow_smem<i8_rows_kernel<MT, GATED, SOURCE>>(smem)) return rc;
    const uint32_t outs = GATED ? W_ROWS / 2 : W_ROWS, tasks = (p.N + outs - 1) / outs, most = 2 * DEFAULT_SMS;
    return note_cuda(el::launch(i8_rows_kernel<MT, GATED, SOURCE>, dim3(tasks < most ? tasks : most), ROWS_THREADS, smem, 1, p.stream, source, p.w_codes,
                                p.w_scales, p.y, p.type, p.ldy, p.pre, p.ld_pre, p.M, p.N, p.K, p.act));
}
template <bool GATED, typename SOURCE>
int launch_rows_by_count(const Product &p, const SOURCE &source)
{
    if (p.M == 1) return launch_rows<1, GATED>(p, source);
    return p.M == 2 ? launch_rows<2, GATED>(p, source) : launch_rows<4, GATED>(p, source);
}
template <typename SOURCE>
int product_of_rows(const Product &p, const SOURCE &source)
{
    return p.gated ? launch_rows_by_count<true>(p, source) : launch_rows_by_count<false>(p, source);
}

template <bool GATED>
int product_on_tensor_cores(const Product &p)
{
    if (p.type == OMC_TYPE_F16) return launch_any<__half, GATED>(p, Usual());
    if (p.type == OMC_TYPE_BF16) return launch_any<__nv_bfloat16, GATED>(p, Usual());
    const Trial trial = take_trial();
    return trial.what ? launch_any<float, GATED>(p, trial) : launch_any<float, GATED>(p, Usual());
}

int product(const Product &p)
{
    if (i8::few_rows(p.M, p.K)) return product_of_rows(p, Codes{p.x_codes, p.x_scales});
    return p.gated ? product_on_tensor_cores<true>(p) : product_on_tensor_cores<false>(p);
}

template <typename TX>
int product_of_values(const Product &p, const void *x, uint64_t ld)
{
    if (el::aligned16(x) && ld * sizeof(TX) % 16 == 0) return product_of_rows(p, Values<TX, true>{static_cast<const TX *>(x), ld});
    return product_of_rows(p, Values<TX, false>{static_cast<const TX *>(x), ld});
}

// p without its X: values, quantised inside the product where that has few rows, else into the workspace.
int linear(Product p, const void *x, int type, uint64_t ldx, uint8_t *workspace)
{
    if (i8::few_rows(p.M, p.K))
        return type == OMC_TYPE_F32 ? product_of_values<float>(p, x, ldx) : type == OMC_TYPE_F16 ? product_of_values<__half>(p, x, ldx) : product_of_values<__nv_bfloat16>(p, x, ldx);
    int8_t *const codes = reinterpret_cast<int8_t *>(workspace);
    float *const scales = reinterpret_cast<float *>(workspace + p.M * i8::row_bytes(p.K));
    if (const int rc = omc_byte_quantise(x, type, p.M, p.K, ldx, codes, scales, nullptr, nullptr, nullptr, p.stream)) return rc;
    p.x_codes = codes;
    p.x_scales = scales;
    return product(p);
}

bool product_shape_ok(uint64_t M, uint64_t N, uint64_t K)
{
    return i8_shape_ok(M, K) && i8_shape_ok(N, K) && M <= 128ull * 65535 && K <= i8::MOST_K;
}
bool off(const void *p, uint64_t size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

// Checks that the four calls share.
int check(const Product &p, uint64_t M, uint64_t N, uint64_t K)
{
    if (!el::type_ok(p.type) || p.act < OMC_GATE_SIGMOID || p.act > OMC_GATE_GELU) return OMC_ERR_INVALID_ARG;
    if (!p.w_codes || !p.w_scales || !p.y || !p.status) return OMC_ERR_NULL_PTR;
    if (!product_shape_ok(M, N, K) || (p.gated && !i8_shape_ok(2 * N, K)) || p.ldy < N || (p.pre && p.ld_pre < 2 * N)) return OMC_ERR_INVALID_ARG;
    const uint64_t size = el::size_of(p.type);
    return !el::aligned16(p.w_codes) || off(p.w_scales, 4) || off(p.y, size) || off(p.pre, size) || off(p.status, 4) ? OMC_ERR_MISALIGNED : OMC_OK;
}

int of_codes(const Product &p, uint64_t M, uint64_t N, uint64_t K)
{
    if (!p.x_codes || !p.x_scales) return OMC_ERR_NULL_PTR;
    if (const int rc = check(p, M, N, K)) return rc;
    if (!el::aligned16(p.x_codes) || off(p.x_scales, 4)) return OMC_ERR_MISALIGNED;
    return product(p);
}

int of_values(const Product &p, uint64_t M, uint64_t N, uint64_t K, const void *x, int type, uint64_t ldx, uint8_t *workspace)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!x || !workspace) return OMC_ERR_NULL_PTR;
    if (const int rc = check(p, M, N, K)) return rc;
    if (ldx < K) return OMC_ERR_INVALID_ARG;
    if (off(x, el::size_of(type)) || !el::aligned16(workspace)) return OMC_ERR_MISALIGNED;
    return linear(p, x, type, ldx, workspace);
}

}  // namespace

extern "C" int omc_byte_matmul(const int8_t *x_codes, const float *x_scales, uint64_t M, const int8_t *w_codes, const float *w_scales, uint64_t N, uint64_t K,
                             void *y, int type, uint64_t ldy, uint32_t *status, void *stream)
{
    return of_codes({x_codes, x_scales, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, false, 0, y, ldy, nullptr, 0, type, status, stream}, M, N, K);
}

extern "C" int omc_byte_linear(const void *x, int type, uint64_t M, uint64_t K, uint64_t ldx, const int8_t *w_codes, const float *w_scales, uint64_t N, void *y,
                             int y_type, uint64_t ldy, uint8_t *workspace, uint32_t *status, void *stream)
{
    return of_values({nullptr, nullptr, w_codes, w_scales, (uint32_t)M, (uint32_t)N, (uint32_t)K, false, 0, y, ldy, nullptr, 0, y_type, status, stream}, M, N, K,
                     x, type, ldx, workspace);
}

extern "C" int omc_byte_gated(const int8_t *x_codes, const float *x_scales, uint64_t M, const int8_t *w_codes, const float *w_scales, uint64_t F, uint64_t K,
                            int activation, void *y, int type, uint64_t ldy, void *pre, uint64_t ld_pre, uint32_t *status, void *stream)
{
    return of_codes({x_codes, x_scales, w_codes, w_scales, (uint32_t)M, (uint32_t)F, (uint32_t)K, true, activation, y, ldy, pre, ld_pre, type, status, stream}, M,
                    F, K);
}

extern "C" int omc_byte_gated_linear(const void *x, int type, uint64_t M, uint64_t K, uint64_t ldx, const int8_t *w_codes, const float *w_scales, uint64_t F,
                                   int activation, void *y, int y_type, uint64_t ldy, void *pre, uint64_t ld_pre, uint8_t *workspace, uint32_t *status,
                                   void *stream)
{
    return of_values({nullptr, nullptr, w_codes, w_scales, (uint32_t)M, (uint32_t)F, (uint32_t)K, true, activation, y, ldy, pre, ld_pre, y_type, status, stream},
                     M, F, K, x, type, ldx, workspace);
}

extern "C" int omc_byte_inject_wait_timeout(uint32_t polls, int what)
{
    if (polls < 1 || polls > (1u << 16) || (what != OMC_BYTE_COPIES_MISSING && what != OMC_BYTE_RESULTS_LATE)) return OMC_ERR_INVALID_ARG;
    next_trial = {polls, polls, (uint32_t)what};
    return OMC_OK;
}
