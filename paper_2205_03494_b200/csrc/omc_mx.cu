// omc_mx_quantise / omc_mx_dequantise: the 4-bit microscaled format (mx_format.cuh).
//
// Both directions read the values once.  Along the rows 32 bytes of values sit in a lane and a block of 32 values in two
// or four lanes, so that the largest magnitude takes one or two shuffles; along the columns a tile of 128 x 128 goes
// through shared memory and a thread holds whole blocks.  The scale is a power of two, so that scaling is exact and
// the only rounding is the conversion to E2M1.
// Memory bounds the kernels along the rows and back (16384 x 8192 BF16 52 us, 6.5 TB/s; 8192 x 2048 FP32 back 11.0 us, 6.9 TB/s:
// the rate of a plain copy).  Both ways at once (8192 x 8192 BF16 40 us, 5.2 TB/s; 8192 x 2048 FP32 17.6 us, 4.8 TB/s) nothing is
// used up (issue slots 68 %, L1 62 %, DRAM 50 %): each value is scaled and rounded twice, and a CTA loads its one tile, encodes it and stores
// it in turn, with barriers between.  Along the columns alone (32 us, 5.2 TB/s; 12.8 us, 5.9 TB/s) it is these phases too
// (issue slots 48 %, waiting for loads).  Copying the tile past the registers (cp.async) was slower, 54 us.
// Off the 16-byte boundaries the instructions bound both directions: rows are turned in shared memory and 16-bit values move two at a time
// (8192 x 4095 BF16 back 24 us, 1.9 times the time its bytes need, 16384 x 8191 BF16 79 us, 1.5 times; 75 % of the issue slots).
#include <cuda_runtime.h>

#include <type_traits>

#include "element.cuh"
#include "mx_encode.cuh"
#include "mx_format.cuh"
#include "omc_internal.h"

namespace {

using namespace omc;
using el::Word;
using mx::encode_block;
using mx::fp32_bits;
using mx::load;
using mx::max_magnitude;

constexpr int WARPS = 8;

// The scales of the four blocks that 128 / E lanes hold, one byte each.
template <int E>
__device__ __forceinline__ uint32_t gather_scales(uint32_t scale, int lane)
{
    constexpr int LANES = 32 / E;                        // of one block
    uint32_t w = scale << (8 * ((lane / LANES) & 3));
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, LANES);
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2 * LANES);
    return w;
}

// A CTA of the row kernels takes a strip of columns, 32 bytes of values a lane (blockIdx.x), of eight rows at a time, a row a
// warp, and walks down the matrix: from row to row a warp's addresses move by constants.  It asks for the next AHEAD
// rows' pieces while it works on one.
template <bool VECTOR> constexpr int AHEAD = VECTOR ? 3 : 2;                   // (with three, turned rows spill: 16384 x 8191 BF16 100 us, with two 79)
template <typename T> constexpr int LANE_VALUES = 32 / (int)sizeof(T);         // 8 or 16
template <typename T> constexpr uint32_t STRIP = 32 * LANE_VALUES<T>;          // columns: 256 or 512
// CTAs on an SM, as the registers of the pieces on their way allow.
constexpr int ROWS_CTAS = 4;

// Row r's place in the scales of a K step (256 columns): bytes from the place of row 0.
__device__ __forceinline__ uint64_t row_offset(uint32_t r, uint32_t ksteps)
{
    return (uint64_t)(r >> 7) * ksteps * 1024 + ((r & 31) * 16 + ((r >> 5) & 3) * 4);
}

// Rows off the 16-byte boundaries: a strip's words come in from boundary to boundary, neighbouring lanes neighbouring words,
// and are turned in shared memory.  Value e of the strip has place odd + e, odd = 1 where a 16-bit strip begins
// in the upper half of a word; word j of a lane holds the places of word 32 j + lane.  The halves of a word that is
// only partly inside are fetched alone (lane 0 the first, lane 1 the last): nothing outside the row is read.
template <typename T>
struct Turned {
    static constexpr int PLACES = 4 / (int)sizeof(T);      // of a word
    uint32_t w[8], edge;

    static __device__ __forceinline__ uint32_t odd(const T *row) { return PLACES == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(row) >> 1) & 1u : 0u; }
    __device__ __forceinline__ void load(const T *row, uint32_t n, int lane)
    {
        const uint32_t o = odd(row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t p = (32 * j + lane) * PLACES;
            w[j] = p >= o && p + PLACES <= o + n ? *reinterpret_cast<const uint32_t *>(row + p - o) : 0u;
        }
        if constexpr (PLACES == 2) {
            edge = 0u;
            if (lane == 0 && o) edge = *reinterpret_cast<const uint16_t *>(row);
            if (lane == 1 && ((o + n) & 1) && (n > 1 || !o)) edge = *reinterpret_cast<const uint16_t *>(row + n - 1);
        }
    }
    // This lane's E values; room: 260 words of this warp.
    __device__ __forceinline__ void turn(uint32_t *room, uint32_t o, uint32_t n, int lane, uint32_t *v) const
    {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) room[32 * j + lane] = w[j];
        if constexpr (PLACES == 2) {
            if (lane == 2) room[256] = 0u;
            __syncwarp();
            uint16_t *half = reinterpret_cast<uint16_t *>(room);
            if (lane == 0 && o) half[1] = (uint16_t)edge;
            if (lane == 1 && ((o + n) & 1) && (n > 1 || !o)) half[o + n - 1] = (uint16_t)edge;
        }
        __syncwarp();
        const uint4 a = *reinterpret_cast<const uint4 *>(room + lane * 8), b = *reinterpret_cast<const uint4 *>(room + lane * 8 + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        if (o) {
            const uint32_t last = room[lane * 8 + 8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __byte_perm(v[j], j < 7 ? v[j < 7 ? j + 1 : 7] : last, 0x5432);
        }
    }
};

// Along the rows only.
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(32 * WARPS, ROWS_CTAS)
quantise_rows_kernel(const T *x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *__restrict__ codes,
                     uint8_t *__restrict__ scales)
{
    constexpr int E = LANE_VALUES<T>;
    __shared__ __align__(16) uint32_t room[VECTOR ? 1 : WARPS][VECTOR ? 4 : 260];
    const uint32_t ksteps = (cols + 255) / 256;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t rb = mx::row_bytes(cols);
    const uint32_t step = gridDim.y * WARPS, col = blockIdx.x * STRIP<T> + lane * E;
    uint32_t row = blockIdx.y * WARPS + warp, coming = row;
    const T *src = x + coming * ld + blockIdx.x * STRIP<T>, *now = src;        // the strip's first column
    const uint32_t n = min(STRIP<T>, cols - blockIdx.x * STRIP<T>);
    uint8_t *dst = codes + row * rb + col / 2;
    const uint64_t src_step = step * ld, dst_step = step * rb;
    // the lane that stores the scales of four blocks (128 columns), and where
    const uint32_t block = col / 32;
    const bool inside = col / 2 < rb, stores = lane % (128 / E) == 0 && block / 8 < ksteps;
    uint8_t *const strip = scales + (uint64_t)(block / 8) * 1024 + (block / 4 & 1) * 512;
    el::enter_stream_order();
    uint32_t w[VECTOR ? AHEAD<VECTOR> : 1][8];
    Turned<T> t[VECTOR ? 1 : AHEAD<VECTOR>];
    auto fetch = [&](int i) {
        if (coming < rows) {
            if constexpr (VECTOR) load<T, true, E>(src, lane * E, n, w[i]);
            else t[i].load(src, n, lane);
        }
        coming += step;
        src += src_step;
    };
#pragma unroll
    for (int i = 0; i < AHEAD<VECTOR>; ++i) fetch(i);
    while (row < rows) {
#pragma unroll
        for (int i = 0; i < AHEAD<VECTOR>; ++i) {
            if (row >= rows) break;
            uint32_t scale, c[E / 8];
            if constexpr (!VECTOR) {
                t[i].turn(room[warp], Turned<T>::odd(now), n, lane, w[0]);
                now += src_step;
            }
            encode_block<T, E>(w[VECTOR ? i : 0], c, scale);
            fetch(i);
            if constexpr (E == 16) {
                if (inside) *reinterpret_cast<uint2 *>(dst) = make_uint2(c[0], c[1]);
            } else {
                if (inside) *reinterpret_cast<uint32_t *>(dst) = c[0];
            }
            const uint32_t s = gather_scales<E>(scale, lane);
            if (stores) *reinterpret_cast<uint32_t *>(strip + row_offset(row, ksteps)) = s;
            row += step;
            dst += dst_step;
        }
    }
}

// Along the columns, and along the rows too if ROWS: a CTA takes a tile of 128 x 128.
constexpr int TILE = 128;
template <typename T> constexpr int tile_smem() { return TILE * TILE * (int)sizeof(T) + TILE * 64 + 2 * 512; }

// Orders in shared memory without bank conflicts.  The tile: a lane brings 32 bytes of a row, whose first halves are
// stored side by side, then the second halves; place p of a row holds column tile_column(p).
template <typename T>
__device__ __forceinline__ uint32_t tile_column(uint32_t place)
{
    constexpr uint32_t H = LANE_VALUES<T> / 2;           // values of a half
    return (place % 64) / H * (2 * H) + place / 64 * H + place % H;
}
// The codes of the columns, 64 bytes each in four chunks of 16: the chunk's place.
template <typename T>
__device__ __forceinline__ uint32_t code_place(uint32_t col, uint32_t chunk)
{
    const uint32_t turn = sizeof(T) == 2 ? (col >> 2 & 1) | (col >> 3 & 2) : col >> 3 & 3;
    return (col ^ (col >> 1 & 1)) * 64 + (chunk ^ turn) * 16;
}

template <typename T, bool VECTOR, bool ROWS>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 3 : 4)
quantise_tile_kernel(const T *x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *__restrict__ codes,
                     uint8_t *__restrict__ scales, uint8_t *__restrict__ codes_t, uint8_t *__restrict__ scales_t)
{
    extern __shared__ __align__(16) uint8_t smem[];
    T *tile = reinterpret_cast<T *>(smem);
    uint8_t *out = smem + TILE * TILE * sizeof(T);
    uint8_t *atom = out + TILE * 64, *atom_t = atom + 512;
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t col_tiles = (cols + TILE - 1) / TILE, row_tiles = (rows + TILE - 1) / TILE;
    const uint32_t tr = blockIdx.x / col_tiles, tc = blockIdx.x - tr * col_tiles;
    const uint32_t r0 = tr * TILE, c0 = tc * TILE;
    const uint64_t rb = mx::row_bytes(cols), rb_t = mx::row_bytes(rows);
    el::enter_stream_order();

    // 8 or 16 lanes take 128 columns of a row, 32 bytes a lane
    constexpr int E = LANE_VALUES<T>, LANES = TILE / E, STEP = 256 / LANES, BATCH = 4;
    const uint32_t lane_col = (tid % LANES) * E, col = c0 + lane_col;
    auto put_row = [&](uint32_t r, const uint32_t *w) {      // codes and scales along row r of the tile
        uint32_t scale, c[E / 8];
        encode_block<T, E>(w, c, scale);
        if (r0 + r < rows && col / 2 < rb) {
            uint8_t *to = codes + (r0 + r) * rb + col / 2;
            if constexpr (E == 16) *reinterpret_cast<uint2 *>(to) = make_uint2(c[0], c[1]);
            else *reinterpret_cast<uint32_t *>(to) = c[0];
        }
        const uint32_t s = gather_scales<E>(scale, lane);
        if (tid % LANES == 0) *reinterpret_cast<uint32_t *>(atom + (r & 31) * 16 + (r >> 5) * 4) = s;
    };
    if constexpr (VECTOR) {
        // four rows are asked for at a time, and encoded along the rows on their way to shared memory
#pragma unroll
        for (int i0 = 0; i0 < TILE / STEP; i0 += BATCH) {
            uint32_t w[BATCH][8];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const uint32_t r = r0 + (i0 + i) * STEP + tid / LANES;
                if (r < rows) {
                    load<T, true, E>(x + (uint64_t)r * ld, col, cols, w[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[i][j] = 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const uint32_t r = (i0 + i) * STEP + tid / LANES;
                T *dst = tile + r * TILE + lane_col / 2;
                *reinterpret_cast<uint4 *>(dst) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
                *reinterpret_cast<uint4 *>(dst + TILE / 2) = make_uint4(w[i][4], w[i][5], w[i][6], w[i][7]);
                if constexpr (ROWS) put_row(r, w[i]);
            }
        }
    } else {
        // off the 16-byte boundaries neighbouring lanes take neighbouring values, a column a thread
        const uint32_t c = tid % TILE, half = LANE_VALUES<T> / 2, place = c / (2 * half) * half + c % half + (c / half & 1) * (TILE / 2);
        const T *src = x + (uint64_t)(r0 + tid / TILE) * ld + c0 + c;
#pragma unroll 16
        for (uint32_t r = tid / TILE; r < TILE; r += 2, src += 2 * ld)
            tile[r * TILE + place] = r0 + r < rows && c0 + c < cols ? *src : el::from_float<T>(0.f);
        if constexpr (ROWS) {
            __syncthreads();
#pragma unroll 2
            for (int i = 0; i < TILE / STEP; ++i) {
                const uint32_t r = i * STEP + tid / LANES;
                const T *row = tile + r * TILE + lane_col / 2;
                const uint4 a = *reinterpret_cast<const uint4 *>(row), b = *reinterpret_cast<const uint4 *>(row + TILE / 2);
                const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                put_row(r, w);
            }
        }
    }
    __syncthreads();

    // a thread takes one block of 32 rows of two neighbouring columns
    {
        const int block = tid >> 6, pair = tid & 63;
        using Pair = typename std::conditional<sizeof(T) == 4, float2, uint32_t>::type;      // two columns of a row as they are stored
        Pair p[32];
        uint32_t top_a = 0, top_b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            p[i] = *reinterpret_cast<const Pair *>(tile + (block * 32 + i) * TILE + pair * 2);
            if constexpr (sizeof(T) == 4) {
                top_a = max_magnitude<T>(top_a, __float_as_uint(p[i].x));
                top_b = max_magnitude<T>(top_b, __float_as_uint(p[i].y));
            } else {
                top_a = max_magnitude<T>(top_a, p[i]);
            }
        }
        if constexpr (sizeof(T) == 2) {
            top_b = top_a >> 16;
            top_a &= 0xFFFFu;
        }
        const uint32_t sa = mx::scale_of(fp32_bits<T>(top_a)), sb = mx::scale_of(fp32_bits<T>(top_b));
        const float2 f = make_float2(mx::inverse_scale(sa), mx::inverse_scale(sb));
        uint32_t ca[4], cb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float u[8], w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float2 v;
                if constexpr (sizeof(T) == 4) v = p[8 * i + j];
                else Word<T>::unpack(p[8 * i + j], reinterpret_cast<float *>(&v));
                v = el::mul2(v, f);
                u[j] = v.x;
                w[j] = v.y;
            }
            ca[i] = sa == mx::NAN_SCALE ? 0u : mx::encode8(u);
            cb[i] = sb == mx::NAN_SCALE ? 0u : mx::encode8(w);
        }
        const uint32_t col = tile_column<T>(pair * 2);
        *reinterpret_cast<uint4 *>(out + code_place<T>(col, block)) = make_uint4(ca[0], ca[1], ca[2], ca[3]);
        *reinterpret_cast<uint4 *>(out + code_place<T>(col + 1, block)) = make_uint4(cb[0], cb[1], cb[2], cb[3]);
        uint8_t *scale = atom_t + (col & 31) * 16 + (col >> 5) * 4 + block;      // (an even column: its neighbour is 16 bytes on)
        scale[0] = (uint8_t)sa;
        scale[16] = (uint8_t)sb;
    }
    __syncthreads();

#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t col = i * 64 + (tid >> 2), chunk = tid & 3;
        const uint64_t at = r0 / 2 + chunk * 16;
        if (c0 + col < cols && at < rb_t)
            *reinterpret_cast<uint4 *>(codes_t + (c0 + col) * rb_t + at) = *reinterpret_cast<const uint4 *>(out + code_place<T>(col, chunk));
    }
    // 512 bytes of scales per direction; behind the last odd one its partner's zeros
    if (tid < 128) {
        uint8_t *dst = scales_t + ((uint64_t)tc * ((rows + 255) / 256) + tr / 2) * 1024 + (tr & 1) * 512;
        reinterpret_cast<uint32_t *>(dst)[tid] = reinterpret_cast<const uint32_t *>(atom_t)[tid];
        if (tr + 1 == row_tiles && !(tr & 1)) reinterpret_cast<uint32_t *>(dst)[128 + tid] = 0u;
    } else if (ROWS) {
        const int t = tid - 128;
        uint8_t *dst = scales + ((uint64_t)tr * ((cols + 255) / 256) + tc / 2) * 1024 + (tc & 1) * 512;
        reinterpret_cast<uint32_t *>(dst)[t] = reinterpret_cast<const uint32_t *>(atom)[t];
        if (tc + 1 == col_tiles && !(tc & 1)) reinterpret_cast<uint32_t *>(dst)[128 + t] = 0u;
    }
}

// A warp takes a strip of a row, 32 bytes of values a lane, stored at once: two 16-byte stores would write every 32-byte
// sector in two halves (8192 x 2048 FP32 17 us instead of 11).  Rows off the 16-byte boundaries, 256 columns at a time, are
// turned in shared memory, so that neighbouring lanes store neighbouring values (16-bit types in pairs that lie on 4-byte boundaries).
template <typename T, bool VECTOR> constexpr uint32_t VALUES_STRIP = VECTOR ? STRIP<T> : 256;

template <typename T, bool VECTOR>
__global__ void __launch_bounds__(32 * WARPS)
dequantise_kernel(const uint8_t *codes, const uint8_t *scales, uint32_t rows, uint32_t cols,
                  T *__restrict__ out, uint64_t ld)
{
    constexpr int N = Word<T>::N, E = VALUES_STRIP<T, VECTOR> / 32;
    __shared__ __align__(16) T turned[VECTOR ? 1 : WARPS][VECTOR ? 8 : 256 + 8];
    const uint32_t ksteps = (cols + 255) / 256;
    const int lane = threadIdx.x & 31;
    const uint64_t rb = mx::row_bytes(cols);
    const uint32_t col = blockIdx.x * VALUES_STRIP<T, VECTOR> + lane * E;
    el::enter_stream_order();
    for (uint32_t row = blockIdx.y * WARPS + (threadIdx.x >> 5); row < rows; row += gridDim.y * WARPS) {
        float v[E];
        if (col < cols) {
            const uint8_t *src = codes + row * rb + col / 2;
            const float2 s = el::twice(mx::scale_value(scales[mx::scale_offset(row, col / 32, ksteps)]));
            if constexpr (E == 16) {
                const uint2 c = *reinterpret_cast<const uint2 *>(src);
                mx::decode8(c.x, v);
                mx::decode8(c.y, v + 8);
            } else {
                mx::decode8(*reinterpret_cast<const uint32_t *>(src), v);
            }
#pragma unroll
            for (int j = 0; j < E / 2; ++j) reinterpret_cast<float2 *>(v)[j] = el::mul2(reinterpret_cast<float2 *>(v)[j], s);
        }
        T *to = out + row * ld + blockIdx.x * VALUES_STRIP<T, VECTOR>;
        if constexpr (VECTOR) {
            T *dst = to + lane * E;
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = Word<T>::pack(v + N * j);
            if (col + E <= cols && (reinterpret_cast<uintptr_t>(dst) & 31u) == 0) {
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                             ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
            } else if (col + E <= cols) {
                *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(dst + E / 2) = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (col + j < cols) dst[j] = el::from_float<T>(v[j]);
            }
        } else {
            T *mine = turned[threadIdx.x >> 5];
            const uint32_t n = min(256u, cols - blockIdx.x * 256);
            const uint32_t odd = sizeof(T) == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(to) >> 1) & 1u : 0u;      // values before the first boundary
            // value e goes to place odd + e: with odd = 1 a lane's words are its own moved by a half, led by its neighbour's last value
            uint32_t w[8 / N];
#pragma unroll
            for (int j = 0; j < 8 / N; ++j) w[j] = Word<T>::pack(v + N * j);
            __syncwarp();
            if constexpr (sizeof(T) == 2) {
                const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, w[3], 1);
                if (odd) {
                    if (lane == 31) mine[256] = el::from_float<T>(v[7]);
                    w[3] = __byte_perm(w[2], w[3], 0x5432);
                    w[2] = __byte_perm(w[1], w[2], 0x5432);
                    w[1] = __byte_perm(w[0], w[1], 0x5432);
                    w[0] = __byte_perm(before, w[0], 0x5432);
                }
            }
#pragma unroll
            for (int j = 0; j < 8 / N; j += 4) *reinterpret_cast<uint4 *>(mine + lane * 8 + j * N) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
            __syncwarp();
            if constexpr (sizeof(T) == 2) {
                // pair p: places 2 p and 2 p + 1, values 2 p - odd and 2 p + 1 - odd
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t e = 2 * (j * 32 + lane);
                    if (e >= odd && e + 1 < odd + n)
                        *reinterpret_cast<uint32_t *>(to + e - odd) = *reinterpret_cast<const uint32_t *>(mine + e);
                }
                // what has no partner: the first value before a boundary, the last one behind
                if (lane == 0 && odd) to[0] = mine[1];
                if (lane == 1 && ((odd + n) & 1) && (n > 1 || !odd)) to[n - 1] = mine[odd + n - 1];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j * 32 + lane < n) to[j * 32 + lane] = mine[j * 32 + lane];
            }
        }
    }
}

// As many CTAs to a strip of columns as are resident at once, or, with so many strips that this would come out
// uneven, about four times as many as are resident.
dim3 strips(uint32_t rows, uint32_t cols, uint32_t strip, int per_sm)
{
    const uint32_t resident = per_sm * el::sm_count(), across = (cols + strip - 1) / strip, groups = (rows + WARPS - 1) / WARPS;
    uint32_t down = resident / across;
    if (down < 4) down = (4 * resident + across - 1) / across;
    return dim3(across, groups < down ? groups : down);
}

template <typename T, bool VECTOR>
int quantise(const void *x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
             uint8_t *scales_t, void *stream)
{
    const T *src = static_cast<const T *>(x);
    if (!codes_t) {
        return note_cuda(el::launch(quantise_rows_kernel<T, VECTOR>, strips(rows, cols, STRIP<T>, ROWS_CTAS), 32 * WARPS, 0, 1,
                                    stream, src, rows, cols, ld, codes, scales));
    }
    auto kernel = codes ? quantise_tile_kernel<T, VECTOR, true> : quantise_tile_kernel<T, VECTOR, false>;
    const int rc = codes ? el::allow_smem<quantise_tile_kernel<T, VECTOR, true>>(tile_smem<T>())
                         : el::allow_smem<quantise_tile_kernel<T, VECTOR, false>>(tile_smem<T>());
    if (rc) return rc;
    const uint64_t tiles = (uint64_t)((rows + TILE - 1) / TILE) * ((cols + TILE - 1) / TILE);
    return note_cuda(el::launch(kernel, dim3((uint32_t)tiles), 256, tile_smem<T>(), 1, stream, src, rows, cols, ld, codes, scales,
                                codes_t, scales_t));
}

template <typename T, bool VECTOR>
int dequantise(const uint8_t *codes, const uint8_t *scales, uint32_t rows, uint32_t cols, void *out, uint64_t ld, void *stream)
{
    const uint32_t groups = (rows + WARPS - 1) / WARPS;
    return note_cuda(el::launch(dequantise_kernel<T, VECTOR>, dim3((cols + VALUES_STRIP<T, VECTOR> - 1) / VALUES_STRIP<T, VECTOR>, groups < 65535 ? groups : 65535), 32 * WARPS, 0, 1, stream,
                                codes, scales, rows, cols, static_cast<T *>(out), ld));
}

bool vector_rows(const void *p, uint64_t ld, int type) { return el::aligned16(p) && ld * el::size_of(type) % 16 == 0; }

}  // namespace

namespace omc {
// A shape the kernels' 32-bit indices cover (more than the device's memory holds otherwise).
bool mx_shape_ok(uint64_t rows, uint64_t cols)
{
    return rows >= 1 && cols >= 1 && rows < (1ull << 31) && cols < (1ull << 31) &&
           rows * ((cols + 255) / 256) < (1ull << 32) && cols * ((rows + 255) / 256) < (1ull << 32);
}
}  // namespace omc

extern "C" int omc_mx_sizes(uint64_t rows, uint64_t cols, uint64_t *codes_bytes, uint64_t *scales_bytes)
{
    if (!mx_shape_ok(rows, cols)) return OMC_ERR_INVALID_ARG;
    if (codes_bytes) *codes_bytes = mx::codes_bytes(rows, cols);
    if (scales_bytes) *scales_bytes = mx::scales_bytes(rows, cols);
    return OMC_OK;
}

extern "C" int omc_mx_quantise(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ld, uint8_t *codes, uint8_t *scales,
                               uint8_t *codes_t, uint8_t *scales_t, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!x || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return OMC_ERR_NULL_PTR;
    if (!mx_shape_ok(rows, cols) || ld < cols) return OMC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x) % el::size_of(type) || !el::aligned16(codes) || !el::aligned16(scales) ||
        !el::aligned16(codes_t) || !el::aligned16(scales_t))
        return OMC_ERR_MISALIGNED;
    const bool vec = vector_rows(x, ld, type);
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
#define OMC_CALL(T) (vec ? quantise<T, true>(x, r, c, ld, codes, scales, codes_t, scales_t, stream) \
                         : quantise<T, false>(x, r, c, ld, codes, scales, codes_t, scales_t, stream))
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}

extern "C" int omc_mx_dequantise(const uint8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t cols, void *out, int type,
                                 uint64_t ld, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!codes || !scales || !out) return OMC_ERR_NULL_PTR;
    if (!mx_shape_ok(rows, cols) || ld < cols) return OMC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(out) % el::size_of(type) || !el::aligned16(codes) || !el::aligned16(scales)) return OMC_ERR_MISALIGNED;
    const bool vec = vector_rows(out, ld, type);
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
#define OMC_CALL(T) (vec ? dequantise<T, true>(codes, scales, r, c, out, ld, stream) : dequantise<T, false>(codes, scales, r, c, out, ld, stream))
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}
