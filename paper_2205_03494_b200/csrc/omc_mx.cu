// omc_mx_quantise / omc_mx_dequantise: the 4-bit microscaled format (mx_format.cuh).
//
// Both directions read the values once.  Along the rows eight values sit in a lane and a block of 32 in four
// lanes, so that the largest magnitude takes two shuffles; along the columns a tile of 128 x 128 goes through
// shared memory and a thread holds whole blocks.  The scale is a power of two, so that scaling is exact and
// the only rounding is the conversion to E2M1.
#include <cuda_runtime.h>

#include "element.cuh"
#include "mx_format.cuh"
#include "omc_internal.h"

namespace {

using namespace omc;
using el::Word;

constexpr int WARPS = 8;

// Eight consecutive values as they are stored: four words of 16-bit types, eight of FP32.
template <typename T> constexpr int WORDS8 = 8 / Word<T>::N;

template <typename T, bool VECTOR>
__device__ __forceinline__ void load8(const T *row, uint32_t col, uint32_t cols, uint32_t *w)
{
    if (VECTOR && col + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < WORDS8<T>; i += 4) {
            const uint4 q = *reinterpret_cast<const uint4 *>(row + col + i * Word<T>::N);
            w[i] = q.x;
            w[i + 1] = q.y;
            w[i + 2] = q.z;
            w[i + 3] = q.w;
        }
    } else {                       // zeros behind the row's end
#pragma unroll
        for (int i = 0; i < WORDS8<T>; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = col + i < cols ? reinterpret_cast<const uint32_t *>(row)[col + i] : 0u;
            } else {
                const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + col + 2 * i;
                const uint32_t lo = col + 2 * i < cols ? p[0] : 0u, hi = col + 2 * i + 1 < cols ? p[1] : 0u;
                w[i] = lo | (hi << 16);
            }
        }
    }
}

// Largest magnitude, two 16-bit values at a time: the order of the magnitudes is that of their bit patterns, Inf and
// NaN on top.
template <typename T>
__device__ __forceinline__ uint32_t max_magnitude(uint32_t acc, uint32_t w)
{
    if constexpr (sizeof(T) == 4) return max(acc, w & 0x7FFFFFFFu);
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(acc), "r"(w & 0x7FFF7FFFu));
    return r;
}
// A magnitude of T as FP32 bits (T 16 bits wide: the lower half of m).
template <typename T>
__device__ __forceinline__ uint32_t fp32_bits(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return m;
    float f[2];
    Word<T>::unpack(m, f);
    return __float_as_uint(f[0]);
}

// Codes and scale of the block that four neighbouring lanes hold, eight values each.
template <typename T>
__device__ __forceinline__ uint32_t encode_block(const uint32_t *w, uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < WORDS8<T>; ++i) top = max_magnitude<T>(top, w[i]);
    if constexpr (sizeof(T) == 2) top = max(top >> 16, top & 0xFFFFu);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    scale = mx::scale_of(fp32_bits<T>(top));
    const float2 f = el::twice(mx::inverse_scale(scale));
    float v[8];
#pragma unroll
    for (int i = 0; i < WORDS8<T>; ++i) Word<T>::unpack(w[i], v + Word<T>::N * i);
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float2 *>(v)[i] = el::mul2(reinterpret_cast<float2 *>(v)[i], f);
    const uint32_t codes = mx::encode8(v);
    return scale == mx::NAN_SCALE ? 0u : codes;
}
// The scales of the four blocks that sixteen lanes hold, one byte each.
__device__ __forceinline__ uint32_t gather_scales(uint32_t scale, int lane)
{
    uint32_t w = scale << (8 * ((lane >> 2) & 3));
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, 8);
    return w;
}

// The pieces of a matrix (256 columns of a row) that a warp takes: every `stride`-th, counted along the rows, without a
// division per piece.
struct Walk {
    uint32_t row, k, step_rows, step_k, ksteps;

    __device__ __forceinline__ Walk(uint32_t first, uint32_t stride, uint32_t ksteps_)
        : row(first / ksteps_), k(first % ksteps_), step_rows(stride / ksteps_), step_k(stride % ksteps_), ksteps(ksteps_) {}
    __device__ __forceinline__ void next()
    {
        row += step_rows;
        k += step_k;
        if (k >= ksteps) {
            k -= ksteps;
            ++row;
        }
    }
};

// Along the rows only: a warp walks over pieces and asks for the next AHEAD while it works on one.
constexpr int AHEAD = 4;

template <typename T, bool VECTOR>
__global__ void __launch_bounds__(32 * WARPS)
quantise_rows_kernel(const T *__restrict__ x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *__restrict__ codes,
                     uint8_t *__restrict__ scales)
{
    const uint32_t ksteps = (cols + 255) / 256;
    const int lane = threadIdx.x & 31;
    const uint64_t rb = mx::row_bytes(cols);
    Walk at(blockIdx.x * WARPS + (threadIdx.x >> 5), gridDim.x * WARPS, ksteps), ask = at;
    el::enter_stream_order();
    uint32_t w[AHEAD][WORDS8<T>];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i, ask.next())
        if (ask.row < rows) load8<T, VECTOR>(x + ask.row * ld, ask.k * 256 + lane * 8, cols, w[i]);
    while (at.row < rows) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (at.row >= rows) break;
            const uint32_t col = at.k * 256 + lane * 8;
            uint32_t scale;
            const uint32_t c = encode_block<T>(w[i], scale);
            if (ask.row < rows) load8<T, VECTOR>(x + ask.row * ld, ask.k * 256 + lane * 8, cols, w[i]);
            if (col / 2 < rb) *reinterpret_cast<uint32_t *>(codes + at.row * rb + col / 2) = c;
            const uint32_t s = gather_scales(scale, lane);
            if ((lane & 15) == 0)
                *reinterpret_cast<uint32_t *>(scales + mx::scale_offset(at.row, (uint64_t)at.k * 8 + (lane >> 2), ksteps)) = s;
            at.next();
            ask.next();
        }
    }
}

// Along the columns, and along the rows too if ROWS: a CTA takes a tile of 128 x 128.
constexpr int TILE = 128, COLUMN_PITCH = 80;      // bytes between the staged code columns (64 and a skew against bank conflicts)
template <typename T> constexpr int tile_smem() { return TILE * TILE * (int)sizeof(T) + TILE * COLUMN_PITCH + 2 * 512; }

template <typename T, bool VECTOR, bool ROWS>
__global__ void __launch_bounds__(256)
quantise_tile_kernel(const T *__restrict__ x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *__restrict__ codes,
                     uint8_t *__restrict__ scales, uint8_t *__restrict__ codes_t, uint8_t *__restrict__ scales_t)
{
    extern __shared__ __align__(16) uint8_t smem[];
    T *tile = reinterpret_cast<T *>(smem);
    uint8_t *out = smem + TILE * TILE * sizeof(T);
    uint8_t *atom = out + TILE * COLUMN_PITCH, *atom_t = atom + 512;
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t col_tiles = (cols + TILE - 1) / TILE, row_tiles = (rows + TILE - 1) / TILE;
    const uint32_t tr = blockIdx.x / col_tiles, tc = blockIdx.x - tr * col_tiles;
    const uint32_t r0 = tr * TILE, c0 = tc * TILE;
    const uint64_t rb = mx::row_bytes(cols), rb_t = mx::row_bytes(rows);
    el::enter_stream_order();

    // sixteen lanes take 128 columns of a row; four rows are asked for at a time
    constexpr int BATCH = sizeof(T) == 4 ? 4 : 8;
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += BATCH) {
        uint32_t w[BATCH][WORDS8<T>];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const uint32_t r = r0 + (i0 + i) * 16 + (tid >> 4);
            if (r < rows) {
                load8<T, VECTOR>(x + (uint64_t)r * ld, c0 + (tid & 15) * 8, cols, w[i]);
            } else {
#pragma unroll
                for (int j = 0; j < WORDS8<T>; ++j) w[i][j] = 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const uint32_t r = (i0 + i) * 16 + (tid >> 4), col = c0 + (tid & 15) * 8;
            uint4 *dst = reinterpret_cast<uint4 *>(tile + r * TILE + (tid & 15) * 8);
#pragma unroll
            for (int j = 0; j < WORDS8<T> / 4; ++j) dst[j] = make_uint4(w[i][4 * j], w[i][4 * j + 1], w[i][4 * j + 2], w[i][4 * j + 3]);
            if constexpr (ROWS) {
                uint32_t scale;
                const uint32_t c = encode_block<T>(w[i], scale);
                if (r0 + r < rows && col / 2 < rb) *reinterpret_cast<uint32_t *>(codes + (r0 + r) * rb + col / 2) = c;
                const uint32_t s = gather_scales(scale, lane);
                if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(atom + (r & 31) * 16 + (r >> 5) * 4) = s;
            }
        }
    }
    __syncthreads();

    // a thread takes one block of 32 rows of two neighbouring columns
    {
        const int block = tid >> 6, pair = tid & 63;
        float2 v[32];
        uint32_t top_a = 0, top_b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const T *p = tile + (block * 32 + i) * TILE + pair * 2;
            if constexpr (sizeof(T) == 4) {
                v[i] = *reinterpret_cast<const float2 *>(p);
                top_a = max_magnitude<T>(top_a, __float_as_uint(v[i].x));
                top_b = max_magnitude<T>(top_b, __float_as_uint(v[i].y));
            } else {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
                top_a = max_magnitude<T>(top_a, w);
                Word<T>::unpack(w, reinterpret_cast<float *>(v + i));
            }
        }
        if constexpr (sizeof(T) == 2) {
            top_b = top_a >> 16;
            top_a &= 0xFFFFu;
        }
        const uint32_t sa = mx::scale_of(fp32_bits<T>(top_a)), sb = mx::scale_of(fp32_bits<T>(top_b));
        const float2 f = make_float2(mx::inverse_scale(sa), mx::inverse_scale(sb));
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = el::mul2(v[i], f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float u[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = h ? v[8 * i + j].y : v[8 * i + j].x;
                c[i] = (h ? sb : sa) == mx::NAN_SCALE ? 0u : mx::encode8(u);
            }
            const int col = pair * 2 + h;
            *reinterpret_cast<uint4 *>(out + col * COLUMN_PITCH + block * 16) = make_uint4(c[0], c[1], c[2], c[3]);
            atom_t[(col & 31) * 16 + (col >> 5) * 4 + block] = (uint8_t)(h ? sb : sa);
        }
    }
    __syncthreads();

#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t col = i * 64 + (tid >> 2), chunk = tid & 3;
        const uint64_t at = r0 / 2 + chunk * 16;
        if (c0 + col < cols && at < rb_t)
            *reinterpret_cast<uint4 *>(codes_t + (c0 + col) * rb_t + at) = *reinterpret_cast<const uint4 *>(out + col * COLUMN_PITCH + chunk * 16);
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

// A warp walks over pieces.  Rows off the 16-byte boundaries are turned in shared memory, so that neighbouring lanes store
// neighbouring values (16-bit types in pairs that lie on 4-byte boundaries).
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(32 * WARPS)
dequantise_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t rows, uint32_t cols,
                  T *__restrict__ out, uint64_t ld)
{
    __shared__ __align__(16) T turned[VECTOR ? 1 : WARPS][VECTOR ? 8 : 256 + 8];
    const uint32_t ksteps = (cols + 255) / 256;
    const int lane = threadIdx.x & 31;
    const uint64_t rb = mx::row_bytes(cols);
    Walk at(blockIdx.x * WARPS + (threadIdx.x >> 5), gridDim.x * WARPS, ksteps), ask = at;
    el::enter_stream_order();
    uint32_t c[AHEAD], b[AHEAD];
    auto fetch = [&](int i) {
        const uint32_t col = ask.k * 256 + lane * 8;
        if (ask.row < rows && col < cols) {
            c[i] = *reinterpret_cast<const uint32_t *>(codes + ask.row * rb + col / 2);
            b[i] = scales[mx::scale_offset(ask.row, (uint64_t)ask.k * 8 + (lane >> 2), ksteps)];
        }
        ask.next();
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i);
    while (at.row < rows) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (at.row >= rows) break;
            const uint32_t col = at.k * 256 + lane * 8;
            float v[8];
            mx::decode8(c[i], v);
            const float2 s = el::twice(mx::scale_value(b[i] & 255u));
            fetch(i);
            uint32_t w[WORDS8<T>];
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<float2 *>(v)[j] = el::mul2(reinterpret_cast<float2 *>(v)[j], s);
#pragma unroll
            for (int j = 0; j < WORDS8<T>; ++j) w[j] = Word<T>::pack(v + Word<T>::N * j);
            if (VECTOR) {
                T *dst = out + at.row * ld + col;
                if (col + 8 <= cols) {
#pragma unroll
                    for (int j = 0; j < WORDS8<T>; j += 4) *reinterpret_cast<uint4 *>(dst + j * Word<T>::N) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (col + j < cols) dst[j] = el::from_float<T>(v[j]);
                }
            } else {
                T *mine = turned[threadIdx.x >> 5];
                T *dst = out + at.row * ld + at.k * 256;
                const uint32_t n = min(256u, cols - at.k * 256);
                const uint32_t odd = sizeof(T) == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(dst) >> 1) & 1u : 0u;      // values before the first boundary
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) mine[odd + lane * 8 + j] = el::from_float<T>(v[j]);      // value e at odd + e
                __syncwarp();
                if constexpr (sizeof(T) == 2) {
                    // pair p: places 2 p and 2 p + 1, values 2 p - odd and 2 p + 1 - odd
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t e = 2 * (j * 32 + lane);
                        if (e >= odd && e + 1 < odd + n)
                            *reinterpret_cast<uint32_t *>(dst + e - odd) = *reinterpret_cast<const uint32_t *>(mine + e);
                    }
                    // what has no partner: the first value before a boundary, the last one behind
                    if (lane == 0 && odd) dst[0] = mine[1];
                    if (lane == 1 && ((odd + n) & 1) && (n > 1 || !odd)) dst[n - 1] = mine[odd + n - 1];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j * 32 + lane < n) dst[j * 32 + lane] = mine[j * 32 + lane];
                }
            }
            at.next();
        }
    }
}

// CTAs for a walk over so many pieces: what is resident (eight CTAs on an SM), or one piece a warp.
uint32_t walk_ctas(uint64_t pieces)
{
    const uint64_t most = 8ull * DEFAULT_SMS, wanted = (pieces + WARPS - 1) / WARPS;
    return (uint32_t)(wanted < most ? wanted : most);
}

template <typename T, bool VECTOR>
int quantise(const void *x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
             uint8_t *scales_t, void *stream)
{
    const T *src = static_cast<const T *>(x);
    if (!codes_t) {
        return note_cuda(el::launch(quantise_rows_kernel<T, VECTOR>, dim3(walk_ctas((uint64_t)rows * ((cols + 255) / 256))), 32 * WARPS, 0, 1,
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
    return note_cuda(el::launch(dequantise_kernel<T, VECTOR>, dim3(walk_ctas((uint64_t)rows * ((cols + 255) / 256))), 32 * WARPS, 0, 1, stream,
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
