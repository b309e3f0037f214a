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

// Eight consecutive values of a row as FP32, zeros behind the row's end.
template <typename T, bool VECTOR>
__device__ __forceinline__ void load8(const T *row, uint32_t col, uint32_t cols, float *v)
{
    if (VECTOR && col + 8 <= cols) {
        constexpr int N = Word<T>::N;
#pragma unroll
        for (int i = 0; i < 2 / N; ++i) {
            const uint4 w = *reinterpret_cast<const uint4 *>(row + col + 4 * N * i);
            Word<T>::unpack(w.x, v + N * (4 * i));
            Word<T>::unpack(w.y, v + N * (4 * i + 1));
            Word<T>::unpack(w.z, v + N * (4 * i + 2));
            Word<T>::unpack(w.w, v + N * (4 * i + 3));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? el::to_float(row[col + i]) : 0.f;
    }
}

// Codes and scale of the block that four neighbouring lanes hold, eight values each.
__device__ __forceinline__ uint32_t encode_block(const float *v, uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, mx::magnitude(v[i]));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    scale = mx::scale_of(top);
    const float f = mx::inverse_scale(scale);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = v[i] * f;
    const uint32_t codes = mx::encode8(u);
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

// Along the rows only: a warp takes PIECES times 256 columns, one piece after the other through the matrix, and asks for all
// of them before it works on the first.
template <typename T, bool VECTOR, int PIECES>
__global__ void __launch_bounds__(32 * WARPS)
quantise_rows_kernel(const T *__restrict__ x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *__restrict__ codes,
                     uint8_t *__restrict__ scales)
{
    el::enter_stream_order();
    const uint32_t ksteps = (cols + 255) / 256;
    const uint32_t first = (blockIdx.x * WARPS + (threadIdx.x >> 5)) * PIECES;
    const int lane = threadIdx.x & 31;
    const uint64_t rb = mx::row_bytes(cols);
    uint32_t row = first / ksteps, k = first % ksteps;
    uint32_t row_of[PIECES], k_of[PIECES];
    float v[PIECES][8];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        row_of[i] = row;
        k_of[i] = k;
        if (row < rows) load8<T, VECTOR>(x + row * ld, k * 256 + lane * 8, cols, v[i]);
        if (++k == ksteps) {
            k = 0;
            ++row;
        }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        if (row_of[i] >= rows) break;
        const uint32_t col = k_of[i] * 256 + lane * 8;
        uint32_t scale;
        const uint32_t c = encode_block(v[i], scale);
        if (col / 2 < rb) *reinterpret_cast<uint32_t *>(codes + row_of[i] * rb + col / 2) = c;
        const uint32_t w = gather_scales(scale, lane);
        if ((lane & 15) == 0)
            *reinterpret_cast<uint32_t *>(scales + mx::scale_offset(row_of[i], (uint64_t)k_of[i] * 8 + (lane >> 2), ksteps)) = w;
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
    el::enter_stream_order();
    extern __shared__ __align__(16) uint8_t smem[];
    T *tile = reinterpret_cast<T *>(smem);
    uint8_t *out = smem + TILE * TILE * sizeof(T);
    uint8_t *atom = out + TILE * COLUMN_PITCH, *atom_t = atom + 512;
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t col_tiles = (cols + TILE - 1) / TILE, row_tiles = (rows + TILE - 1) / TILE;
    const uint32_t tc = blockIdx.x % col_tiles, tr = blockIdx.x / col_tiles;
    const uint32_t r0 = tr * TILE, c0 = tc * TILE;
    const uint64_t rb = mx::row_bytes(cols), rb_t = mx::row_bytes(rows);

    // sixteen lanes take 128 columns of a row
#pragma unroll 4
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = i * 16 + (tid >> 4), col = c0 + (tid & 15) * 8;
        float v[8];
        if (r0 + r < rows) {
            load8<T, VECTOR>(x + (uint64_t)(r0 + r) * ld, col, cols, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
        if constexpr (ROWS) {
            uint32_t scale;
            const uint32_t c = encode_block(v, scale);
            if (r0 + r < rows && col / 2 < rb) *reinterpret_cast<uint32_t *>(codes + (r0 + r) * rb + col / 2) = c;
            const uint32_t w = gather_scales(scale, lane);
            if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(atom + (r & 31) * 16 + (r >> 5) * 4) = w;
        }
        T *dst = tile + r * TILE + (tid & 15) * 8;
        constexpr int N = Word<T>::N;
#pragma unroll
        for (int j = 0; j < 2 / N; ++j)
            reinterpret_cast<uint4 *>(dst)[j] = make_uint4(Word<T>::pack(v + N * (4 * j)), Word<T>::pack(v + N * (4 * j + 1)),
                                                           Word<T>::pack(v + N * (4 * j + 2)), Word<T>::pack(v + N * (4 * j + 3)));
    }
    __syncthreads();

    // a thread takes one block of 32 rows of two neighbouring columns
    {
        const int block = tid >> 6, pair = tid & 63;
        float a[32], b[32];
        uint32_t top_a = 0, top_b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const T *p = tile + (block * 32 + i) * TILE + pair * 2;
            if constexpr (sizeof(T) == 4) {
                const float2 f = *reinterpret_cast<const float2 *>(p);
                a[i] = f.x;
                b[i] = f.y;
            } else {
                float f[2];
                Word<T>::unpack(*reinterpret_cast<const uint32_t *>(p), f);
                a[i] = f[0];
                b[i] = f[1];
            }
            top_a = max(top_a, mx::magnitude(a[i]));
            top_b = max(top_b, mx::magnitude(b[i]));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float *v = h ? b : a;
            const uint32_t scale = mx::scale_of(h ? top_b : top_a);
            const float f = mx::inverse_scale(scale);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= f;
            uint4 c = make_uint4(mx::encode8(v), mx::encode8(v + 8), mx::encode8(v + 16), mx::encode8(v + 24));
            if (scale == mx::NAN_SCALE) c = make_uint4(0u, 0u, 0u, 0u);
            const int col = pair * 2 + h;
            *reinterpret_cast<uint4 *>(out + col * COLUMN_PITCH + block * 16) = c;
            atom_t[(col & 31) * 16 + (col >> 5) * 4 + block] = (uint8_t)scale;
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

// A warp takes 256 columns of one row.
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(32 * WARPS)
dequantise_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t rows, uint32_t cols,
                  T *__restrict__ out, uint64_t ld)
{
    el::enter_stream_order();
    const uint32_t ksteps = (cols + 255) / 256;
    const uint32_t item = blockIdx.x * WARPS + (threadIdx.x >> 5);
    const uint32_t row = item / ksteps, k = item % ksteps;
    if (row >= rows) return;
    const int lane = threadIdx.x & 31;
    const uint32_t col = k * 256 + lane * 8;
    if (col >= cols) return;
    const uint32_t c = *reinterpret_cast<const uint32_t *>(codes + row * mx::row_bytes(cols) + col / 2);
    const float s = mx::scale_value(scales[mx::scale_offset(row, (uint64_t)k * 8 + (lane >> 2), ksteps)]);
    float v[8];
    mx::decode8(c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
    T *dst = out + row * ld + col;
    if (VECTOR && col + 8 <= cols) {
        constexpr int N = Word<T>::N;
#pragma unroll
        for (int j = 0; j < 2 / N; ++j)
            reinterpret_cast<uint4 *>(dst)[j] = make_uint4(Word<T>::pack(v + N * (4 * j)), Word<T>::pack(v + N * (4 * j + 1)),
                                                           Word<T>::pack(v + N * (4 * j + 2)), Word<T>::pack(v + N * (4 * j + 3)));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) dst[i] = el::from_float<T>(v[i]);
    }
}

template <typename T, bool VECTOR>
int quantise(const void *x, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
             uint8_t *scales_t, void *stream)
{
    const T *src = static_cast<const T *>(x);
    if (!codes_t) {
        const uint64_t items = (uint64_t)rows * ((cols + 255) / 256);
        // few pieces: one a warp, so that more warps share them
        if (items <= 148 * 64)
            return note_cuda(el::launch(quantise_rows_kernel<T, VECTOR, 1>, dim3((uint32_t)((items + WARPS - 1) / WARPS)), 32 * WARPS, 0, 1,
                                        stream, src, rows, cols, ld, codes, scales));
        return note_cuda(el::launch(quantise_rows_kernel<T, VECTOR, 4>, dim3((uint32_t)((items + 4 * WARPS - 1) / (4 * WARPS))), 32 * WARPS,
                                    0, 1, stream, src, rows, cols, ld, codes, scales));
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
    const uint64_t items = (uint64_t)rows * ((cols + 255) / 256);
    return note_cuda(el::launch(dequantise_kernel<T, VECTOR>, dim3((uint32_t)((items + WARPS - 1) / WARPS)), 32 * WARPS, 0, 1, stream,
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
