// omc_gated_backward: from the gradient of y = act(a) b and the (a | b) that the forward pass left,
//     da = dy b act'(a),   db = dy act(a)
// as a matrix of the activations' type, and / or as 8-bit integers along its rows and its columns (i8_quantise.cuh), which the two products of the
// layer's backward pass take: (da | db) is made again in the second kernel instead of being written and read (16 bytes a value
// of dy for 16-bit types instead of 22).
#include <cuda_runtime.h>

#include "element.cuh"
#include "gate.cuh"
#include "i8_format.cuh"
#include "i8_quantise.cuh"
#include "omc_internal.h"

namespace omc {
bool i8_shape_ok(uint64_t rows, uint64_t cols);
}

namespace {

using namespace omc;
using el::Word;

// Pieces of dy, a and b read, of da and db made.
template <typename T_, bool VECTOR>
struct Gradients {
    using T = T_;
    static constexpr int IN = 3, OUT = 2;
    const T *dy, *pre;
    T *dpre;                  // NULL: not wanted
    uint64_t ld_dy, ld_pre, ld_dpre;
    uint32_t width;
    int act;
    __device__ __forceinline__ void fetch(uint32_t row, uint32_t col, uint32_t cols, uint32_t (*raw)[4]) const
    {
        mx::load<T, VECTOR, i8::PIECE<T>>(dy + row * ld_dy, col, cols, raw[0]);
        mx::load<T, VECTOR, i8::PIECE<T>>(pre + row * ld_pre, col, cols, raw[1]);
        mx::load<T, VECTOR, i8::PIECE<T>>(pre + row * ld_pre + width, col, cols, raw[2]);
    }
    template <int ACT>
    static __device__ __forceinline__ void make_with(const uint32_t (*raw)[4], uint32_t (*out)[4])
    {
        constexpr int N = Word<T>::N;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float g[N], a[N], b[N];
            Word<T>::unpack(raw[0][i], g);
            Word<T>::unpack(raw[1][i], a);
            Word<T>::unpack(raw[2][i], b);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float v, d;
                gate::act_slope<ACT>(a[j], v, d);
                a[j] = g[j] * b[j] * d;
                b[j] = g[j] * v;
            }
            out[0][i] = Word<T>::pack(a);
            out[1][i] = Word<T>::pack(b);
        }
    }
    __device__ __forceinline__ void make(const uint32_t (*raw)[4], uint32_t (*out)[4]) const
    {
        if (act == OMC_GATE_SILU) make_with<OMC_GATE_SILU>(raw, out);
        else if (act == OMC_GATE_SIGMOID) make_with<OMC_GATE_SIGMOID>(raw, out);
        else make_with<OMC_GATE_GELU>(raw, out);
    }
    __device__ __forceinline__ void emit(uint32_t row, uint32_t col, uint32_t cols, const uint32_t (*w)[4]) const
    {
        if (!dpre) return;
        constexpr int E = i8::PIECE<T>;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            T *to = dpre + row * ld_dpre + (o ? width : 0u) + col;
            if (VECTOR && col + E <= cols) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(w[o][0], w[o][1], w[o][2], w[o][3]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col + e < cols) {
                        if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(to)[e] = w[o][e % 4];
                        else reinterpret_cast<uint16_t *>(to)[e] = (uint16_t)(w[o][e / 2] >> (16 * (e & 1)));
                    }
            }
        }
    }
};

template <typename T, bool VECTOR>
int backward(const void *dy, uint64_t ld_dy, const void *pre, uint64_t ld_pre, uint32_t rows, uint32_t width, int act, void *dpre, uint64_t ld_dpre,
             int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace, void *stream)
{
    const Gradients<T, VECTOR> src = {static_cast<const T *>(dy), static_cast<const T *>(pre), static_cast<T *>(dpre), ld_dy, ld_pre, ld_dpre, width, act};
    return i8::quantise<2>(src, rows, width, codes, scales, codes_t, scales_t, workspace, stream);
}

bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// Whether rows x cols matrices of pitch ld have a byte in common, taken from their first to their last.
bool overlap(const void *a, uint64_t ld_a, uint64_t cols_a, const void *b, uint64_t ld_b, uint64_t cols_b, uint64_t rows, uint64_t size)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    const uint64_t na = ((rows - 1) * ld_a + cols_a) * size, nb = ((rows - 1) * ld_b + cols_b) * size;
    return p < q + nb && q < p + na;
}

}  // namespace

extern "C" int omc_gated_backward_workspace(uint64_t rows, uint64_t width, uint64_t *bytes)
{
    if (!bytes) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, width) || !i8_shape_ok(rows, 2 * width)) return OMC_ERR_INVALID_ARG;
    *bytes = 2 * i8::parts_bytes(rows, width);
    return OMC_OK;
}

extern "C" int omc_gated_backward(const void *dy, uint64_t ld_dy, const void *pre, uint64_t ld_pre, int type, uint64_t rows, uint64_t width, int activation,
                                  void *dpre, uint64_t ld_dpre, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace,
                                  void *stream)
{
    if (!el::type_ok(type) || activation < OMC_GATE_SIGMOID || activation > OMC_GATE_GELU) return OMC_ERR_INVALID_ARG;
    if (!dy || !pre || (!dpre && !codes && !codes_t) || !codes != !scales || !codes_t != !scales_t || (codes_t && !workspace)) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, width) || !i8_shape_ok(rows, 2 * width) || ld_dy < width || ld_pre < 2 * width || (dpre && ld_dpre < 2 * width))
        return OMC_ERR_INVALID_ARG;
    const uint64_t size = el::size_of(type);
    if (reinterpret_cast<uintptr_t>(dy) % size || reinterpret_cast<uintptr_t>(pre) % size || reinterpret_cast<uintptr_t>(dpre) % size ||
        !el::aligned16(codes) || !aligned4(scales) || !el::aligned16(codes_t) || !aligned4(scales_t) || !el::aligned16(workspace))
        return OMC_ERR_MISALIGNED;
    if (dpre && (overlap(dpre, ld_dpre, 2 * width, dy, ld_dy, width, rows, size) || overlap(dpre, ld_dpre, 2 * width, pre, ld_pre, 2 * width, rows, size)))
        return OMC_ERR_INVALID_ARG;
    const bool vec = el::aligned16(dy) && el::aligned16(pre) && el::aligned16(dpre) && ld_dy * size % 16 == 0 && ld_pre * size % 16 == 0 &&
                     (!dpre || ld_dpre * size % 16 == 0) && width * size % 16 == 0;
    const uint32_t r = (uint32_t)rows, w = (uint32_t)width;
#define OMC_CALL(T) (vec ? backward<T, true>(dy, ld_dy, pre, ld_pre, r, w, activation, dpre, ld_dpre, codes, scales, codes_t, scales_t, workspace, stream) \
                         : backward<T, false>(dy, ld_dy, pre, ld_pre, r, w, activation, dpre, ld_dpre, codes, scales, codes_t, scales_t, workspace, stream))
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}
