// The gradients of a gated layer's gate and value, as a source of the 8-bit quantisation (i8_quantise.cuh); compiled for each activation in a file of its own
// (with the activation chosen at run time the kernels' code did not fit the instruction cache: 13 % of the second kernel's issue slots waited for it).
#pragma once
#include "element.cuh"
#include "gate.cuh"
#include "i8_format.cuh"
#include "i8_quantise.cuh"
#include "omc_internal.h"

namespace omc {
namespace gate {

using el::Word;

// Pieces of dy, a and b read, of da and db made.
template <typename T_, bool WHOLE, int ACT>
struct Gradients {
    using T = T_;
    static constexpr int OUT = 2, HEAVY = WHOLE ? 1 : 2;
    static constexpr bool WHOLE_ROWS = WHOLE;
    const T *dy, *pre;
    T *dpre;                  // NULL: not wanted
    uint64_t ld_dy, ld_pre, ld_dpre;
    uint32_t rows, width;
    struct Raw {
        i8::Piece<T, WHOLE> g, a, b;
    };
    __device__ __forceinline__ void fetch(uint32_t row, uint32_t col, uint32_t cols, Raw &raw) const
    {
        const bool in = i8::inside<T>(row, rows, cols);
        const T *const p = pre + row * ld_pre + col;
        raw.g.load(dy + row * ld_dy + col, in);
        raw.a.load(p, in);
        raw.b.load(p + width, in);
    }
    template <bool EDGE>
    __device__ __forceinline__ void fetch4(uint32_t row, uint32_t col, Raw *raw) const
    {
        const i8::Nearest<WHOLE> near(row, rows);
        const uint32_t first = EDGE ? near.first() : row;
        const T *p = dy + first * ld_dy + col, *q = pre + first * ld_pre + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            raw[i].g.load(p, true);
            raw[i].a.load(q, true);
            raw[i].b.load(q + width, true);
            if (!EDGE || near.on(i)) p += ld_dy, q += ld_pre;
        }
    }
    static __device__ __forceinline__ void make_with(const uint32_t *gs, const uint32_t *as, const uint32_t *bs, uint32_t (*out)[4])
    {
        constexpr int N = Word<T>::N;
#pragma unroll
        for (int i = 0; i < 4; i += 2 / N) {              // two values
            float g[2], a[2], b[2];
#pragma unroll
            for (int j = 0; j < 2 / N; ++j) {
                Word<T>::unpack(gs[i + j], g + j);
                Word<T>::unpack(as[i + j], a + j);
                Word<T>::unpack(bs[i + j], b + j);
            }
            float2 v, d;
            gate::act_slope2<ACT, sizeof(T) == 4>(make_float2(a[0], a[1]), v, d);
            const float2 g2 = make_float2(g[0], g[1]), da = el::mul2(el::mul2(g2, make_float2(b[0], b[1])), d), db = el::mul2(g2, v);
            const float x[2] = {da.x, da.y}, y[2] = {db.x, db.y};
#pragma unroll
            for (int j = 0; j < 2 / N; ++j) {
                out[0][i + j] = Word<T>::pack(x + j);
                out[1][i + j] = Word<T>::pack(y + j);
            }
        }
    }
    __device__ __forceinline__ void make(uint32_t row, uint32_t col, uint32_t cols, const Raw &raw, uint32_t (*out)[4]) const
    {
        uint32_t g[4], a[4], b[4];
        const bool in = WHOLE || i8::inside<T>(row, rows, cols);
        const T *const p = pre + row * ld_pre + col;
        raw.g.words(dy + row * ld_dy + col, cols - col, in, g);
        raw.a.words(p, cols - col, in, a);
        raw.b.words(p + width, cols - col, in, b);
        make_with(g, a, b, out);
    }
    __device__ __forceinline__ void emit(uint32_t row, uint32_t col, uint32_t cols, const uint32_t (*w)[4]) const
    {
        if (!dpre) return;
        constexpr int E = i8::PIECE<T>;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            T *to = dpre + row * ld_dpre + (o ? width : 0u) + col;
            if (WHOLE) {
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

struct Backward {
    const void *dy, *pre;
    uint64_t ld_dy, ld_pre;
    int type;
    uint32_t rows, width;
    bool whole;               // every row on a 16-byte boundary and a multiple of 16 bytes wide
    void *dpre;
    uint64_t ld_dpre;
    int8_t *codes;
    float *scales;
    int8_t *codes_t;
    float *scales_t;
    void *workspace, *stream;
};

template <typename T, bool WHOLE, int ACT>
int backward(const Backward &c)
{
    const T *const g = static_cast<const T *>(c.dy), *const p = static_cast<const T *>(c.pre);
    const Gradients<T, WHOLE, ACT> src = {g, p, static_cast<T *>(c.dpre), c.ld_dy, c.ld_pre, c.ld_dpre, c.rows, c.width};
    return i8::quantise<2>(src, c.rows, c.width, c.codes, c.scales, c.codes_t, c.scales_t, c.workspace, c.stream);
}
template <int ACT>
int backward(const Backward &c)
{
    if (c.type == OMC_TYPE_F32) return c.whole ? backward<float, true, ACT>(c) : backward<float, false, ACT>(c);
    if (c.type == OMC_TYPE_F16) return c.whole ? backward<__half, true, ACT>(c) : backward<__half, false, ACT>(c);
    return c.whole ? backward<__nv_bfloat16, true, ACT>(c) : backward<__nv_bfloat16, false, ACT>(c);
}
int backward_sigmoid(const Backward &c);
int backward_silu(const Backward &c);
int backward_gelu(const Backward &c);

}  // namespace gate
}  // namespace omc
