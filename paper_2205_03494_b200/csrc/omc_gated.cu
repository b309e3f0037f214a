// omc_gated_backward: from the gradient of y = act(a) b and the (a | b) that the forward pass left,
//     da = dy b act'(a),   db = dy act(a)
// as a matrix of the activations' type, and / or as 8-bit integers along its rows and its columns (i8_quantise.cuh), which the two products of the
// layer's backward pass take: (da | db) is made again in the second kernel instead of being written by the first and read by the second (16 bytes a value
// of dy for 16-bit types instead of 18; the other way, with a second kernel of fewer registers, has not been tried).
// The matrix alone is bound by memory: 8192 x 8192 BF16 107 us, 6.3 TB/s.  With the codes along both axes 8192 x 8192 BF16 takes 232 us (SiLU; sigmoid 228, GELU 253),
// 4.6 TB/s of what both kernels read and write (more than half of it the second's): the second kernel waits for the latencies of its arithmetic, 168 registers leaving three CTAs of four
// warps an SM.  Rows off the 16-byte boundaries: 506 us at 8192 x 8191.
#include <cuda_runtime.h>

#include "element.cuh"
#include "gated.cuh"
#include "i8_quantise.cuh"
#include "omc_internal.h"

namespace omc {
bool i8_shape_ok(uint64_t rows, uint64_t cols);
}

namespace {

using namespace omc;

bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// Whether matrices of `rows` rows share a byte: of one pitch exactly (column ranges of one buffer do not), else by the ranges from their first to their last byte.
bool overlap(const void *a, uint64_t ld_a, uint64_t cols_a, const void *b, uint64_t ld_b, uint64_t cols_b, uint64_t rows, uint64_t size)
{
    using Wide = __int128;
    const Wide pitch = (Wide)ld_a * size, other = (Wide)ld_b * size, na = (Wide)cols_a * size, nb = (Wide)cols_b * size, last = rows - 1;
    const Wide d = (Wide)reinterpret_cast<uintptr_t>(b) - (Wide)reinterpret_cast<uintptr_t>(a);          // where b starts, counted from a
    if (d >= last * pitch + na || d + last * other + nb <= 0) return false;
    if (pitch != other) return true;
    // row j of b and row j - k of a: d + k pitch into it, which lies within one row's width for two values of k at most
    const Wide k = d >= 0 ? -(d / pitch) : (-d) / pitch;
    for (Wide i = k - 1; i <= k + 1; ++i)
        if (i >= -last && i <= last && d + i * pitch < na && d + i * pitch + nb > 0) return true;
    return false;
}

}  // namespace

extern "C" int omc_gated_backward_workspace(uint64_t rows, uint64_t width, uint64_t *bytes)
{
    if (!bytes) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, width) || !i8_shape_ok(rows, 2 * width)) return OMC_ERR_INVALID_ARG;
    *bytes = i8::maxima_bytes(rows, width, 2);
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
    const bool whole = el::aligned16(dy) && el::aligned16(pre) && el::aligned16(dpre) && ld_dy * size % 16 == 0 && ld_pre * size % 16 == 0 &&
                     (!dpre || ld_dpre * size % 16 == 0) && width * size % 16 == 0;
    const gate::Backward c = {dy, pre, ld_dy, ld_pre, type, (uint32_t)rows, (uint32_t)width, whole, dpre, ld_dpre, codes, scales, codes_t, scales_t, workspace, stream};
    return activation == OMC_GATE_SILU ? gate::backward_silu(c) : activation == OMC_GATE_GELU ? gate::backward_gelu(c) : gate::backward_sigmoid(c);
}
