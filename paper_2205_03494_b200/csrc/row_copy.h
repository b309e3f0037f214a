// Which bytes a row that does not start on a 16-byte boundary is copied in, 16 at a time (omc_norm.cu).  Plain C++, so that the
// bounds can be checked on the host.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define OMC_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define OMC_HOST_DEVICE inline
#endif

namespace omc {

// Rows whose 16-byte boundary lies below the matrix's first byte, `pitch` bytes from row to row: they are the first ones, all
// that begin in the 16 bytes in which the matrix does (of narrow matrices several).
inline uint32_t rows_from_below(uintptr_t matrix, uint64_t pitch)
{
    const uint32_t skip = (uint32_t)matrix & 15u;
    return skip == 0 ? 0u : pitch >= 16 ? 1u : (15u - skip) / (uint32_t)pitch + 1u;
}

// Bytes from the 16-byte boundary at or below a row to the row.
OMC_HOST_DEVICE uint32_t row_skip(uintptr_t row) { return (uint32_t)row & 15u; }

// Whether piece k of a row, the 16 bytes at row - row_skip(row) + 16 k, is taken value by value from the row's own first byte on.
OMC_HOST_DEVICE bool by_value(uint32_t k, bool from_below) { return k == 0 && from_below; }

}  // namespace omc
