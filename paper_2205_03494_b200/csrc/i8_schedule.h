// Which kernel a product of two 8-bit matrices takes (omc_byte_matmul.cu), by its shape.  Sums of integers are exact, so the choice does
// not show in the results.  Plain C++, so that the rule can be checked on the host.
#pragma once
#include <stdint.h>

namespace omc {
namespace i8 {

constexpr uint32_t LAID_OUT_SMS = 148, STEP_K = 128;

struct Schedule {
    uint32_t tile;          // rows of X in a tile: 16, 32, 64 or 128 (the small kernel), 256 (pairs of SMs)
    uint32_t splits;        // CTAs, a cluster, among which a tile's K is divided: 1, 2, 4 or 8
};

// Up to four rows are multiplied without the tensor cores, if their codes fit in shared memory with two CTAs on an SM.
inline bool few_rows(uint64_t M, uint64_t K) { return M <= 4 && (M > 2 ? 4 : M) * ((K + 15) / 16 * 16) <= 96 * 1024; }

inline uint64_t small_tiles(uint64_t M, uint64_t N, uint32_t tile) { return (N + 127) / 128 * ((M + tile - 1) / tile); }

// Pairs of SMs where they have tiles for half of the SMs; else the small kernel, with the narrowest tile that holds X's rows, K divided while
// all CTAs are resident at once, two to an SM, and a CTA keeps four steps.
inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K, bool gated)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K, columns = gated ? 128 : 256;
    const uint64_t pair_tiles = (M + 255) / 256 * ((N + columns - 1) / columns);
    if (M > 128 && pair_tiles * 4 >= LAID_OUT_SMS) return {256u, 1u};
    Schedule s = {M <= 16 ? 16u : M <= 32 ? 32u : M <= 64 || gated ? 64u : 128u, 1u};
    const uint64_t tiles = small_tiles(M, N, s.tile), resident = gated && s.tile > 32 ? LAID_OUT_SMS : 2 * LAID_OUT_SMS;
    while (s.splits < 8 && tiles * s.splits * 2 <= resident && ksteps >= s.splits * 8) s.splits *= 2;
    return s;
}

}  // namespace i8
}  // namespace omc
