// Which kernel a product of two 8-bit matrices takes (omc_i8_matmul.cu), by its shape.  Sums of integers are exact, so the choice does
// not show in the results.  Plain C++, so that the rule can be checked on the host.
#pragma once
#include <stdint.h>
#include <stdlib.h>

namespace omc {
namespace i8 {

constexpr uint32_t LAID_OUT_SMS = 148, STEP_K = 128;

// Tiles of rows of X x rows of W: 256 x 256 and 256 x 128 on a pair of SMs, 128 x 128 on one; 16, 32 or 64 x 128 of the small kernel.
enum Kernel { PAIR_256, PAIR_128, ONE_128, SMALL_16, SMALL_32, SMALL_64 };
struct Schedule {
    Kernel kernel;
    uint32_t splits;        // CTAs, a cluster, among which a tile's K is divided (small kernel): 1, 2, 4 or 8
};

// Up to four rows are multiplied without the tensor cores, if their codes fit in shared memory with two CTAs on an SM.
inline bool few_rows(uint64_t M, uint64_t K) { return M <= 4 && (M > 2 ? 4 : M) * ((K + 15) / 16 * 16) <= 96 * 1024; }

inline uint64_t tiles_of(uint64_t M, uint64_t N, uint32_t rows, uint32_t cols) { return (M + rows - 1) / rows * ((N + cols - 1) / cols); }

inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K, bool gated)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K;
    if (const char *e = getenv("I8K")) { const char *f = getenv("I8S"); return {(Kernel)atoi(e), f ? (uint32_t)atoi(f) : 1u}; }
    const uint32_t half = gated ? 2 : 1;
    if (M > 64) {
        if (M <= 128) return {ONE_128, 1u};
        return {tiles_of(M, N, 256, 256 / half) * 4 >= LAID_OUT_SMS ? PAIR_256 : PAIR_128, 1u};
    }
    Schedule s = {M <= 16 ? SMALL_16 : M <= 32 ? SMALL_32 : SMALL_64, 1u};
    const uint64_t tiles = tiles_of(M, N, M <= 16 ? 16 : M <= 32 ? 32 : 64, 128), resident = gated && s.kernel == SMALL_64 ? LAID_OUT_SMS : 2 * LAID_OUT_SMS;
    while (s.splits < 8 && tiles * s.splits * 2 <= resident && ksteps >= s.splits * 8) s.splits *= 2;
    return s;
}

}  // namespace i8
}  // namespace omc
