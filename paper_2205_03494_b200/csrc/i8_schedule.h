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

// Up to 64 rows: the small kernel with the narrowest tile that holds them, K divided among 4 or 8 CTAs where they are all resident at once, two to an SM, and each
// keeps two steps (divided in two it gains nothing: joining takes as long as half the steps of a short sum).  More rows: whichever tile takes least time by
// its number of rounds over the SMs and what a tile of it costs; measured in us, tiles of 256 x 256 on two SMs 0.30 a step and 1.1 a tile, 256 x 128 0.2 and 1.1,
// 128 x 128 on one 0.2 and 1.0.
inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K, bool gated)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K;
    if (const char *e = getenv("I8K")) { const char *f = getenv("I8S"); return {(Kernel)atoi(e), f ? (uint32_t)atoi(f) : 1u}; }
    const uint32_t half = gated ? 2 : 1;
    if (M > 64) {
        const uint64_t pairs = LAID_OUT_SMS / 2;
        const uint64_t r256 = (tiles_of(M, N, 256, 256 / half) + pairs - 1) / pairs, r128 = (tiles_of(M, N, 256, 128 / half) + pairs - 1) / pairs;
        const uint64_t r1 = (tiles_of(M, N, 128, 128 / half) + LAID_OUT_SMS - 1) / LAID_OUT_SMS;
        const uint64_t c256 = r256 * (30 * ksteps + 110), c128 = r128 * (20 * ksteps + 110), c1 = r1 * (20 * ksteps + 100);
        return {c1 <= c128 && c1 <= c256 ? ONE_128 : c128 <= c256 ? PAIR_128 : PAIR_256, 1u};
    }
    Schedule s = {M <= 16 ? SMALL_16 : M <= 32 ? SMALL_32 : SMALL_64, 1u};
    const uint64_t tiles = tiles_of(M, N, M <= 16 ? 16 : M <= 32 ? 32 : 64, 128), resident = gated && s.kernel == SMALL_64 ? LAID_OUT_SMS : 2 * LAID_OUT_SMS;
    for (uint32_t n = 4; n <= 8; n *= 2)
        if (tiles * n <= resident && ksteps >= 2 * n) s.splits = n;
    return s;
}

}  // namespace i8
}  // namespace omc
