// Which kernel a product of two 8-bit matrices takes (omc_i8_matmul.cu), by its shape.  Sums of integers are exact, so the choice does
// not show in the results.  Plain C++, so that the rule can be checked on the host.
#pragma once
#include <stdint.h>

namespace omc {
namespace i8 {

constexpr uint32_t LAID_OUT_SMS = 148, STEP_K = 128;

// Tiles of rows of X x rows of W: 256 x 256 on a pair of SMs, 128 x 128 on one; 16, 32 or 64 x 128 of the small kernel.
enum Kernel { PAIR_256, ONE_128, SMALL_16, SMALL_32, SMALL_64 };
struct Schedule {
    Kernel kernel;
    uint32_t splits;        // CTAs, a cluster, among which a tile's K is divided (small kernel): 1, 2, 4 or 8
};

// Up to four rows are multiplied without the tensor cores, if their codes fit in shared memory with two CTAs on an SM.
inline bool few_rows(uint64_t M, uint64_t K) { return M <= 4 && (M > 2 ? 4 : M) * ((K + 15) / 16 * 16) <= 96 * 1024; }

inline uint64_t tiles_of(uint64_t M, uint64_t N, uint32_t rows, uint32_t cols) { return (M + rows - 1) / rows * ((N + cols - 1) / cols); }

// CTAs among which the small kernel divides the K of `tiles` tiles: eight while each has an SM, four while two share one, and each CTA has a step.
// (In two it gains nothing: joining takes as long as half the steps of a short sum.)
inline uint32_t splits_of(uint64_t tiles, uint64_t ksteps, uint64_t resident)
{
    return tiles * 8 <= LAID_OUT_SMS && ksteps >= 8 ? 8u : tiles * 4 <= resident && ksteps >= 4 ? 4u : 1u;
}

// Whichever kernel takes least time by what was measured, in 1/100 us: `base` with one tile's results, `step` for each K step of 128, and a further tile of the
// same SMs as long as its steps or the results of the one before, whichever is longer.
//   256 x 256 on a pair    480 + 31 a step, 37 while results are stored, 290 for results (gated 550)
//   128 x 128 on an SM     390 + 24, 175 (290)
//   (256 x 128 on a pair is no faster than 128 x 128 on an SM: 8.5 and 7.8 us at 512 x 2048 x 2048 BF16, 17.0 and 18.7 at 3000 x 2002 x 1000 FP32)
//   small kernel           440 + 28 (two CTAs on an SM: 45), 90 more with divided K
inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K, bool gated)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K;
    const uint32_t half = gated ? 2 : 1, rows = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    const Kernel small = M <= 16 ? SMALL_16 : M <= 32 ? SMALL_32 : SMALL_64;
    const uint64_t tiles = tiles_of(M, N, rows, 128), resident = gated && small == SMALL_64 ? LAID_OUT_SMS : 2 * LAID_OUT_SMS;
    const uint32_t splits = splits_of(tiles, ksteps, resident);
    const uint64_t ctas = tiles * splits, mine = (ksteps + splits - 1) / splits, rounds = (ctas + resident - 1) / resident;
    Schedule best = {small, splits};
    uint64_t least = rounds * (440 + mine * (ctas > LAID_OUT_SMS ? 45 : 28)) + (splits > 1 ? 90 : 0);
    auto consider = [&](Kernel kernel, uint64_t all, uint64_t units, uint64_t base, uint64_t step, uint64_t later_step, uint64_t results) {
        const uint64_t further = (all + units - 1) / units - 1, later = ksteps * later_step;
        const uint64_t cost = base + ksteps * step + further * (later > results ? later : results);
        if (cost < least) {
            least = cost;
            best = {kernel, 1u};
        }
    };
    consider(ONE_128, tiles_of(M, N, 128, 128 / half), LAID_OUT_SMS, 390, 24, 24, gated ? 290 : 175);
    consider(PAIR_256, tiles_of(M, N, 256, 256 / half), LAID_OUT_SMS / 2, 480, 31, 37, gated ? 550 : 290);
    return best;
}

}  // namespace i8
}  // namespace omc
