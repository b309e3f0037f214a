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
    uint32_t splits;        // CTAs, a cluster, among which a tile's K is divided (small kernel): 1, 4 or 8
};

// Up to four rows are multiplied without the tensor cores, if their codes fit in shared memory with two CTAs on an SM.
inline bool few_rows(uint64_t M, uint64_t K) { return M <= 4 && (M > 2 ? 4 : M) * ((K + 15) / 16 * 16) <= 96 * 1024; }

inline uint64_t tiles_of(uint64_t M, uint64_t N, uint32_t rows, uint32_t cols) { return (M + rows - 1) / rows * ((N + cols - 1) / cols); }

// Small kernel, 1/100 us: time without K steps, and a step's (gated: two tiles of W).  A CTA gives the others of its cluster their rows' sums and
// stores its own, so a divided tile's results take less, joining takes the more the more CTAs there are.
//   8 x 512 x 512 BF16   1 CTA a tile 3.4 us, 4: 3.6        8 x 4096 x 1024: 4.6, 4.2        gated 8 x 512 x 512: 4.9, 4.2
//   64 x 512 x 2048      1 CTA a tile 10.1 us, 8: 6.8       gated 64 x 512 x 2048: 15.5, 10.3
constexpr uint32_t SMALL_BASE[2][3][3] = {{{245, 330, 315}, {405, 405, 345}, {630, 500, 445}}, {{350, 375, 360}, {590, 530, 445}, {950, 730, 690}}};
constexpr uint32_t SMALL_STEP[2] = {25, 39};

// Whichever kernel takes least time by what was measured, in 1/100 us: `base` with one tile's results, `step` for each K step of 128, and a further tile of the
// same SMs as long as its steps or the results of the one before, whichever is longer.  Results whose rows do not start on 16-byte boundaries (not `whole`)
// take longer and hold up the steps meanwhile (ONE_128 at 64 x 700 x 512 BF16 takes 6.6 us, with 704 columns 4.4; 4000 x 3001 x 2000 FP32: 50.6, PAIR_256 36.4).
//   256 x 256 on a pair    480 + 31 a step, 37 while results are stored, 290 for results (gated 550)
//   128 x 128 on an SM     390 + 24, 175 (290)
//   (256 x 128 on a pair is no faster than 128 x 128 on an SM: 8.5 and 7.8 us at 512 x 2048 x 2048 BF16, 17.0 and 18.7 at 3000 x 2002 x 1000 FP32)
inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K, bool gated, bool whole)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K;
    const uint32_t half = gated ? 2 : 1, size = M <= 16 ? 0 : M <= 32 ? 1 : 2;
    const Kernel small = size == 0 ? SMALL_16 : size == 1 ? SMALL_32 : SMALL_64;
    // (a gated CTA of 64 rows has an SM to itself)
    const uint64_t tiles = tiles_of(M, N, 16u << size, 128), resident = gated && small == SMALL_64 ? LAID_OUT_SMS : 2 * LAID_OUT_SMS;
    // one CTA an SM does not keep memory busy with a W that L2 cannot hold (gated 8 x 4096 x 8192: four CTAs a tile 19.3 us, eight 14.5)
    const bool streams = half * N * K > (48ull << 20);
    Schedule best = {small, 1u};
    uint64_t least = ~0ull;
    for (uint32_t i = 0; i < 3; ++i) {
        const uint64_t splits = i == 0 ? 1 : 2u << i, ctas = tiles * splits, mine = (ksteps + splits - 1) / splits;
        // A divided tile's CTAs, a cluster, all run at once.  (Clusters of eight with an SM for each CTA do not fill the GPU: gated 64 x 2048 x 2048
        // takes 15.6 us with 128 CTAs, 9.2 with 64 in fours; 77 x 777 x 1000 8.0 with 112, 8.7 with 56.)
        if (splits > 1 && (ctas > (resident == LAID_OUT_SMS && splits == 8 ? 112 : resident) || ksteps < splits)) continue;
        const uint64_t step = SMALL_STEP[gated] * (ctas > LAID_OUT_SMS ? 8 : streams ? 15 : 5) / 5;
        const uint64_t cost = (ctas + resident - 1) / resident * (SMALL_BASE[gated][size][i] + mine * step) + ctas * (splits - 1) / 8;
        if (cost < least) {
            least = cost;
            best.splits = (uint32_t)splits;
        }
    }
    auto consider = [&](Kernel kernel, uint64_t all, uint64_t units, uint64_t base, uint64_t step, uint64_t later_step, uint64_t results, uint64_t longer) {
        const uint64_t further = (all + units - 1) / units - 1, later = ksteps * later_step;
        const uint64_t each = !whole ? later + results + longer : later > results ? later : results;
        const uint64_t cost = base + (whole ? 0 : longer) + ksteps * step + further * each;
        if (cost < least) {
            least = cost;
            best = {kernel, 1u};
        }
    };
    consider(ONE_128, tiles_of(M, N, 128, 128 / half), LAID_OUT_SMS, 390, 24, 24, gated ? 290 : 175, gated ? 370 : 300);
    consider(PAIR_256, tiles_of(M, N, 256, 256 / half), LAID_OUT_SMS / 2, 480, 31, 37, gated ? 550 : 290, gated ? 850 : 600);
    return best;
}

}  // namespace i8
}  // namespace omc
