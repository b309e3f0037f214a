// Tile and division of K of a product of two quantised matrices (omc_mx_matmul.cu).  They fix the order in which its sums are
// formed, so they follow from the shape alone, for the 148 SMs that the kernels are laid out for: the device is not
// asked.  Plain C++, so that the rule can be checked on the host.
#pragma once
#include <stdint.h>

namespace omc {
namespace mx {

constexpr uint32_t LAID_OUT_SMS = 148;
constexpr uint32_t TILE_W = 128, STEP_K = 256;        // rows of W in a tile; K of a step

struct Schedule {
    uint32_t tile;          // rows of X in a tile: 16, 32, 64 (the few-row kernel), 128 or 256
    uint32_t splits;        // CTAs, a cluster, among which a tile's K is divided: 1, 2, 4 or 8
};

inline uint64_t tiles_of(uint64_t M, uint64_t N, uint32_t tile) { return (N + TILE_W - 1) / TILE_W * ((M + tile - 1) / tile); }

// Up to 64 rows of X: the narrowest tile that holds them all, K divided while all CTAs are resident at once, two to an SM, and a CTA
// keeps two steps (joining takes 0.5 us, a step 0.4 us).
// More: tiles of 128 or 256 rows, whichever takes less time by its number of rounds over the SMs; measured, a round takes about
// 0.35 (K steps + 2) us with 128 rows, 0.36 (K steps + 5) us with 256 (1024 x 2048 x 2048: 6.7 and 7.7 us; 3000 x 1000 x 1000:
// 7.1 and 6.6 us).  K is divided while the clusters still fit on the SMs at once: joining the parts takes about 2 us, a step
// 0.34 us (128 x 8192 x 8192: 15.0 us undivided, 11.7 us in two; 1999 x 512 x 2048: 6.4 us undivided, 7.5 us in two).  Tiles of 256
// rows are taken only where those of 128 need two rounds, so there are too many of them to divide K.
inline Schedule schedule_of(uint64_t M, uint64_t N, uint64_t K)
{
    const uint64_t ksteps = (K + STEP_K - 1) / STEP_K;
    Schedule s = {M <= 16 ? 16u : M <= 32 ? 32u : 64u, 1u};
    if (M <= 64) {
        const uint64_t tiles = tiles_of(M, N, s.tile);
        while (s.splits < 8 && tiles * s.splits <= LAID_OUT_SMS && ksteps >= s.splits * 4) s.splits *= 2;
        return s;
    }
    const uint64_t rounds128 = (tiles_of(M, N, 128) + LAID_OUT_SMS - 1) / LAID_OUT_SMS, rounds256 = (tiles_of(M, N, 256) + LAID_OUT_SMS - 1) / LAID_OUT_SMS;
    s.tile = rounds128 * (ksteps + 2) <= rounds256 * (ksteps + 5) ? 128u : 256u;
    while (s.tile == 128 && s.splits < 4 && tiles_of(M, N, s.tile) * s.splits * 2 <= LAID_OUT_SMS && ksteps >= 16) s.splits *= 2;
    return s;
}

}  // namespace mx
}  // namespace omc
