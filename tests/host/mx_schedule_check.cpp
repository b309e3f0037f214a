// The schedule of a product (tile and division of K) over many shapes: what the kernels rely on.  Exit status 0 if it holds.
#include <stdint.h>
#include <stdio.h>

#include <vector>

#include "../../paper_2205_03494_b200/csrc/mx_schedule.h"

using namespace omc::mx;

static int fail(const char *what, uint64_t M, uint64_t N, uint64_t K)
{
    printf("%s: %llu x %llu x %llu\n", what, (unsigned long long)M, (unsigned long long)N, (unsigned long long)K);
    return 1;
}

int main()
{
    std::vector<uint64_t> sizes;
    for (uint64_t v = 1; v <= 1100; v += v < 300 ? 1 : 37) sizes.push_back(v);
    for (uint64_t v = 2048; v < (1ull << 31); v *= 2) {
        sizes.push_back(v - 1);
        sizes.push_back(v);
        sizes.push_back(v + 1);
    }
    const uint64_t lengths[] = {1, 31, 256, 257, 512, 1000, 1024, 2048, 3840, 3841, 4096, 8192, 100000, (1ull << 31) - 1};
    for (uint64_t M : sizes)
        for (uint64_t N : sizes)
            for (uint64_t K : lengths) {
                if (M > 128ull * 65535) continue;
                const Schedule s = schedule_of(M, N, K);
                const uint64_t steps = (K + STEP_K - 1) / STEP_K, ctas = tiles_of(M, N, s.tile) * s.splits;
                if (s.splits != 1 && s.splits != 2 && s.splits != 4 && s.splits != 8) return fail("division", M, N, K);
                if (s.tile <= 64) {
                    if (M > s.tile) return fail("tile does not hold every row", M, N, K);
                    if (s.splits > 1 && (steps < 2 * s.splits || ctas > 2 * LAID_OUT_SMS)) return fail("few rows, division", M, N, K);
                } else {
                    if (M <= 64 || (s.tile != 128 && s.tile != 256)) return fail("tile", M, N, K);
                    if (s.tile == 256 && s.splits != 1) return fail("division of a tile of 256 rows, which its kernel cannot", M, N, K);
                    // a CTA owns at least 32 rows of the tile and four steps, and every cluster has its SMs
                    if (s.splits > 1 && (s.tile / s.splits < 32 || steps < 4 * s.splits || ctas > LAID_OUT_SMS)) return fail("division of a tile", M, N, K);
                }
            }
    return 0;
}
