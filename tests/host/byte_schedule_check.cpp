// The kernel of an 8-bit product and its division of K over many shapes: what the kernels rely on, and that every kernel is chosen for some shape.
// Exit status 0 if it holds.
#include <stdint.h>
#include <stdio.h>

#include <vector>

#include "../../paper_2205_03494_b200/csrc/i8_schedule.h"

using namespace omc::i8;

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
    const uint64_t lengths[] = {1, 31, 128, 129, 512, 1000, 1024, 1025, 2048, 4096, 8192, 100000, (1ull << 17) - 1};
    bool chosen[2][5] = {};
    for (int form = 0; form < 4; ++form)
        for (uint64_t M : sizes)
            for (uint64_t N : sizes)
                for (uint64_t K : lengths) {
                    const int gated = form % 2;
                    if (M > 128ull * 65535 || (gated && N >= (1ull << 30))) continue;
                    const Schedule s = schedule_of(M, N, K, gated != 0, form >= 2);
                    const uint64_t steps = (K + STEP_K - 1) / STEP_K;
                    chosen[gated][s.kernel] = true;
                    if (s.kernel < SMALL_16) {
                        if (s.splits != 1) return fail("division of a tile that is not divided", M, N, K);
                        continue;
                    }
                    if (s.splits != 1 && s.splits != 4 && s.splits != 8) return fail("division", M, N, K);
                    if (steps < s.splits) return fail("a CTA without a step", M, N, K);
                    const uint32_t tile = s.kernel == SMALL_16 ? 16 : s.kernel == SMALL_32 ? 32 : 64;
                    if (tile < 64 && M > tile) return fail("tile does not hold every row", M, N, K);
                    // a cluster whose CTAs wait for one another has to be on the GPU as a whole
                    if (s.splits > 1 && tiles_of(M, N, tile, 128) * s.splits > 2 * LAID_OUT_SMS) return fail("more CTAs than the SMs hold", M, N, K);
                }
    for (int gated = 0; gated < 2; ++gated)
        for (int k = 0; k < 5; ++k)
            if (!chosen[gated][k]) {
                printf("kernel %d is never chosen (gated %d)\n", k, gated);
                return 1;
            }
    if (!few_rows(4, 24576) || few_rows(4, 24577) || few_rows(5, 1) || !few_rows(1, 98304) || few_rows(1, 98305)) return fail("few rows", 0, 0, 0);
    return 0;
}
