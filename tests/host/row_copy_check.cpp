// Walks over the pieces of every row of many small matrices: nothing outside the matrix is read, every byte of a
// row is, and pieces that are copied whole start on 16-byte boundaries.  Exit status 0 if so.
#include <stdint.h>
#include <stdio.h>

#include <vector>

#include "../../paper_2205_03494_b200/csrc/row_copy.h"

int main()
{
    const uintptr_t boundary = 1 << 20;
    long matrices = 0;
    for (uint32_t size = 2; size <= 4; size += 2)
        for (uint32_t offset = 0; offset < 16; offset += size)
            for (uint32_t ld = 1; ld <= 24; ++ld)
                for (uint32_t cols = 1; cols <= ld; ++cols)
                    for (uint32_t rows = 1; rows <= 20; ++rows, ++matrices) {
                        const uintptr_t matrix = boundary + offset, end = matrix + ((rows - 1) * ld + cols) * size;
                        const uint32_t below = omc::rows_from_below(matrix, ld * size);
                        for (uint32_t r = 0; r < rows; ++r) {
                            const uintptr_t row = matrix + r * ld * size, start = row - omc::row_skip(row);
                            std::vector<int> seen(cols * size, 0);
                            const uint32_t skip = omc::row_skip(row), total = skip + cols * size;
                            for (uint32_t k = 0; 16 * k < total; ++k) {
                                const bool single = omc::by_value(k, r < below);
                                if (single && skip == 0) return 1;      // (nothing to leave out)
                                for (uint32_t j = single ? skip : 0; j < 16 && 16 * k + j < total; ++j) {
                                    const uintptr_t at = start + 16 * k + j;
                                    if (at < matrix || at >= end) {
                                        printf("%u-byte values, offset %u, ld %u, cols %u, row %u: reads byte %ld of the matrix\n", size, offset, ld, cols, r,
                                               (long)(at - matrix));
                                        return 2;
                                    }
                                    if (at >= row && at < row + cols * size) ++seen[at - row];
                                }
                            }
                            for (int n : seen)
                                if (n != 1) return 3;
                        }
                    }
    printf("%ld matrices\n", matrices);
    return 0;
}
