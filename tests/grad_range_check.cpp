// block_range over outputs and widths up to the widest that a call takes, for every block of 32 by 32 results of every tile that can
// begin in the matrix: never more than what is left of it, and every element that is to be written within it.  Prints the number of blocks.
#include <cstdio>
#include <cstdlib>

#include "star_worker.h"

int main() {
    const int64_t outs[] = {1, 31, 32, 33, 64, 96, 255, 256, 257, 289, 1025, 1056, 2049, 4095};
    const int64_t widths[] = {1, 33, 1000, 65537, 2396745, 2410000, 3000000, (1 << 22) - 1, 1 << 22};
    long blocks = 0;
    for (int64_t out : outs)
        for (int64_t width : widths)
            for (int tile : {64, 128, 256})
                for (int bytes : {2, 4}) {
                    const int64_t all = out * width, rows = (out + tile - 1) / tile * tile, columns = (width + tile - 1) / tile * tile;
                    for (int64_t n = 0; n < rows; n += 32)
                        for (int64_t k : {(int64_t)0, columns - tile, columns - 32}) {
                            const int64_t base = n * width + k;
                            const int range = star::block_range(all, base, bytes);
                            ++blocks;
                            const int64_t left = base < all ? (all - base) * bytes : 0;
                            // the last element that is this block's, and the first that is not: column `width` of the first row
                            const int64_t row = (n + 31 < out ? n + 31 : out - 1) - n, column = (k + 31 < width ? 31 : width - 1 - k);
                            const bool any = row >= 0 && column >= 0;
                            const int64_t end = any ? (row * width + column + 1) * bytes : 0;
                            // the furthest offset a lane forms for a column that is not there (31 rows of 2^22 in fp32 behind kBlockRange) fits an int
                            const int64_t furthest = star::kBlockRange + 31 * width * bytes;
                            if (range < 0 || range > left || range > star::kBlockRange || end > range || furthest > 0x7fffffff) {
                                std::fprintf(stderr, "out %ld width %ld tile %d bytes %d n %ld k %ld: range %d, left %ld, needed %ld\n", (long)out, (long)width, tile,
                                             bytes, (long)n, (long)k, range, (long)left, (long)end);
                                return 1;
                            }
                        }
                }
    std::printf("%ld blocks in range\n", blocks);
    return 0;
}
