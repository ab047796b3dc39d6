// linear_reach_driver.cpp -- every offset that the 256-tile gradient kernel loads
// its int8 operand from (reach.hpp, as the kernel calls it): the steps of a sum and
// the three that are fetched past its end, at row lengths up to the longest.
#include "reach.hpp"

#include <cstdio>
#include <initializer_list>

using namespace roi;

static int failures = 0;

int main()
{
    const int64_t sums[] = {1, 2, 63, 64, 65, 127, 128, 129, 1000, 2100, 4096};
    const int64_t lengths[] = {4, 124, 256, 4096, 18944, ((int64_t)1 << 22) - 4};
    for (int64_t K : sums)
        for (int64_t cols : lengths)
            for (int64_t k0 = 0; k0 < (K + 63) / 64 * 64 + 3 * 64; k0 += 64)
                for (int item = 0; item < 64; ++item)
                    for (int64_t byte : {(int64_t)0, cols - 4, cols, (int64_t)252}) {
                        const bool in_row = byte < cols;
                        const LoadAt at = row_load(item, (int)(K - k0), (uint32_t)byte, in_row,
                                                   (uint32_t)cols);
                        // read: whole words of the operand; else past the buffer's 2^31 - 1
                        // bytes by the lane's offset alone.  The wave's never wraps.
                        const bool read = at.lane != kNowhere;
                        const int64_t end = k0 * cols + at.lane + (int64_t)at.wave + 4;
                        const int64_t row = k0 + item < K ? k0 + item : K - 1;
                        const bool right = at.wave < kNowhere &&
                                           (read ? in_row && k0 < K && end == row * cols + byte + 4
                                                 : !in_row || k0 >= K);
                        if (!right && ++failures <= 10)
                            std::printf("FAIL K %lld cols %lld k0 %lld item %d byte %lld: lane %u wave %u\n",
                                        (long long)K, (long long)cols, (long long)k0, item,
                                        (long long)byte, at.lane, at.wave);
                    }
    if (failures) return 1;
    std::printf("linear reach ok\n");
    return 0;
}
