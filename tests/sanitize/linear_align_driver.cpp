// linear_align_driver.cpp -- which alignments the calls of the 8-bit linear layer
// take (paper_2608_23048_amd/csrc/checks.cpp): scales that a product or a gradient
// reads may start at any of their rows, everything else at 16 bytes.  Pointers are
// fake and never dereferenced.
#include "checks.hpp"

#include <cstdio>
#include <initializer_list>

using namespace roi;

static int failures = 0;

static void expect(const char* what, int offset, long long got, long long want)
{
    if (got != want) {
        std::printf("FAIL %s + %d: %lld, expected %lld (%s)\n", what, offset, got, want,
                    g_last_error.c_str());
        ++failures;
    }
}

template <typename T>
static T* fake(uintptr_t a) { return reinterpret_cast<T*>(a); }

int main()
{
    const uintptr_t B = 0x100000000000ull, G = 1ull << 40;
    const char* const linear[] = {"xq", "xs", "wq", "meta", "ws", "bias", "y", "workspace"};
    const char* const grad[] = {"grad_y", "q", "scale", "out", "workspace"};
    for (int offset : {0, 1, 2, 4, 8, 12, 16, 20}) {
        bool todo;
        for (int which = 0; which < 8; ++which) {
            uintptr_t p[8];
            for (int i = 0; i < 8; ++i) p[i] = B + (uintptr_t)i * G + (uintptr_t)(i == which ? offset : 0);
            const bool scales = which == 1 || which == 4;
            expect(linear[which], offset,
                   validate_linear_i8(fake<const int8_t>(p[0]), fake<const float>(p[1]),
                                      fake<const int8_t>(p[2]), fake<const uint32_t>(p[3]),
                                      fake<const float>(p[4]), fake<const uint16_t>(p[5]), 40, 8, 64,
                                      fake<const void>(p[6]), ROI_BF16, fake<const void>(p[7]), 64, 64,
                                      &todo),
                   offset % (scales ? 4 : 16) ? ROI_E_INVAL : ROI_OK);
        }
        for (int which = 0; which < 5; ++which) {
            uintptr_t p[5];
            for (int i = 0; i < 5; ++i) p[i] = B + (uintptr_t)i * G + (uintptr_t)(i == which ? offset : 0);
            expect(grad[which], offset,
                   validate_grad_i8(fake<const uint16_t>(p[0]), fake<const int8_t>(p[1]),
                                    fake<const float>(p[2]), 40, 40, 8, 64, fake<const uint16_t>(p[3]), 8,
                                    fake<const void>(p[4]), 64, 64, &todo),
                   offset % (which == 2 ? 4 : 16) ? ROI_E_INVAL : ROI_OK);
        }
    }
    if (failures) return 1;
    std::printf("linear alignments ok\n");
    return 0;
}
