// linear_checks_driver.cpp -- the host-side checks and plans of the 8-bit linear
// layer (paper_2608_23048_amd/csrc/checks.cpp) under the host compiler's address
// and undefined-behaviour sanitizers: statuses of edge cases, and for sizes up to
// the largest that a plan covers its work, fits its launch and needs no more
// workspace than it says.  Pointers are fake and never dereferenced.
#include "checks.hpp"

#include <cstdio>

using namespace roi;

static int failures = 0;

static void expect(const char* what, long long got, long long want)
{
    if (got != want) {
        std::printf("FAIL %s: %lld, expected %lld (%s)\n", what, got, want, g_last_error.c_str());
        ++failures;
    }
}

template <typename T>
static T* fake(uintptr_t a) { return reinterpret_cast<T*>(a); }

// Every tile once: `full` whole ones, and the others in `splits` parts of at
// least one step each.
static void check_cut(const Cut& c, int64_t m, int64_t n, int64_t k, int64_t step)
{
    expect("tile", c.tile == 128 || c.tile == 256, 1);
    expect("tm", c.tm, (m + c.tile - 1) / c.tile);
    expect("tn", c.tn, (n + c.tile - 1) / c.tile);
    expect("steps", c.steps, (k + step - 1) / step);
    const int64_t rest = c.tm * c.tn - c.full;
    expect("full", c.full >= 0 && rest >= 0, 1);
    expect("splits", c.splits >= 1 && (c.splits == 1 || c.splits * 2 <= c.steps), 1);
    expect("cut only with parts", (rest > 0) == (c.splits > 1), 1);
    expect("bytes", c.bytes, rest > 0 ? rest * c.splits * c.tile * c.tile * 4 : 0);
    if (rest > 0) expect("parts within a round", rest * c.splits <= 512, 1);
}

int main()
{
    const uintptr_t B = 0x100000000000ull, G = 1ull << 40;
    bool todo;
    auto rows = [&](int dtype, int64_t r, int64_t c, bool out) {
        return validate_rows_i8(fake<void>(B), dtype, fake<const int8_t>(B + G),
                                fake<const float>(B + 2 * G), r, c, out, &todo);
    };
    expect("rows", rows(ROI_BF16, 3, 5, false), ROI_OK);
    expect("todo", todo, 1);
    expect("no columns", rows(ROI_FP32, 3, 0, false), ROI_OK);
    expect("scales to write", todo, 1);
    expect("nothing to restore", rows(ROI_FP32, 3, 0, true), ROI_OK);
    expect("nothing", todo, 0);
    expect("dtype", rows(5, 3, 5, false), ROI_E_INVAL);
    expect("rows < 0", rows(ROI_BF16, -3, 5, false), ROI_E_INVAL);
    expect("rows too many", rows(ROI_BF16, (int64_t)1 << 31, 1, false), ROI_E_UNSUPPORTED);
    expect("largest sizes", check_linear_sizes(((int64_t)1 << 30) - 1, ((int64_t)1 << 22) - 1,
                                               ((int64_t)1 << 22) - 1), ROI_OK);
    expect("tokens", check_linear_sizes((int64_t)1 << 30, 1, 1), ROI_E_UNSUPPORTED);
    expect("rows", check_linear_sizes(1, (int64_t)1 << 22, 1), ROI_E_UNSUPPORTED);
    expect("cols < 0", check_linear_sizes(1, 1, INT64_MIN), ROI_E_INVAL);
    auto linear = [&](int64_t t, int64_t r, int64_t c, bool packed, int64_t bytes, int64_t need) {
        return validate_linear_i8(fake<const int8_t>(B), fake<const float>(B + G),
                                  fake<const int8_t>(B + 2 * G),
                                  packed ? fake<const uint32_t>(B + 3 * G) : nullptr,
                                  fake<const float>(B + 4 * G), nullptr, t, r, c,
                                  fake<const void>(B + 5 * G), ROI_BF16, fake<const void>(B + 6 * G),
                                  bytes, need, &todo);
    };
    expect("linear", linear(3, 5, 131071, false, 0, 0), ROI_OK);
    expect("sum too long", linear(3, 5, 131072, false, 0, 0), ROI_E_UNSUPPORTED);
    expect("packed", linear(3, 5, 96, true, 0, 0), ROI_OK);
    expect("packed odd", linear(3, 5, 100, true, 0, 0), ROI_E_INVAL);
    expect("workspace", linear(3, 5, 96, true, 1023, 1024), ROI_E_INVAL);
    expect("workspace enough", linear(3, 5, 96, true, 1024, 1024), ROI_OK);

    const int64_t sizes[] = {0, 1, 63, 64, 128, 129, 255, 256, 257, 896, 1024, 3584, 4100, 8192,
                             18944, 131071, ((int64_t)1 << 22) - 1};
    for (int64_t m : sizes)
        for (int64_t n : sizes)
            for (int64_t k : sizes) {
                for (int sum_rows = 0; sum_rows < 2; ++sum_rows) {
                    const GradPlan p = plan_grad(m, n, k, sum_rows != 0);
                    const int64_t len = sum_rows ? m : k, dy_rows = sum_rows ? k : m;
                    check_cut(p.cut, m, n, k, 64);
                    expect("grad bytes", p.bytes,
                           p.dy_bytes + p.q_bytes + p.ready_bytes + p.cut.bytes);
                    expect("dy rows", p.dy_row >= len && p.dy_row < len + 64 && p.dy_row % 8 == 0, 1);
                    expect("dy copied", p.dy_bytes,
                           p.dy_row == len ? 0 : (2 * dy_rows * p.dy_row + 255) / 256 * 256);
                    expect("q rows", p.q_row >= n && p.q_row < n + 128 && (p.ready || p.q_row % (p.deep ? 16 : 4) == 0), 1);
                    if (p.deep)
                        expect("deep blocks", p.cut.tile == 128 && p.cut.full + (p.cut.tm * p.cut.tn - p.cut.full) *
                                                  p.cut.splits <= 256, 1);
                    expect("q copied", p.q_bytes,
                           p.q_row == n ? 0 : (k * p.q_row + 255) / 256 * 256);
                    expect("ready bytes", p.ready_bytes,
                           p.ready ? (2 * n * p.ready_k + 255) / 256 * 256 : 0);
                    if (p.ready) {
                        expect("ready tile", p.cut.tile, 256);
                        expect("ready k", p.ready_k >= k && p.ready_k % 64 == 0, 1);
                        expect("ready launch", p.ready_k / 64 * ((n + 127) / 128) < (1 << 24), 1);
                    }
                }
                for (int packed = 0; packed < 2; ++packed) {
                    const LinearPlan l = plan_linear(n, m, k, packed != 0);
                    if (n <= 32) expect("few", l.few, 1);
                    if (n > 1024) expect("many", l.few, 0);
                    if (l.few) continue;
                    check_cut(l.cut, m, n, k, 128);
                    expect("row", l.row >= k && l.row < k + 128 && l.row % 16 == 0, 1);
                    expect("copied", (l.x_bytes > 0) == (l.row != k), 1);
                    expect("linear bytes", l.bytes, l.x_bytes + l.w_bytes + l.cut.bytes);
                    if (l.x_bytes)
                        expect("room", l.x_bytes >= n * l.row && l.w_bytes >= m * l.row, 1);
                }
            }
    // the longest sums and the most tokens
    check_cut(plan_grad(64, 64, ((int64_t)1 << 30) - 1, true).cut, 64, 64, ((int64_t)1 << 30) - 1, 64);
    check_cut(plan_linear(((int64_t)1 << 30) - 1, 16, 64, false).cut, 16, ((int64_t)1 << 30) - 1, 64,
              128);
    const Cut huge = plan_linear(((int64_t)1 << 30) - 1, ((int64_t)1 << 22) - 1, 64, false).cut;
    expect("more blocks than a launch", huge.fits, 0);
    if (failures) return 1;
    std::printf("linear checks ok\n");
    return 0;
}
