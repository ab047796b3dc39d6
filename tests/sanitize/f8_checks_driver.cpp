// f8_checks_driver.cpp -- the host-side checks and plans of the training step in 8-bit
// floats (paper_2608_23048_amd/csrc/checks.cpp) under the host compiler's address and
// undefined-behaviour sanitizers: statuses of edge cases, plans for sizes up to the
// largest, and the way that each call in ways.txt takes (lines "tokens rows cols" in,
// the same with the way behind it out).  Pointers are fake and never dereferenced.
#include "checks.hpp"

#include <cmath>
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

static void check_plan(int64_t tokens, int64_t rows, int64_t cols)
{
    const LinearPlan p = plan_linear_f8(tokens, rows, cols);
    if (p.few) {
        expect("few needs no workspace", p.bytes, 0);
        expect("few or empty", tokens <= 1024 || cols == 0, 1);
        return;
    }
    const Cut& c = p.cut;
    expect("a sum to make", cols > 0, 1);
    expect("tile", c.tile == 128 || c.tile == 256, 1);
    expect("tm", c.tm, (rows + c.tile - 1) / c.tile);
    expect("tn", c.tn, (tokens + c.tile - 1) / c.tile);
    expect("steps", c.steps, (cols + 127) / 128);
    const int64_t rest = c.tm * c.tn - c.full;
    expect("full", c.full >= 0 && rest >= 0, 1);
    expect("splits", c.splits >= 1 && (c.splits == 1 || c.splits * 2 <= c.steps), 1);
    expect("cut only with parts", (rest > 0) == (c.splits > 1), 1);
    expect("bytes", p.bytes, rest > 0 ? rest * c.splits * c.tile * c.tile * 4 : 0);
    if (rest > 0) expect("parts within a round", rest * c.splits <= (c.tile == 256 ? kUnits : 2 * kUnits), 1);
    expect("time", std::isfinite(c.us) && c.us > 0, 1);
}

static void print_ways()
{
    std::FILE* f = std::fopen("ways.txt", "r");
    if (!f) return;
    long long t, r, c;
    while (std::fscanf(f, "%lld %lld %lld", &t, &r, &c) == 3) {
        std::printf("%lld %lld %lld: ", t, r, c);
        const LinearPlan p = plan_linear_f8(t, r, c);
        if (p.few) {
            std::printf("few\n");
            continue;
        }
        const long long rest = p.cut.tm * p.cut.tn - p.cut.full, blocks = p.cut.full + rest * p.cut.splits;
        const long long round = p.cut.tile == 256 ? kUnits : 2 * kUnits;
        std::printf("%d%s%s%s%s\n", p.cut.tile, p.cut.tile == 128 && blocks <= kUnits ? " alone" : "",
                    p.cut.full > 0 ? " whole" : "", rest > 0 ? " cut" : "", blocks > round ? " rounds" : "");
    }
    std::fclose(f);
}

int main()
{
    const uintptr_t B = 0x100000000000ull, G = 1ull << 42;
    bool todo;
    const int64_t most = (int64_t)1 << 31;
    auto quantize = [&](int64_t r, int64_t c, bool square, int64_t stride, bool t, int64_t stride_t) {
        return validate_quantize_f8(fake<void>(B), ROI_FP32, r, c, square, ROI_E4M3, fake<uint8_t>(B + G),
                                    stride, fake<uint8_t>(B + 2 * G), t ? fake<uint8_t>(B + 3 * G) : nullptr,
                                    stride_t, t ? fake<uint8_t>(B + 4 * G) : nullptr, &todo);
    };
    expect("quantize", quantize(3, 5, false, 16, true, 16), ROI_OK);
    expect("todo", todo, 1);
    expect("no columns", quantize(3, 0, true, 0, false, 0), ROI_OK);
    expect("nothing", todo, 0);
    expect("longest row", quantize(1, most - 1, false, most, false, 0), ROI_OK);
    expect("most rows", quantize(most - 1, 1, true, 16, true, most), ROI_OK);
    expect("rows", quantize(most, 1, false, 16, false, 0), ROI_E_UNSUPPORTED);
    expect("cols", quantize(1, INT64_MIN, false, 16, false, 0), ROI_E_INVAL);
    expect("stride", quantize(1, 1, false, INT64_MAX - 15, false, 0), ROI_E_UNSUPPORTED);
    expect("stride < 0", quantize(2, 1, false, INT64_MIN, false, 0), ROI_E_INVAL);
    expect("stride_t short", quantize(17, 5, false, 16, true, 16), ROI_E_INVAL);
    // the whole of two largest sides overlaps everything
    expect("both", quantize(most - 1, most - 1, false, most, false, 0), ROI_E_INVAL);

    auto restore = [&](int64_t r, int64_t c, bool square, int64_t stride) {
        return validate_dequantize_f8(fake<uint8_t>(B), stride, fake<uint8_t>(B + G), r, c, square, ROI_E5M2,
                                      fake<void>(B + 2 * G), ROI_BF16, &todo);
    };
    expect("restore", restore(300, 77, true, 80), ROI_OK);
    expect("longest", restore(1, most - 1, false, most), ROI_OK);
    expect("restore stride", restore(2, 77, false, 88), ROI_E_INVAL);

    auto linear = [&](int64_t t, int64_t r, int64_t c, int64_t xs, int64_t ws, int64_t bytes, int64_t need) {
        return validate_linear_f8(fake<uint8_t>(B), xs, fake<uint8_t>(B + G), ROI_E4M3, fake<uint8_t>(B + 2 * G),
                                  ws, fake<uint8_t>(B + 3 * G), true, nullptr, t, r, c, fake<uint16_t>(B + 4 * G),
                                  fake<void>(B + 6 * G), bytes, need, &todo);
    };
    expect("linear", linear(3, 5, 7, 16, 32, 0, 0), ROI_OK);
    expect("widest", linear(3, 5, kMaxLinearDim - 1, kMaxStride, kMaxStride, 0, 0), ROI_OK);
    expect("no sum", linear(3, 5, 0, 0, 0, 0, 0), ROI_OK);
    expect("its result", todo, 1);
    expect("no tokens", linear(0, 5, 7, 16, 16, 0, 0), ROI_OK);
    expect("no result", todo, 0);
    expect("too wide", linear(3, 5, 7, kMaxStride + 16, 16, 0, 0), ROI_E_UNSUPPORTED);
    expect("workspace", linear(3, 5, 7, 16, 16, 1023, 1024), ROI_E_INVAL);

    roi_step_params opt{};
    opt.lr = 1e-3;
    opt.beta1 = 0.9;
    opt.beta2 = 0.999;
    opt.eps = 1e-8;
    opt.t = 1;
    AdamStep step;
    auto adamw = [&](int64_t numel, uint64_t offset, const roi_step_params& o) {
        const roi_step_tensor t{fake<float>(B),           fake<void>(B + 4 * G),     fake<void>(B + 8 * G),
                                fake<void>(B + 12 * G),   fake<uint8_t>(B + 13 * G), fake<uint8_t>(B + 14 * G),
                                numel, offset};
        return validate_step(&t, 1, ROI_FP32, 8, &o, &step, &todo);
    };
    expect("step", adamw(5, 0, opt), ROI_OK);
    expect("largest", adamw(kMaxStepValues - 1, 0, opt), ROI_OK);
    expect("too large", adamw(kMaxStepValues, 0, opt), ROI_E_UNSUPPORTED);
    expect("last offset", adamw(3, UINT64_MAX - 3, opt), ROI_OK);
    expect("past it", adamw(4, UINT64_MAX - 3, opt), ROI_E_INVAL);
    expect("empty", adamw(0, 0, opt), ROI_OK);
    expect("nothing to step", todo, 0);
    roi_step_params late = opt;
    late.t = INT64_MAX;
    expect("late", adamw(5, 0, late), ROI_OK);
    expect("corrected", step.inv_sqrt_bc2 == 1.0f, 1);
    late.beta1 = std::nan("");
    expect("nan", adamw(5, 0, late), ROI_E_INVAL);

    const int64_t sizes[] = {0, 1, 16, 31, 33, 128, 129, 256, 257, 896, 1024, 1025, 3584, 4100, 8192,
                             18944, 131071, kMaxLinearDim - 1};
    for (int64_t t : sizes)
        for (int64_t r : sizes)
            for (int64_t c : sizes) check_plan(t, r, c);
    check_plan(kMaxTokens - 1, 16, 64);
    expect("blocks in 32 bits", plan_linear_f8(kMaxTokens - 1, kMaxLinearDim - 1, 64).cut.fits, 0);
    expect("a launch's threads", plan_linear_f8(kMaxTokens - 1, 1, 0).cut.fits, 0);
    expect("few fit", plan_linear_f8(1024, kMaxLinearDim - 1, 0).cut.fits, 1);
    print_ways();
    if (failures) return 1;
    std::printf("f8 checks ok\n");
    return 0;
}
