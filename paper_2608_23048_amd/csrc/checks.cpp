// checks.cpp -- the host-side argument checks of the C ABI (checks.hpp).
#include "checks.hpp"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>

namespace roi {

thread_local std::string g_last_error;

int fail(int status, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_last_error = buf;
    return status;
}

int ok()
{
    g_last_error.clear();
    return ROI_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb)
{
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + nb && b0 < a0 + na;
}

// Sorted by start, a range overlaps an earlier one exactly when it starts
// before the largest end seen so far (of any range, for an output; of the
// outputs, for an input).
int check_overlaps(std::vector<Range>& r)
{
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.p < b.p; });
    uintptr_t end_any = 0, end_out = 0;
    for (const Range& x : r) {
        if (x.out ? x.p < end_any : x.p < end_out)
            return fail(ROI_E_INVAL, "an output overlaps another input or output");
        end_any = std::max(end_any, x.p + x.n);
        if (x.out) end_out = std::max(end_out, x.p + x.n);
    }
    return ROI_OK;
}

void add_range(std::vector<Range>& r, const void* p, size_t n, bool out)
{
    if (p && n) r.push_back({(uintptr_t)p, n, out});
}

int check_common(int n, int m, float tau, float lambda)
{
    if (m < 1 || n < 1 || n > m)
        return fail(ROI_E_INVAL, "pattern n:m = %d:%d needs 1 <= n <= m", n, m);
    if (m != 4 && m != 8 && m != 16 && m != 32)
        return fail(ROI_E_UNSUPPORTED, "m = %d is not built (supported: 4, 8, 16, 32)", m);
    if (!(tau > 0.0f) || !std::isfinite(tau))
        return fail(ROI_E_INVAL, "tau must be finite and > 0");
    if (!(lambda > 0.0f) || !std::isfinite(lambda))
        return fail(ROI_E_INVAL, "lambda must be finite and > 0");
    return ROI_OK;
}

int check_shape(int64_t rows, int64_t cols, int n, int m, float tau, float lambda,
                uint64_t elem_offset, Shape* sh)
{
    if (rows < 0 || cols < 0) return fail(ROI_E_INVAL, "rows (%lld) and cols (%lld) must be >= 0",
                                          (long long)rows, (long long)cols);
    if (int st = check_common(n, m, tau, lambda)) return st;
    if (cols % m != 0) return fail(ROI_E_INVAL, "cols (%lld) must be a multiple of m (%d)",
                                   (long long)cols, m);
    // rows * cols >= 2^62 exactly when cols > (2^62 - 1) / rows (integer division);
    // below it, the byte sizes of fp32 arrays (4 rows cols) fit in 64 bits
    if (rows > 0 && cols > (((int64_t)1 << 62) - 1) / rows)
        return fail(ROI_E_INVAL, "rows * cols must be below 2^62");
    if (elem_offset % (uint64_t)m != 0)
        return fail(ROI_E_INVAL, "elem_offset (%llu) must be a multiple of m (%d)",
                    (unsigned long long)elem_offset, m);
    const int64_t numel = rows * cols;
    if (elem_offset > UINT64_MAX - (uint64_t)numel)
        return fail(ROI_E_INVAL, "elem_offset + rows * cols overflows 64 bits");
    sh->numel = numel;
    sh->ngroups = numel / m;
    return ROI_OK;
}

int check_count(const void* t, int count)
{
    if (count < 0) return fail(ROI_E_INVAL, "count must be >= 0");
    if (count > 0 && !t) return fail(ROI_E_INVAL, "tensors must not be NULL");
    return ROI_OK;
}

namespace {

// Params: roi_adamw_params or roi_step_params.
template <typename Params>
int fold_adamw(const Params* o, AdamStep* st)
{
    if (!o) return fail(ROI_E_INVAL, "the AdamW parameters must not be NULL");
    // in fp32, which the step is taken in
    if (!(o->lr >= 0) || !std::isfinite((float)o->lr))
        return fail(ROI_E_INVAL, "AdamW lr must be finite and >= 0");
    if (!(o->beta1 >= 0 && o->beta1 < 1) || !(o->beta2 >= 0 && o->beta2 < 1))
        return fail(ROI_E_INVAL, "AdamW betas must lie in [0, 1)");
    if (!((float)o->eps > 0) || !std::isfinite((float)o->eps))
        return fail(ROI_E_INVAL, "AdamW eps must be finite and > 0");
    if (!(o->weight_decay >= 0) || !std::isfinite((float)o->weight_decay))
        return fail(ROI_E_INVAL, "AdamW weight_decay must be finite and >= 0");
    if (o->t < 1) return fail(ROI_E_INVAL, "AdamW step count t must be >= 1");
    const double lr = o->lr, b1 = o->beta1, b2 = o->beta2;
    const double bc1 = 1.0 - std::pow(b1, (double)o->t);
    const double bc2 = 1.0 - std::pow(b2, (double)o->t);
    st->decay = (float)(1.0 - lr * (double)o->weight_decay);
    st->beta1 = (float)b1;
    st->beta2 = (float)b2;
    st->one_m_beta1 = (float)(1.0 - b1);
    st->one_m_beta2 = (float)(1.0 - b2);
    st->step_size = (float)(lr / bc1);
    st->inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    st->eps = (float)o->eps;
    return ROI_OK;
}

} // namespace

int check_adamw(const roi_adamw_params* o, AdamStep* st) { return fold_adamw(o, st); }

int validate_fwd(const roi_fwd_tensor* t, int count, int n, int m, float tau, float lambda,
                 int* with_s, int* with_idx)
{
    *with_s = *with_idx = -1; // -1: no nonempty tensor seen yet
    if (int st = check_common(n, m, tau, lambda)) return st;
    if (int st = check_count(t, count)) return st;
    std::vector<Range> ranges;
    for (int i = 0; i < count; ++i) {
        Shape sh;
        if (int st = check_shape(t[i].rows, t[i].cols, n, m, tau, lambda, t[i].elem_offset, &sh))
            return count > 1 ? fail(st, "tensor %d: %s", i, g_last_error.c_str()) : st;
        if (sh.numel == 0) continue;
        if (!t[i].W || !t[i].logits || !t[i].W_masked)
            return fail(ROI_E_INVAL, "tensor %d: W, logits and W_masked must not be NULL", i);
        if (!aligned16(t[i].W) || !aligned16(t[i].logits) || !aligned16(t[i].W_masked) ||
            (t[i].soft_mask && !aligned16(t[i].soft_mask)) ||
            (t[i].sel_idx && !aligned16(t[i].sel_idx)))
            return fail(ROI_E_INVAL, "tensor %d: device pointers must be 16-byte aligned", i);
        const int s_i = t[i].soft_mask != nullptr, x_i = t[i].sel_idx != nullptr;
        if ((*with_s >= 0 && s_i != *with_s) || (*with_idx >= 0 && x_i != *with_idx))
            return fail(ROI_E_INVAL,
                        "soft_mask and sel_idx must each be given for every tensor or for none");
        *with_s = s_i;
        *with_idx = x_i;
        const size_t nb2 = (size_t)sh.numel * 2, nb4 = (size_t)sh.numel * 4;
        add_range(ranges, t[i].W, nb2, false);
        add_range(ranges, t[i].logits, nb4, false);
        add_range(ranges, t[i].W_masked, nb2, true);
        add_range(ranges, t[i].soft_mask, nb4, true);
        add_range(ranges, t[i].sel_idx, (size_t)sh.ngroups * (size_t)n, true);
    }
    if (*with_s < 0) return ok(); // nothing to do
    if (int st = check_overlaps(ranges)) return st;
    return ok();
}

int validate_bwd(const BwdDesc* t, int count, int n, int m, float tau, float lambda,
                 const roi_adamw_params* opt, AdamStep* astep, bool* any)
{
    *any = false;
    if (int st = check_common(n, m, tau, lambda)) return st;
    const bool adam = opt != nullptr;
    if (adam)
        if (int st = check_adamw(opt, astep)) return st;
    if (int st = check_count(t, count)) return st;
    std::vector<Range> ranges;
    for (int i = 0; i < count; ++i) {
        Shape sh;
        if (int st = check_shape(t[i].rows, t[i].cols, n, m, tau, lambda, t[i].off, &sh))
            return count > 1 ? fail(st, "tensor %d: %s", i, g_last_error.c_str()) : st;
        if (sh.numel == 0) continue;
        if (!t[i].G || !t[i].W || !t[i].phi || (!adam && !t[i].dphi) ||
            (adam && (!t[i].m || !t[i].v)))
            return fail(ROI_E_INVAL, adam ? "tensor %d: grad_W_masked, W, logits, exp_avg and "
                                            "exp_avg_sq must not be NULL"
                                          : "tensor %d: grad_W_masked, W, logits and grad_logits "
                                            "must not be NULL", i);
        if (!aligned16(t[i].G) || !aligned16(t[i].W) || !aligned16(t[i].phi) ||
            (t[i].dphi && !aligned16(t[i].dphi)) || (t[i].m && !aligned16(t[i].m)) ||
            (t[i].v && !aligned16(t[i].v)))
            return fail(ROI_E_INVAL, "tensor %d: device pointers must be 16-byte aligned", i);
        const size_t nb2 = (size_t)sh.numel * 2, nb4 = (size_t)sh.numel * 4;
        add_range(ranges, t[i].G, nb2, false);
        add_range(ranges, t[i].W, nb2, false);
        add_range(ranges, t[i].phi, nb4, adam); // updated in place by the AdamW step
        add_range(ranges, t[i].dphi, nb4, true);
        if (adam) {
            add_range(ranges, t[i].m, nb4, true);
            add_range(ranges, t[i].v, nb4, true);
        }
        *any = true;
    }
    if (!*any) return ok();
    if (int st = check_overlaps(ranges)) return st;
    return ok();
}

int validate_cat(bool fwd, const uint16_t* W, const float* alpha, const uint16_t* G, int64_t rows,
                 int64_t cols, int n, int m, float tau, float lambda, uint64_t group_offset,
                 const uint16_t* W_masked, const float* S, const uint8_t* choice,
                 const float* dalpha, int64_t* ngroups_out, int* C_out)
{
    *ngroups_out = 0;
    *C_out = 0;
    if (rows < 0 || cols < 0) return fail(ROI_E_INVAL, "rows and cols must be >= 0");
    if (m < 1 || n < 1 || n > m)
        return fail(ROI_E_INVAL, "pattern n:m = %d:%d needs 1 <= n <= m", n, m);
    if (m != 4 && m != 8)
        return fail(ROI_E_UNSUPPORTED, "the categorical sampler is built for m = 4 and 8");
    if (cols % m != 0) return fail(ROI_E_INVAL, "cols must be a multiple of m");
    if (rows > 0 && cols > (((int64_t)1 << 62) - 1) / rows)
        return fail(ROI_E_INVAL, "rows * cols must be below 2^62");
    if (!(tau > 0.0f) || !std::isfinite(tau)) return fail(ROI_E_INVAL, "tau must be finite, > 0");
    if (!(lambda > 0.0f) || !std::isfinite(lambda))
        return fail(ROI_E_INVAL, "lambda must be finite and > 0");
    int C = 1; // binom(m, n)
    for (int k = 1; k <= n; ++k) C = C * (m - n + k) / k;
    const int64_t ngroups = rows * cols / m;
    // the logits and their gradient hold 4 C bytes per group
    if (ngroups > ((int64_t)1 << 62) / (4 * (int64_t)C))
        return fail(ROI_E_INVAL, "the %d logits per group of %lld groups exceed 2^62 bytes", C,
                    (long long)ngroups);
    const uint64_t B = (uint64_t)(C + 3) / 4;
    if (ngroups > 0 && group_offset > (UINT64_MAX / (4 * B)) - (uint64_t)ngroups)
        return fail(ROI_E_INVAL, "group_offset + groups overflows the noise index space");
    *ngroups_out = ngroups;
    *C_out = C;
    if (ngroups == 0) return ok();
    if (!W || !alpha || (fwd ? !W_masked : (!G || !dalpha)))
        return fail(ROI_E_INVAL, "a required pointer is NULL");
    const void* ptrs[] = {W, alpha, G, W_masked, S, choice, dalpha};
    for (const void* p : ptrs)
        if (p && !aligned16(p)) return fail(ROI_E_INVAL, "device pointers must be 16-byte aligned");
    const size_t numel = (size_t)ngroups * (size_t)m, nc = (size_t)ngroups * (size_t)C;
    std::vector<Range> r;
    add_range(r, W, numel * 2, false);
    add_range(r, alpha, nc * 4, false);
    add_range(r, G, numel * 2, false);
    add_range(r, W_masked, numel * 2, true);
    add_range(r, S, numel * 4, true);
    add_range(r, choice, (size_t)ngroups, true);
    add_range(r, dalpha, nc * 4, true);
    if (int st = check_overlaps(r)) return st;
    return ok();
}

namespace {

struct Buffer {
    const void* p;
    size_t n;
    bool out;
    unsigned align = 16;
};

// The products and gradients read scales one by one: those of a batch cut at any
// token serve.
constexpr unsigned kScaleAlign = 4;

// Present, aligned, and no output over anything else (an empty buffer's
// pointer is not looked at).
int check_buffers(const Buffer* b, int count)
{
    for (int i = 0; i < count; ++i) {
        if (b[i].n == 0) continue;
        if (!b[i].p) return fail(ROI_E_INVAL, "a required pointer is NULL");
        if ((uintptr_t)b[i].p % b[i].align)
            return fail(ROI_E_INVAL, "device pointers must be 16-byte aligned%s",
                        b[i].align < 16 ? " (scales: to their 4 bytes)" : "");
    }
    for (int i = 0; i < count; ++i)
        for (int j = i + 1; j < count; ++j)
            if ((b[i].out || b[j].out) && overlap(b[i].p, b[i].n, b[j].p, b[j].n))
                return fail(ROI_E_INVAL, "an output overlaps another input or output");
    return ROI_OK;
}

int check_workspace(const void* workspace, int64_t bytes, int64_t need)
{
    if (bytes < 0) return fail(ROI_E_INVAL, "workspace_bytes must be >= 0");
    if (bytes < need)
        return fail(ROI_E_INVAL, "the workspace has %lld bytes, %lld are needed", (long long)bytes,
                    (long long)need);
    if (need > 0 && !workspace) return fail(ROI_E_INVAL, "the workspace must not be NULL");
    return ROI_OK;
}

int check_dtype(int dtype)
{
    if (dtype != ROI_BF16 && dtype != ROI_FP32)
        return fail(ROI_E_INVAL, "dtype must be ROI_BF16 or ROI_FP32 (got %d)", dtype);
    return ROI_OK;
}

} // namespace

int validate_rows_i8(const void* x, int dtype, const int8_t* q, const float* scale, int64_t rows,
                     int64_t cols, bool x_out, bool* todo)
{
    *todo = false;
    if (int st = check_dtype(dtype)) return st;
    if (rows < 0 || cols < 0)
        return fail(ROI_E_INVAL, "rows (%lld) and cols (%lld) must be >= 0", (long long)rows,
                    (long long)cols);
    if (rows >= kMaxRowsI8 || cols >= kMaxRowsI8)
        return fail(ROI_E_UNSUPPORTED, "rows and cols must be below 2^31");
    const size_t n = (size_t)rows * (size_t)cols; // below 2^62
    const Buffer b[] = {{x, n * (dtype == ROI_FP32 ? 4 : 2), x_out},
                        {q, n, !x_out},
                        {scale, (size_t)rows * 4, !x_out}};
    if (int st = check_buffers(b, 3)) return st;
    *todo = x_out ? n > 0 : rows > 0;
    return ok();
}

int check_linear_sizes(int64_t tokens, int64_t rows, int64_t cols)
{
    if (tokens < 0 || rows < 0 || cols < 0)
        return fail(ROI_E_INVAL, "tokens (%lld), rows (%lld) and cols (%lld) must be >= 0",
                    (long long)tokens, (long long)rows, (long long)cols);
    if (tokens >= kMaxTokens || rows >= kMaxLinearDim || cols >= kMaxLinearDim)
        return fail(ROI_E_UNSUPPORTED, "tokens must be below 2^30, rows and cols below 2^22");
    return ROI_OK;
}

int check_linear_sum(int64_t cols, bool packed)
{
    if (cols > kMaxI8Sum)
        return fail(ROI_E_UNSUPPORTED, "cols (%lld) must be at most %lld for an exact int32 sum",
                    (long long)cols, (long long)kMaxI8Sum);
    if (packed && cols % 32 != 0)
        return fail(ROI_E_INVAL, "2:4 weights need cols %% 32 == 0 (got %lld)", (long long)cols);
    return ROI_OK;
}

namespace {

constexpr int64_t kMostSplits = 64;
constexpr double kPartBytesPerUs = 6.0e6; // of parts, written and read again
constexpr double kSumLaunchUs = 6.5;
constexpr double kSumPartUs = 0.06;       // of a sum, for each of its parts

// One tile size: the tiles of whole rounds over the units are whole.  The last
// round's are cut where that is expected to take less time, into as many parts
// as do: more parts have fewer steps each, fewer have fewer bytes to pass on.
Cut cut_tiles(int64_t m, int64_t n, int64_t k, int64_t step, int tile, const TileCost& cost)
{
    Cut c{};
    c.tile = tile;
    c.tm = (m + tile - 1) / tile;
    c.tn = (n + tile - 1) / tile;
    c.steps = (k + step - 1) / step;
    const int64_t tiles = c.tm * c.tn, slots = kUnits * (tile == 256 ? 1 : 2);
    const double rest_us = tile == 256 ? cost.rest256 : cost.rest128;
    // of a round of so many blocks, each of so many steps
    auto round = [&](int64_t blocks, int64_t steps) {
        const double one = tile == 256 ? cost.step256 : blocks > kUnits ? cost.two128 : cost.step128;
        return (double)steps * one + rest_us;
    };
    const int64_t rest = tiles % slots;
    const double rounds = (double)(tiles / slots) * round(slots, c.steps);
    c.full = tiles;
    c.splits = 1;
    c.us = rounds + (rest ? round(rest, c.steps) : 0);
    // a part of a sum has two steps at least
    const int64_t most = rest ? std::min(std::min(slots / rest, c.steps / 2), kMostSplits) : 0;
    for (int64_t splits = 2; splits <= most; ++splits) {
        const int64_t bytes = rest * splits * tile * tile * 4;
        const double us = rounds + round(rest * splits, (c.steps + splits - 1) / splits) +
                          (double)bytes / kPartBytesPerUs + kSumLaunchUs + kSumPartUs * (double)splits;
        if (us < c.us) {
            c.us = us;
            c.full = tiles - rest;
            c.splits = splits;
            c.bytes = bytes;
        }
    }
    // a launch has fewer than 2^32 threads
    c.fits = (c.full + rest * c.splits) * (tile == 256 ? 512 : 256) < ((int64_t)1 << 32);
    return c;
}

} // namespace

Cut cut_product(int64_t m, int64_t n, int64_t k, int64_t step, const TileCost& cost)
{
    const Cut big = cut_tiles(m, n, k, step, 256, cost);
    const Cut small = cut_tiles(m, n, k, step, 128, cost);
    return small.us < big.us && small.fits ? small : big;
}

namespace {

// Of a copy of rows into the workspace: bytes read and written.
double copy_us(double bytes) { return 2 + bytes / 4.0e6; }

// The length of copied rows: what a tile loads of a row is then one cache line.
int64_t whole_lines(int64_t bytes) { return (bytes + 127) / 128 * 128; }

// The streaming kernel's expected time: it takes 32 tokens at a time, the first
// with the weight from memory, the others from the caches, in blocks of 32 or 16
// rows of which 512 (256 at 2:4) run at once.  Fitted to 40 to 512 tokens through
// ten weights: 64 tokens through 3584 x 3584 take 5.6 us so and 14.7 in tiles,
// through 18944 x 3584 26 and 20; 128 tokens 8.3 and 14.8, 44 and 23.
double few_us(int64_t tokens, int64_t rows, int64_t cols, bool packed)
{
    const int64_t groups = (tokens + 31) / 32;
    const double blocks = (double)((rows + 31) / 32) * (double)groups;
    const double weight = (double)rows * (double)cols;
    const double first = packed ? 8.0e6 : 5.0e6, again = packed ? 10.0e6 : 8.0e6;
    if (cols % 16) return 3.5 + (double)groups * weight / 2.5e6;
    return 2.2 + blocks * (packed ? 1.77 / 256 : 1.5 / 512) + weight / first +
           (double)(groups - 1) * weight / again;
}

} // namespace

LinearPlan plan_linear(int64_t tokens, int64_t rows, int64_t cols, bool packed)
{
    LinearPlan p{};
    p.few = tokens <= 32;
    if (p.few) return p;
    const TileCost& cost = packed ? kPackedCost : kLinearCost;
    p.cut = cut_product(rows, tokens, cols, 128, cost);
    p.row = cols % 16 == 0 ? cols : whole_lines(cols);
    double tiles_us = p.cut.us;
    // few tiles: their steps may be less work than reading the weight
    if (tokens <= 128)
        tiles_us += std::max(0.0, (double)rows * (double)cols * (packed ? 0.625 : 1) / 5.0e6 -
                                      (double)(p.cut.steps / p.cut.splits) * cost.step128);
    if (p.row != cols) {
        p.x_bytes = padded256(tokens * p.row);
        p.w_bytes = padded256(rows * p.row);
        tiles_us += copy_us(2.0 * (double)(tokens + rows) * (double)cols);
    }
    p.bytes = p.x_bytes + p.w_bytes + p.cut.bytes;
    p.few = tokens <= 1024 && few_us(tokens, rows, cols, packed) < tiles_us;
    return p;
}

GradPlan plan_grad(int64_t m, int64_t n, int64_t k, bool sum_rows)
{
    constexpr int64_t kStep = 64;
    GradPlan p{};
    p.cut = cut_product(m, n, k, kStep, kGradCost);
    const int64_t dy_len = sum_rows ? m : k, dy_rows = sum_rows ? k : m;
    p.dy_row = dy_len % 8 == 0 ? dy_len : whole_lines(2 * dy_len) / 2;
    if (p.dy_row != dy_len) p.dy_bytes = padded256(2 * dy_rows * p.dy_row);
    const int64_t ready_k = (k + kStep - 1) / kStep * kStep;
    // offsets within a tile of the transposed operand stay below 2^31, and the
    // pass that writes it has fewer than 2^32 threads (256 for 64 x 128 elements)
    if (m > 0 && n > 0 && k > 0 && k <= ((int64_t)1 << 21) &&
        ready_k / 64 * ((n + 127) / 128) < (int64_t)1 << 24) {
        const Cut c = cut_tiles(m, n, k, kStep, 256, kReadyCost);
        const double us = c.us + 3 + 3 * (double)ready_k * (double)n / 4.0e6;
        const double fused_us = p.cut.us + (n % 16 ? copy_us(2.0 * (double)k * (double)n) : 0);
        if (us < fused_us && c.fits) {
            p.ready = true;
            p.ready_k = ready_k;
            p.ready_bytes = padded256(2 * n * ready_k);
            p.cut = c;
        }
    }
    const Cut& c = p.cut;
    p.deep = !p.ready && c.tile == 128 && c.full + (c.tm * c.tn - c.full) * c.splits <= kUnits;
    p.q_row = n;
    if (!p.ready && n % (p.deep ? 16 : 4)) {
        p.q_row = whole_lines(n);
        p.q_bytes = padded256(k * p.q_row);
    }
    p.bytes = p.dy_bytes + p.q_bytes + p.ready_bytes + p.cut.bytes;
    return p;
}

int validate_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq, const uint32_t* meta,
                       const float* ws, const uint16_t* bias, int64_t tokens, int64_t rows,
                       int64_t cols, const void* y, int dtype, const void* workspace,
                       int64_t workspace_bytes, int64_t need, bool* todo)
{
    *todo = false;
    if (int st = check_dtype(dtype)) return st;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    if (int st = check_linear_sum(cols, meta != nullptr)) return st;
    if (int st = check_workspace(workspace, workspace_bytes, need)) return st;
    const size_t t = (size_t)tokens, r = (size_t)rows, c = (size_t)cols;
    const Buffer b[] = {{xq, t * c, false},
                        {xs, t * 4, false, kScaleAlign},
                        {wq, meta ? r * (c / 2) : r * c, false},
                        {meta, meta ? r * (c / 32) * 4 : 0, false},
                        {ws, r * 4, false, kScaleAlign},
                        {bias, bias ? r * 2 : 0, false},
                        {y, t * r * (dtype == ROI_FP32 ? 4 : 2), true},
                        {workspace, (size_t)need, true}};
    if (int st = check_buffers(b, 8)) return st;
    *todo = tokens > 0 && rows > 0;
    return ok();
}

int validate_grad_i8(const uint16_t* grad_y, const int8_t* q, const float* scale, int64_t krows,
                     int64_t tokens, int64_t rows, int64_t cols, const uint16_t* out,
                     int64_t out_rows, const void* workspace, int64_t workspace_bytes,
                     int64_t need, bool* todo)
{
    *todo = false;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    if (int st = check_workspace(workspace, workspace_bytes, need)) return st;
    const size_t c = (size_t)cols;
    const Buffer b[] = {{grad_y, (size_t)tokens * (size_t)rows * 2, false},
                        {q, (size_t)krows * c, false},
                        {scale, (size_t)krows * 4, false, kScaleAlign},
                        {out, (size_t)out_rows * c * 2, true},
                        {workspace, (size_t)need, true}};
    if (int st = check_buffers(b, 5)) return st;
    *todo = out_rows > 0 && cols > 0;
    return ok();
}

namespace {

constexpr int64_t scale_bytes(int64_t cols) { return (cols + 511) / 512 * 4; }

// Rows of 8-bit values, `stride` bytes apart: the bytes from the first to the last.
size_t f8_bytes(int64_t rows, int64_t cols, int64_t stride)
{
    return rows > 0 && cols > 0 ? (size_t)(rows - 1) * (size_t)stride + (size_t)cols : 0;
}
size_t f8_scales(int64_t rows, int64_t cols, bool square)
{
    return (size_t)(square ? (rows + 127) / 128 : rows) * (size_t)scale_bytes(cols);
}

int check_stride(const char* what, int64_t stride, int64_t cols, int64_t most)
{
    if (stride % 16 != 0 || stride < cols)
        return fail(ROI_E_INVAL, "%s (%lld) must be a multiple of 16 and at least %lld", what,
                    (long long)stride, (long long)cols);
    if (stride > most)
        return fail(ROI_E_UNSUPPORTED, "%s (%lld) must be at most %lld", what, (long long)stride,
                    (long long)most);
    return ROI_OK;
}

int check_format(int format)
{
    if (format != ROI_E4M3 && format != ROI_E5M2)
        return fail(ROI_E_INVAL, "the format must be ROI_E4M3 or ROI_E5M2 (got %d)", format);
    return ROI_OK;
}

int check_f8_sizes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0)
        return fail(ROI_E_INVAL, "rows (%lld) and cols (%lld) must be >= 0", (long long)rows,
                    (long long)cols);
    if (rows >= kMaxRowsI8 || cols >= kMaxRowsI8)
        return fail(ROI_E_UNSUPPORTED, "rows and cols must be below 2^31");
    return ROI_OK;
}

} // namespace

namespace {

// The 8-bit floats' tiles, which a block goes through without a pause: microseconds of
// a step of `blocks` tiles at a time (the clock falls as units fill), of a tile's results
// beside the next one's steps, and of the launch with its first loads and last
// results.  Fitted to 32 products of 33 to 18944 tokens, each in whole tiles of both
// sizes and in all numbers of parts; expected within 8 % of 1024 x 18944 x 3584 (256-tiles
// in four parts 75.8 us, whole 84.7, 128-tiles 91) and of 256 x 3584 x 3584 (128-tiles 17.4,
// 256-tiles in eight parts 24.5, the streaming kernel 16).
double f8_step_us(int tile, int64_t blocks)
{
    const double b = (double)blocks / (double)kUnits;
    if (tile == 256) return 1.05 + 0.40 * b;
    return b <= 1 ? 0.40 + 0.12 * b : 0.92 + 0.18 * (b - 1);
}
constexpr double kF8Launch[2] = {10, 5.5}, kF8Result[2] = {4, 0.8}, kF8SumUs = 4;
constexpr double kF8PartBytesPerUs = 4.5e6; // as kPartBytesPerUs

// One tile size: the last round's tiles are cut as in cut_tiles.
Cut cut_f8(int64_t m, int64_t n, int64_t k, int tile)
{
    Cut c{};
    c.tile = tile;
    c.tm = (m + tile - 1) / tile;
    c.tn = (n + tile - 1) / tile;
    c.steps = (k + 127) / 128;
    const int64_t tiles = c.tm * c.tn, slots = kUnits * (tile == 256 ? 1 : 2), rest = tiles % slots;
    const int small = tile == 128;
    const double rounds = (double)(tiles / slots) * ((double)c.steps * f8_step_us(tile, slots) + kF8Result[small]) +
                          kF8Launch[small];
    c.full = tiles;
    c.splits = 1;
    c.us = rounds + (rest ? (double)c.steps * f8_step_us(tile, rest) : 0);
    const int64_t most = rest ? std::min(std::min(slots / rest, c.steps / 2), kMostSplits) : 0;
    for (int64_t splits = 2; splits <= most; ++splits) {
        const int64_t bytes = rest * splits * tile * tile * 4;
        const double us = rounds + (double)((c.steps + splits - 1) / splits) * f8_step_us(tile, rest * splits) +
                          (double)bytes / kF8PartBytesPerUs + kF8SumUs + kSumPartUs * (double)splits;
        if (us < c.us) {
            c.us = us;
            c.full = tiles - rest;
            c.splits = splits;
            c.bytes = bytes;
        }
    }
    // blocks are counted in 32 bits
    c.fits = c.full + rest * c.splits < ((int64_t)1 << 31);
    return c;
}

// The streaming kernel's expected time, as few_us: 64 tokens through 3584 x 3584 take
// 6.7 us so and 14.2 in tiles, 128 through 18944 x 3584 44 and 18.
double f8_few_us(int64_t tokens, int64_t rows, int64_t cols)
{
    const int64_t groups = (tokens + 31) / 32;
    const double blocks = (double)((rows + 31) / 32) * (double)groups;
    const double weight = (double)rows * (double)cols;
    return 2.2 + blocks * 1.2 / 512 + weight / 5.0e6 + (double)(groups - 1) * weight / 9.5e6;
}

} // namespace

LinearPlan plan_linear_f8(int64_t tokens, int64_t rows, int64_t cols)
{
    LinearPlan p{};
    p.few = tokens <= 32 || cols == 0;
    if (!p.few) {
        const Cut big = cut_f8(rows, tokens, cols, 256), small = cut_f8(rows, tokens, cols, 128);
        p.cut = small.us < big.us && small.fits ? small : big;
        // few tiles: their steps may be less work than reading the weight
        const double weight_us = (double)rows * (double)cols / 5.0e6;
        p.few = tokens <= 1024 && f8_few_us(tokens, rows, cols) < std::max(p.cut.us, weight_us);
    }
    if (p.few) {
        p.cut = Cut{};
        // blocks of 256 threads, a launch having fewer than 2^32
        p.cut.fits = (rows + 15) / 16 * ((tokens + 31) / 32) < (1 << 24);
    }
    p.bytes = p.cut.bytes;
    return p;
}

int validate_quantize_f8(const void* x, int dtype, int64_t rows, int64_t cols, bool square, int format,
                         const uint8_t* q, int64_t q_stride, const uint8_t* scale, const uint8_t* qt,
                         int64_t qt_stride, const uint8_t* scale_t, bool* todo)
{
    *todo = false;
    if (int st = check_dtype(dtype)) return st;
    if (int st = check_format(format)) return st;
    if (int st = check_f8_sizes(rows, cols)) return st;
    if (int st = check_stride("q_stride", q_stride, cols, kMaxRowsI8)) return st;
    if (!qt != !scale_t && rows > 0 && cols > 0)
        return fail(ROI_E_INVAL, "qt and scale_t are given together or not at all");
    if (qt)
        if (int st = check_stride("qt_stride", qt_stride, rows, kMaxRowsI8)) return st;
    const Buffer b[] = {{x, (size_t)rows * (size_t)cols * (dtype == ROI_FP32 ? 4 : 2), false},
                        {q, f8_bytes(rows, cols, q_stride), true},
                        {scale, f8_scales(rows, cols, square), true, kScaleAlign},
                        {qt, qt ? f8_bytes(cols, rows, qt_stride) : 0, true},
                        {scale_t, qt ? f8_scales(cols, rows, square) : 0, true, kScaleAlign}};
    if (int st = check_buffers(b, 5)) return st;
    *todo = rows > 0 && cols > 0;
    return ok();
}

int validate_dequantize_f8(const uint8_t* q, int64_t q_stride, const uint8_t* scale, int64_t rows,
                           int64_t cols, bool square, int format, const void* x, int dtype,
                           bool* todo)
{
    *todo = false;
    if (int st = check_dtype(dtype)) return st;
    if (int st = check_format(format)) return st;
    if (int st = check_f8_sizes(rows, cols)) return st;
    if (int st = check_stride("q_stride", q_stride, cols, kMaxRowsI8)) return st;
    const Buffer b[] = {{x, (size_t)rows * (size_t)cols * (dtype == ROI_FP32 ? 4 : 2), true},
                        {q, f8_bytes(rows, cols, q_stride), false},
                        {scale, f8_scales(rows, cols, square), false, kScaleAlign}};
    if (int st = check_buffers(b, 3)) return st;
    *todo = rows > 0 && cols > 0;
    return ok();
}

int validate_linear_f8(const uint8_t* xq, int64_t x_stride, const uint8_t* xs, int x_format,
                       const uint8_t* wq, int64_t w_stride, const uint8_t* ws, bool w_square,
                       const uint16_t* bias, int64_t tokens, int64_t rows, int64_t cols,
                       const uint16_t* y, const void* workspace, int64_t workspace_bytes,
                       int64_t need, bool* todo)
{
    *todo = false;
    if (int st = check_format(x_format)) return st;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    if (int st = check_stride("x_stride", x_stride, cols, kMaxStride)) return st;
    if (int st = check_stride("w_stride", w_stride, cols, kMaxStride)) return st;
    if (int st = check_workspace(workspace, workspace_bytes, need)) return st;
    const size_t t = (size_t)tokens, r = (size_t)rows;
    const Buffer b[] = {{xq, f8_bytes(tokens, cols, x_stride), false},
                        {xs, f8_scales(tokens, cols, false), false, kScaleAlign},
                        {wq, f8_bytes(rows, cols, w_stride), false},
                        {ws, f8_scales(rows, cols, w_square), false, kScaleAlign},
                        {bias, bias ? r * 2 : 0, false},
                        {y, t * r * 2, true},
                        {workspace, (size_t)need, true}};
    if (int st = check_buffers(b, 7)) return st;
    *todo = tokens > 0 && rows > 0;
    return ok();
}

int validate_step(const roi_step_tensor* t, int count, int grad_dtype, int bits,
                  const roi_step_params* opt, AdamStep* step, bool* todo)
{
    *todo = false;
    if (int st = check_dtype(grad_dtype)) return st;
    if (bits != 8 && bits != 32)
        return fail(ROI_E_INVAL, "the moments' bits must be 8 or 32 (got %d)", bits);
    if (int st = fold_adamw(opt, step)) return st;
    if (step->eps < FLT_MIN) // whose reciprocal the step multiplies with
        return fail(ROI_E_INVAL, "AdamW eps must be at least 2^-126");
    if (int st = check_count(t, count)) return st;
    std::vector<Range> ranges;
    ranges.reserve((size_t)count * 6);
    for (int i = 0; i < count; ++i) {
        const roi_step_tensor& s = t[i];
        if (s.numel < 0)
            return fail(ROI_E_INVAL, "tensor %d: numel (%lld) must be >= 0", i, (long long)s.numel);
        if (s.numel >= kMaxStepValues)
            return fail(ROI_E_UNSUPPORTED, "tensor %d: numel must be below 2^40", i);
        if (s.elem_offset % 4 != 0)
            return fail(ROI_E_INVAL, "tensor %d: elem_offset must be a multiple of 4", i);
        if (s.elem_offset > UINT64_MAX - (uint64_t)s.numel)
            return fail(ROI_E_INVAL, "tensor %d: elem_offset + numel overflows 64 bits", i);
        if (s.numel == 0) continue;
        if (!s.param || !s.grad || !s.exp_avg || !s.exp_avg_sq ||
            (bits == 8 && (!s.avg_scale || !s.sq_scale)))
            return fail(ROI_E_INVAL, "tensor %d: a required pointer is NULL", i);
        if (!aligned16(s.param) || !aligned16(s.grad) || !aligned16(s.exp_avg) ||
            !aligned16(s.exp_avg_sq) ||
            (bits == 8 && ((uintptr_t)s.avg_scale % kScaleAlign || (uintptr_t)s.sq_scale % kScaleAlign)))
            return fail(ROI_E_INVAL,
                        "tensor %d: device pointers must be 16-byte aligned (scales: to 4 bytes)", i);
        const size_t n = (size_t)s.numel, moment = bits == 8 ? n : 4 * n;
        add_range(ranges, s.param, 4 * n, true);
        add_range(ranges, s.grad, n * (grad_dtype == ROI_FP32 ? 4 : 2), false);
        add_range(ranges, s.exp_avg, moment, true);
        add_range(ranges, s.exp_avg_sq, moment, true);
        if (bits == 8) {
            add_range(ranges, s.avg_scale, (size_t)scale_bytes(s.numel), true);
            add_range(ranges, s.sq_scale, (size_t)scale_bytes(s.numel), true);
        }
        *todo = true;
    }
    if (int st = check_overlaps(ranges)) {
        *todo = false;
        return st;
    }
    return ok();
}

} // namespace roi
