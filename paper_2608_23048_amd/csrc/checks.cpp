// checks.cpp -- the host-side argument checks of the C ABI (checks.hpp).
#include "checks.hpp"

#include <algorithm>
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

int check_adamw(const roi_adamw_params* o, AdamStep* st)
{
    if (!o) return fail(ROI_E_INVAL, "the AdamW parameters must not be NULL");
    if (!(o->lr >= 0.0f) || !std::isfinite(o->lr))
        return fail(ROI_E_INVAL, "AdamW lr must be finite and >= 0");
    if (!(o->beta1 >= 0.0f && o->beta1 < 1.0f) || !(o->beta2 >= 0.0f && o->beta2 < 1.0f))
        return fail(ROI_E_INVAL, "AdamW betas must lie in [0, 1)");
    if (!(o->eps > 0.0f) || !std::isfinite(o->eps))
        return fail(ROI_E_INVAL, "AdamW eps must be finite and > 0");
    if (!(o->weight_decay >= 0.0f) || !std::isfinite(o->weight_decay))
        return fail(ROI_E_INVAL, "AdamW weight_decay must be finite and >= 0");
    if (o->t < 1) return fail(ROI_E_INVAL, "AdamW step count t must be >= 1");
    const double lr = o->lr, b1 = o->beta1, b2 = o->beta2;
    const double bc1 = 1.0 - std::pow(b1, (double)o->t);
    const double bc2 = 1.0 - std::pow(b2, (double)o->t);
    st->decay = (float)(1.0 - lr * (double)o->weight_decay);
    st->beta1 = o->beta1;
    st->beta2 = o->beta2;
    st->one_m_beta1 = (float)(1.0 - b1);
    st->one_m_beta2 = (float)(1.0 - b2);
    st->step_size = (float)(lr / bc1);
    st->inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    st->eps = o->eps;
    return ROI_OK;
}

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

} // namespace roi
