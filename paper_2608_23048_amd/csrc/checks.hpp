// checks.hpp -- the library's host-side argument checks.  Plain C++ with no
// GPU code, so that the same file also builds with the host compiler alone
// (and its address and undefined-behaviour sanitizers).  Every entry point of
// the C ABI runs these before it launches anything; a failure returns a
// status and leaves its detail in the thread-local error text.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <string>
#include <vector>

#include "roi.h"

namespace roi {

// Thread-local detail of the last failure (returned by roi_last_error).
extern thread_local std::string g_last_error;

// Records a printf-style detail and returns `status`.
int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the detail and returns ROI_OK.
int ok();
bool aligned16(const void* p);
// Whether [a, a + na) and [b, b + nb) share a byte (empty ranges share none).
bool overlap(const void* a, size_t na, const void* b, size_t nb);

// One checked address range of a call: [p, p + n), an input or an output.
struct Range {
    uintptr_t p;
    size_t n;
    bool out;
};
// Fails when an output overlaps any other range (inputs may overlap inputs).
int check_overlaps(std::vector<Range>& r);
void add_range(std::vector<Range>& r, const void* p, size_t n, bool out);

// The sizes of one [rows, cols] tensor of groups of m.
struct Shape {
    int64_t numel = 0;
    int64_t ngroups = 0;
};
// Pattern (1 <= n <= m, m in {4, 8, 16, 32}), finite positive temperatures.
int check_common(int n, int m, float tau, float lambda);
// check_common plus the tensor's sizes and its global element offset.
int check_shape(int64_t rows, int64_t cols, int n, int m, float tau, float lambda,
                uint64_t elem_offset, Shape* sh);
// A descriptor array of `count` entries (NULL only when empty).
int check_count(const void* t, int count);

// One AdamW step folded into constants (host, fp64, rounded once):
// phi <- phi * decay - step_size * m' / (sqrt(v') * inv_sqrt_bc2 + eps),
// m' = beta1 m + (1 - beta1) g, v' = beta2 v + (1 - beta2) g^2.
struct AdamStep {
    float decay;        // 1 - lr * weight_decay
    float beta1, beta2;
    float one_m_beta1, one_m_beta2;
    float step_size;    // lr / (1 - beta1^t)
    float inv_sqrt_bc2; // 1 / sqrt(1 - beta2^t)
    float eps;
};
int check_adamw(const roi_adamw_params* o, AdamStep* st);

// The forward's tensors: sets *with_s / *with_idx to whether the soft mask and
// the indices are requested (-1 when every tensor is empty: nothing to do).
int validate_fwd(const roi_fwd_tensor* t, int count, int n, int m, float tau, float lambda,
                 int* with_s, int* with_idx);

// One tensor of a backward call; phi is overwritten with the updated logits
// when the AdamW step is fused (m and v set).
struct BwdDesc {
    const uint16_t* G;
    const uint16_t* W;
    const float* phi;
    float* dphi;
    float* m;
    float* v;
    int64_t rows, cols;
    uint64_t off;
};
// The backward's tensors (opt: the fused AdamW step or NULL, folded into *st);
// *any is false when every tensor is empty.
int validate_bwd(const BwdDesc* t, int count, int n, int m, float tau, float lambda,
                 const roi_adamw_params* opt, AdamStep* st, bool* any);

// The categorical sampler's arguments (m in {4, 8}): sets the group count and
// the number of candidates C = binom(m, n) per group.
int validate_cat(bool fwd, const uint16_t* W, const float* alpha, const uint16_t* G, int64_t rows,
                 int64_t cols, int n, int m, float tau, float lambda, uint64_t group_offset,
                 const uint16_t* W_masked, const float* S, const uint8_t* choice,
                 const float* dalpha, int64_t* ngroups, int* C);

// One int8-rows call (roi_quantize_rows, roi_dequantize_rows).  x_out: x is the
// output.  *todo is false when there is nothing to write.
int validate_rows_i8(const void* x, int dtype, const int8_t* q, const float* scale, int64_t rows,
                     int64_t cols, bool x_out, bool* todo);

// The longest int8 row and the most of them; the largest product and gradient
// sizes (kernels count tokens, rows and columns in 32 bits); and the longest
// exact int32 sum of products of two int8 values (131071 * 2^14 < 2^31).
constexpr int64_t kMaxRowsI8 = (int64_t)1 << 31;
constexpr int64_t kMaxLinearDim = (int64_t)1 << 22;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int64_t kMaxI8Sum = 131071;

constexpr int64_t kUnits = 256; // compute units of an MI355X

// How a product of m x n results over a sum of k is cut: square tiles, of which
// the first `full` are whole and the sums of the others are cut into `splits`
// parts, which pass through the workspace as 32-bit values.
struct Cut {
    int tile;
    int64_t tm, tn, full;
    int64_t splits;
    int64_t steps; // of the whole sum
    int64_t bytes; // of workspace
    double us;     // what the call is expected to take
    bool fits;     // fewer blocks than a launch takes
};
// Times of the tiled kernels in microseconds, as measured: a step of a 256-tile
// on every compute unit, of one 128-tile on every unit and of two, and what a
// tile takes beside its steps (the launch, its first loads, its results).
struct TileCost {
    double step256, rest256, step128, two128, rest128;
};
constexpr TileCost kLinearCost = {1.36, 9, 0.39, 0.80, 5.5};
constexpr TileCost kPackedCost = {0.80, 8, 0.38, 0.72, 5};
constexpr TileCost kGradCost = {1.70, 14, 0.57, 1.50, 8};
// Of a 256-tile with both operands in bf16 (there is no 128-tile).
constexpr TileCost kReadyCost = {1.40, 12, 0, 0, 0};
Cut cut_product(int64_t m, int64_t n, int64_t k, int64_t step, const TileCost& cost);

// The int8 product's way: with few tokens the kernel that streams the weight
// past them (no workspace), else the tiles of `cut`, before which rows of a
// length that is no multiple of 16 are copied to the workspace (x_bytes, w_bytes),
// to rows of `row` bytes (whole cache lines); the parts of cut tiles follow.
struct LinearPlan {
    bool few;
    int64_t row, x_bytes, w_bytes;
    int64_t bytes; // of workspace
    Cut cut;
};
LinearPlan plan_linear(int64_t tokens, int64_t rows, int64_t cols, bool packed);

// Bytes of workspace arrays, each from a multiple of 256 bytes on.
constexpr int64_t padded256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// A gradient's way (out [m, n], summed over k).  The tiles' loads take whole
// 16-byte pieces of grad_y's rows (k values with `sum_rows` false, else m) and
// words of q's: rows that end within one are first copied to the workspace, to
// rows of dy_row and q_row elements (whole cache lines).  With `ready` q is first written there in
// bf16, transposed, [n, ready_k].  The workspace holds these arrays in this order
// (dy_bytes, q_bytes, ready_bytes; 0: not there), then the parts of cut tiles.
// With `deep` the 128-tiles are no more than the compute units, and q's rows are
// in whole 16-byte pieces.
struct GradPlan {
    bool ready, deep;
    int64_t dy_row, q_row, ready_k;
    int64_t dy_bytes, q_bytes, ready_bytes;
    int64_t bytes; // of workspace
    Cut cut;
};
GradPlan plan_grad(int64_t m, int64_t n, int64_t k, bool sum_rows);

// Sizes of a linear call: ROI_OK, or why the call is refused.
int check_linear_sizes(int64_t tokens, int64_t rows, int64_t cols);
// What a product asks of its sum beside (packed: 2:4 weights).
int check_linear_sum(int64_t cols, bool packed);
int validate_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq, const uint32_t* meta,
                       const float* ws, const uint16_t* bias, int64_t tokens, int64_t rows,
                       int64_t cols, const void* y, int dtype, const void* workspace,
                       int64_t workspace_bytes, int64_t need, bool* todo);
// q [krows, cols] and scale [krows] beside grad_y [tokens, rows]; out has
// out_rows rows of cols.
int validate_grad_i8(const uint16_t* grad_y, const int8_t* q, const float* scale, int64_t krows,
                     int64_t tokens, int64_t rows, int64_t cols, const uint16_t* out,
                     int64_t out_rows, const void* workspace, int64_t workspace_bytes,
                     int64_t need, bool* todo);

// Calls launch(first, count, elem0) for consecutive pieces of [0, items) --
// items of `per_item` elements starting at global element elem_offset -- so
// that within a piece every Philox block index (element / 4) has the same high
// 32 bits.  Pieces end at multiples of 2^34 elements, which per_item divides.
template <typename F>
int for_each_piece(uint64_t elem_offset, int64_t items, int64_t per_item, F&& launch)
{
    int64_t done = 0;
    while (done < items) {
        const uint64_t e0 = elem_offset + (uint64_t)done * (uint64_t)per_item;
        const uint64_t boundary = ((e0 >> 34) + 1) << 34;
        const uint64_t fit = (boundary - e0) / (uint64_t)per_item;
        const int64_t left = items - done;
        const int64_t count = fit < (uint64_t)left ? (int64_t)fit : left;
        if (int st = launch(done, count, e0)) return st;
        done += count;
    }
    return ROI_OK;
}

} // namespace roi
