/*
 * roi.h -- C ABI of the MI355X (gfx950) RoI differentiable N:M mask sampler.
 *
 * The method: "Reservoir of Importance: Learning Semi-Structured Sparsity with
 * Differentiable Subset Sampling" (arxiv 2608.23048).  Every group of m
 * consecutive weights carries m logits phi (one per weight, §4.2.1).  Each
 * training step perturbs them with Gumbel noise into keys (§3.2, §4.2.2),
 * keeps the n largest keys (hard Gumbel-Top-K, §3.2), and relaxes that
 * selection into a soft n-hot mask S by n softmax steps (§3.2 recursion,
 * Appendix Algorithm 1).  The forward emits the hard-masked weights; the
 * backward differentiates through the relaxation (the straight-through
 * variant of the appendix, "Comparison with Straight-Through Gumbel-Top-K").
 *
 * Conventions shared by every entry point
 * ----------------------------------------
 *  - Pointers are DEVICE pointers on the current HIP device, 16-byte aligned,
 *    contiguous; inputs and outputs must not overlap.  The caller owns all
 *    memory; the library allocates none.
 *  - bf16 tensors are passed as their raw 16-bit patterns (uint16_t).
 *  - A weight tensor is row-major [rows, cols] (PyTorch Linear: [out, in]);
 *    groups are m consecutive elements along cols, so cols % m == 0.  Any
 *    back-to-back stack of such tensors is itself a valid [1, total] input:
 *    groups never straddle tensors, and the noise depends only on the global
 *    element index.
 *  - Calls are asynchronous on `stream` (0 = the null stream).  Argument
 *    errors are detected on the host and returned before anything is
 *    launched; nothing is written then.  No exceptions cross the ABI.
 *  - Return value: ROI_OK or a negative roi_status; roi_last_error() gives a
 *    thread-local human-readable detail of the last failure.
 *  - Supported patterns: m in {4, 8, 16, 32} with 1 <= n <= m.
 *
 * Noise (the same definition the forward and the backward use):
 *  - global element index e = elem_offset + (flat index of the element);
 *  - x = word (e mod 4) of Philox4x32-10 (Salmon et al., SC'11) with key
 *    (lo32 seed, hi32 seed) and counter (lo32 e/4, hi32 e/4, lo32 step,
 *    hi32 step);
 *  - u = (2 (x >> 9) + 1) 2^-24, in (0, 1) (Algorithm 1: u ~ Uniform(0,1));
 *  - g = -L(-L(u)) with L the library's deterministic fp32 logarithm
 *    (Algorithm 1: g = -log(-log u)): x = z 2^k with z in [0.703125, 1.40625),
 *    a 128-cell table of (1/c, -ln(1/c)) (the two cells touching 1 hold
 *    (1, 0)), r = fma(z, 1/c, -1), ln(1+r) by its degree-4 series, and
 *    L = fma(k, ln2, -ln(1/c) + ln(1+r)); a fixed sequence of IEEE fp32
 *    operations, so the value is reproducible (max error 1.45 ulp);
 *  - kappa = fl(fl(phi / lambda) + g) in fp32 (§3.2 key; §4.2.3 applies the
 *    trick to phi / lambda).
 *  Given (seed, step, elem_offset) the noise is a pure function, so the
 *  backward regenerates it instead of storing it, and any split of a stack
 *  into calls with matching elem_offset gives identical results.
 */
#ifndef ROI_H
#define ROI_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ROI_OK = 0,
    ROI_E_INVAL = -1,       /* invalid argument (sizes, pattern, temperatures, pointers) */
    ROI_E_UNSUPPORTED = -2, /* valid for the method but not built: m outside {4, 8, 16, 32} */
    ROI_E_HIP = -3          /* the HIP runtime reported an error at launch */
} roi_status;

/*
 * roi_mask_fwd -- one forward sample of the n:m mask for every group.
 *
 * §3.2 / §4.2.2: keys kappa = phi/lambda + g; hard selection = the n largest
 * keys of each group (ties go to the lower index; -0.0 and +0.0 tie).
 * §4.1: W_masked = W (.) hard mask (pruned entries are +0.0, bits 0x0000).
 * §3.2 recursion / Algorithm 1: soft_mask S = sum_{k=1..n} mu^(k) with
 * alpha^(1) = kappa, mu^(k) = softmax(alpha^(k) / tau),
 * alpha^(k+1) = alpha^(k) + log(1 - mu^(k)), computed in fp32 (log(1 - mu) is
 * floored at log(FLT_MIN)).
 *
 *  W          bf16 [rows, cols]          frozen weights (read)
 *  logits     fp32 [rows, cols]          phi (read)
 *  rows, cols sizes, rows >= 0, cols >= 0, cols % m == 0, rows * cols < 2^62
 *  n, m       keep n of every m; m in {4, 8, 16, 32}, 1 <= n <= m
 *  tau        relaxation temperature, finite, > 0 (used only for soft_mask)
 *  lambda     sampling temperature, finite, > 0 (§4.2.3)
 *  seed, step Philox key and step counter
 *  elem_offset global index of element 0; elem_offset % m == 0 (so groups of a
 *             stack keep their positions in the global index space)
 *  W_masked   bf16 [rows, cols]          (written; required)
 *  soft_mask  fp32 [rows, cols] or NULL  (written when not NULL)
 *  sel_idx    uint8 [rows*cols/m, n] or NULL: the kept indices of each group in
 *             selection order (descending key)   (written when not NULL)
 */
int roi_mask_fwd(const uint16_t* W, const float* logits, int64_t rows, int64_t cols, int n,
                 int m, float tau, float lambda, uint64_t seed, uint64_t step,
                 uint64_t elem_offset, uint16_t* W_masked, float* soft_mask, uint8_t* sel_idx,
                 hipStream_t stream);

/*
 * roi_mask_fwd_soft -- the pure soft forward (the paper's default setting:
 * "w/o STE" in the appendix comparison with the straight-through variant;
 * §4.2.2 relaxation used directly in the forward pass).  Same arguments and
 * noise as roi_mask_fwd; the output is
 *   W_soft = bf16_rne(W (.) S), S = sum_{k=1..n} mu^(k) (fp32, §3.2 recursion),
 * and soft_mask / sel_idx, when not NULL, receive S and the hard top-n indices
 * of the same keys.  The backward is roi_mask_bwd (the relaxation is the
 * differentiated path in both settings).
 * S is always evaluated at the exact keys (as in roi_mask_fwd), and W_soft is
 * the bf16 rounding of W (.) S; with soft_mask and sel_idx both NULL a kernel
 * without the selection runs, with the same W_soft bits.
 */
int roi_mask_fwd_soft(const uint16_t* W, const float* logits, int64_t rows, int64_t cols, int n,
                      int m, float tau, float lambda, uint64_t seed, uint64_t step,
                      uint64_t elem_offset, uint16_t* W_soft, float* soft_mask, uint8_t* sel_idx,
                      hipStream_t stream);

/*
 * roi_mask_bwd -- dL/dlogits from dL/dW_masked.
 *
 * Straight-through (Appendix, Comparison with Straight-Through Gumbel-Top-K):
 * the forward value is the hard mask, the backward goes through the
 * relaxation as if W_masked = W (.) S.  So dL/dS = grad_W_masked (.) W (exact
 * in fp32), dL/dkappa is the reverse-mode derivative of the §3.2 recursion,
 * and dL/dphi = dL/dkappa / lambda.  The keys are regenerated from
 * (seed, step, elem_offset) and must match the forward call's arguments: the
 * derivative is taken at exactly the fp32 keys the forward sampled.
 *
 *  grad_W_masked bf16 [rows, cols]       (read)
 *  W, logits, rows, cols, n, m, tau, lambda, seed, step, elem_offset: as in
 *             roi_mask_fwd
 *  grad_logits fp32 [rows, cols]         (overwritten)
 */
int roi_mask_bwd(const uint16_t* grad_W_masked, const uint16_t* W, const float* logits,
                 int64_t rows, int64_t cols, int n, int m, float tau, float lambda, uint64_t seed,
                 uint64_t step, uint64_t elem_offset, float* grad_logits, hipStream_t stream);

/*
 * Grouped calls: one call over many separately allocated tensors (e.g. every
 * linear layer of a model), with the shared pattern, temperatures, seed and
 * step.  Tensor i is processed exactly as the single-tensor call with its own
 * pointers, rows, cols and elem_offset would process it (same outputs, bit
 * for bit); the library launches the work of up to 32 tensor pieces per grid
 * instead of one grid per tensor.  The descriptor array is host memory, read
 * during the call only; the pointers in it follow the conventions above.
 * Tensors with rows * cols == 0 are skipped (their pointers may be NULL).
 * soft_mask and sel_idx must each be non-NULL for every nonempty tensor or
 * for none.  No output may overlap any input or output of any tensor (inputs
 * may overlap each other).  Any argument error returns before anything is
 * launched; roi_last_error() names the offending tensor.
 */
typedef struct {
    const uint16_t* W;     /* bf16 [rows, cols] (read) */
    const float* logits;   /* fp32 [rows, cols] (read) */
    uint16_t* W_masked;    /* bf16 [rows, cols] (written) */
    float* soft_mask;      /* fp32 [rows, cols] or NULL */
    uint8_t* sel_idx;      /* uint8 [rows*cols/m, n] or NULL */
    int64_t rows, cols;
    uint64_t elem_offset;  /* global index of element 0, % m == 0 */
} roi_fwd_tensor;

typedef struct {
    const uint16_t* grad_W_masked; /* bf16 [rows, cols] (read) */
    const uint16_t* W;             /* bf16 [rows, cols] (read) */
    const float* logits;           /* fp32 [rows, cols] (read) */
    float* grad_logits;            /* fp32 [rows, cols] (overwritten) */
    int64_t rows, cols;
    uint64_t elem_offset;
} roi_bwd_tensor;

/* roi_mask_fwd over `count` tensors (count >= 0). */
int roi_mask_fwd_grouped(const roi_fwd_tensor* tensors, int count, int n, int m, float tau,
                         float lambda, uint64_t seed, uint64_t step, hipStream_t stream);
/* roi_mask_fwd_soft over `count` tensors (W_masked receives W_soft). */
int roi_mask_fwd_soft_grouped(const roi_fwd_tensor* tensors, int count, int n, int m, float tau,
                              float lambda, uint64_t seed, uint64_t step, hipStream_t stream);
/* roi_mask_bwd over `count` tensors. */
int roi_mask_bwd_grouped(const roi_bwd_tensor* tensors, int count, int n, int m, float tau,
                         float lambda, uint64_t seed, uint64_t step, hipStream_t stream);

/*
 * roi_mask_bwd_adamw -- roi_mask_bwd with one AdamW step on the logits fused
 * in (appendix: the logits are trained with AdamW, beta1 = 0.9, beta2 = 0.95,
 * weight decay 0.05, a learning rate decaying from 1e-3 to 1e-4; the weights
 * stay frozen).  With g = dL/dlogits of this step, every logit becomes
 *   phi' = phi (1 - lr wd) - (lr / (1 - beta1^t)) m' / (sqrt(v' / (1 - beta2^t)) + eps),
 *   m'   = beta1 m + (1 - beta1) g,   v' = beta2 v + (1 - beta2) g^2
 * (decoupled weight decay, Loshchilov & Hutter; bias-corrected moments,
 * Kingma & Ba), in fp32.  The keys use the logits as they were before the
 * step.  The gradient is never stored unless grad_logits is given, so the
 * step moves 28 bytes per weight instead of 12 (backward) + 28 (optimizer).
 *
 *  logits      fp32 [rows, cols]  read, then overwritten with phi'
 *  exp_avg     fp32 [rows, cols]  m, overwritten with m'
 *  exp_avg_sq  fp32 [rows, cols]  v, overwritten with v'
 *  grad_logits fp32 [rows, cols]  or NULL: also written with g
 *  opt         host struct: lr >= 0, 0 <= beta1, beta2 < 1, eps > 0,
 *              weight_decay >= 0 (all finite), t >= 1 = this step's 1-based
 *              optimizer step count; the caller schedules lr (e.g. with
 *              roi_anneal).
 *  Other arguments as in roi_mask_bwd.  The moments and grad_logits must not
 *  overlap each other, the logits or the inputs.
 */
typedef struct {
    float lr;
    float beta1, beta2;
    float eps;
    float weight_decay;
    int64_t t;
} roi_adamw_params;

int roi_mask_bwd_adamw(const uint16_t* grad_W_masked, const uint16_t* W, float* logits,
                       float* exp_avg, float* exp_avg_sq, float* grad_logits, int64_t rows,
                       int64_t cols, int n, int m, float tau, float lambda, uint64_t seed,
                       uint64_t step, uint64_t elem_offset, const roi_adamw_params* opt,
                       hipStream_t stream);

/* roi_mask_bwd_adamw over `count` tensors (grouped-call conventions above). */
typedef struct {
    const uint16_t* grad_W_masked; /* bf16 [rows, cols] (read) */
    const uint16_t* W;             /* bf16 [rows, cols] (read) */
    float* logits;                 /* fp32 [rows, cols] (read, overwritten) */
    float* exp_avg;                /* fp32 [rows, cols] (read, overwritten) */
    float* exp_avg_sq;             /* fp32 [rows, cols] (read, overwritten) */
    float* grad_logits;            /* fp32 [rows, cols] or NULL */
    int64_t rows, cols;
    uint64_t elem_offset;
} roi_adamw_tensor;

int roi_mask_bwd_adamw_grouped(const roi_adamw_tensor* tensors, int count, int n, int m,
                               float tau, float lambda, uint64_t seed, uint64_t step,
                               const roi_adamw_params* opt, hipStream_t stream);

/*
 * roi_mask_export -- the final mask after training, in dense and compressed
 * form.  §4.2.3 anneals the sampling temperature lambda towards 0; the
 * sampler's lambda -> 0 limit keeps the n largest logits of each group (ties
 * to the lower index, as in the sampler), with no noise.  This call writes
 * that mask:
 *  W_masked bf16 [rows, cols] or NULL: W where kept, +0.0 elsewhere;
 *  values   bf16 [rows*cols/m, n] or NULL: the kept weights of each group in
 *           increasing index order (the compressed sparse weight);
 *  idx      uint8 [rows*cols/m, n] or NULL: their indices, increasing;
 *  meta     uint32 [ceil(rows*cols/m / 8)] or NULL, 2:4 only: group q's two
 *           indices as 2-bit fields in bits 4(q%8) .. 4(q%8)+3 of word q/8,
 *           the lower index in the low two bits (the index metadata that
 *           accompanies 2:4-compressed values).
 * At least one output must be requested.  W may be NULL when only idx and
 * meta are.  logits, W, rows, cols, n, m as in roi_mask_fwd (no temperatures,
 * seed or step).
 */
int roi_mask_export(const float* logits, const uint16_t* W, int64_t rows, int64_t cols, int n,
                    int m, uint16_t* W_masked, uint16_t* values, uint8_t* idx, uint32_t* meta,
                    hipStream_t stream);

/*
 * The categorical mask sampler: the parameterization the paper compares with
 * (appendix, "Optimization Efficiency"), one logit per feasible n-hot mask of
 * a group, Pr(c) = softmax(alpha)_c, sampled with Gumbel-Softmax.  It is a
 * second workload on the same harness: binom(m, n) logits per group instead
 * of m (1.5x the weights at 2:4, 3.5x at 2:8, 8.75x at 4:8).
 *  - candidates: the n-subsets of {0..m-1} in lexicographic order;
 *  - keys kappa_c = fl(fl(alpha_c / lambda) + g_c), g_c the noise of element
 *    4 B Q + c with B = ceil(C / 4), Q = group_offset + local group index;
 *  - hard sample: the candidate of largest key (ties to the lower candidate),
 *    W_masked = W (.) its mask, choice = its index;
 *  - soft mask S_j = sum_c softmax(kappa / tau)_c [j in c];
 *  - backward (straight-through): ybar_c = sum_{j in c} (dL/dW_masked (.) W)_j,
 *    dL/dalpha = softmax (.) (ybar - <softmax, ybar>) / (tau lambda).
 * m in {4, 8}.  cat_logits fp32 [rows*cols/m, C] (group-major).  Other
 * arguments and conventions as for the item sampler.
 */
/* binom(m, n), the logits per group, or -1 for an unsupported pattern. */
int roi_cat_num_candidates(int n, int m);
int roi_cat_mask_fwd(const uint16_t* W, const float* cat_logits, int64_t rows, int64_t cols,
                     int n, int m, float tau, float lambda, uint64_t seed, uint64_t step,
                     uint64_t group_offset, uint16_t* W_masked, float* soft_mask,
                     uint8_t* choice, hipStream_t stream);
int roi_cat_mask_bwd(const uint16_t* grad_W_masked, const uint16_t* W, const float* cat_logits,
                     int64_t rows, int64_t cols, int n, int m, float tau, float lambda,
                     uint64_t seed, uint64_t step, uint64_t group_offset, float* grad_cat_logits,
                     hipStream_t stream);

/*
 * The linear layer around a masked weight, in 8 bits.  Rows of activations
 * (or of weights) are held as int8 with one fp32 scale each: the tokens' rows
 * are the left operand of the layer's product and, kept until the backward,
 * the checkpoint its weight gradient reads; the weights' rows are those of a
 * masked weight (roi_mask_fwd, roi_mask_export), dense or 2:4-compressed.
 *
 * Conventions beside the shared ones above:
 *  - x [tokens, cols], weight [rows, cols], y [tokens, rows]; any sizes >= 0
 *    with rows and cols below 2^22 and tokens below 2^30.  Operands whose rows
 *    are no multiple of 16 bytes cost a copy to the workspace, or slower loads.
 *  - An empty tensor's pointer may be NULL.  A sum over nothing is 0.
 *  - The scales that the product and the gradients read (xs, ws) need only the
 *    4-byte alignment of a float, so that a batch may be cut at any token whose
 *    int8 row is 16-byte aligned.
 *  - workspace: device memory of at least the bytes that the matching
 *    *_workspace call returns (it may be NULL where that is 0), 16-byte
 *    aligned, overlapping nothing; its contents need no preparation and are
 *    undefined afterwards.  Calls that may run at the same time need one each.
 *    For sizes that the call refuses the *_workspace call returns the same
 *    negative roi_status.
 *  - A product or gradient of more than about 2^39 results in tiles of 256 x 256
 *    (more blocks than a launch takes) is refused with ROI_E_UNSUPPORTED.
 *  - Results do not depend on the order in which blocks run: the same inputs
 *    give the same bits.
 */
typedef enum { ROI_BF16 = 0, ROI_FP32 = 1 } roi_dtype;

/*
 * roi_quantize_rows -- symmetric int8 rows with one scale each, by a fixed
 * sequence of IEEE fp32 operations, so that the integers are reproducible:
 *   amax = max_c |x[c]|,
 *   scale = min(max(fl(amax / 127), 2^-126), 0x1.020406p+121)  (the largest fp32
 *          value whose 127-fold is finite: only amax = FLT_MAX is cut to it),
 *   inv  = fl(127 fl(1 / amax)), or 2^126 where scale is 2^-126,
 *   q[c] = rint(fl(x[c] inv))            (ties to even; -127 .. 127).
 * inv is 127 / amax to within 2^-23 of it (2^-21 for amax above 2^126, whose
 * reciprocal is subnormal), so x inv is within 2^-14 of a step of x / scale.
 * A row of zeros gets q = 0.  A row that holds a NaN or an infinity gets
 * q = 0 and scale = NaN, so that everything computed from that row is NaN.
 *  x     bf16 or fp32 [rows, cols] (read; dtype says which)
 *  q     int8 [rows, cols]         (written)
 *  scale fp32 [rows]               (written)
 * rows and cols here are those of x (below 2^31).
 */
int roi_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int8_t* q,
                      float* scale, hipStream_t stream);
/*
 * roi_dequantize_rows -- x[r, c] = q[r, c] scale[r], one fp32 product, rounded
 * to nearest where x is bf16.  Arguments as above, q and scale read, x written.
 */
int roi_dequantize_rows(const int8_t* q, const float* scale, int64_t rows, int64_t cols, void* x,
                        int dtype, hipStream_t stream);

/*
 * roi_linear_i8 -- y[t, r] = xs[t] ws[r] sum_c xq[t, c] wq[r, c] (+ bias[r]).
 * The sum is exact in int32 (cols <= 131071, so that no int8 values can
 * overflow it); then fl(fl(fl(sum) ws) xs), the bias added, in fp32, and one
 * rounding to y's type.  fl(sum) is exact up to 2^24.  Where |sum| ws passes the
 * largest fp32 value, y is infinite, also if xs would bring it back; with ws
 * below 2^97 (weights below 2e31) no sum does that.
 *  xq    int8 [tokens, cols], xs fp32 [tokens]  (roi_quantize_rows)
 *  wq    int8 [rows, cols], or with meta int8 [rows, cols / 2]: the two kept
 *        values of every group of four in increasing index order (the rows of
 *        roi_mask_export's values at 2:4, quantized)
 *  meta  NULL, or roi_mask_export's 2:4 metadata uint32 [rows * cols / 32];
 *        needs cols % 32 == 0 (a row's words are its own)
 *  ws    fp32 [rows]
 *  bias  bf16 [rows] or NULL
 *  y     bf16 or fp32 [tokens, rows] (written; dtype says which)
 */
int64_t roi_linear_i8_workspace(int64_t tokens, int64_t rows, int64_t cols, int packed);
int roi_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq, const uint32_t* meta,
                  const float* ws, const uint16_t* bias, int64_t tokens, int64_t rows,
                  int64_t cols, void* y, int dtype, void* workspace, int64_t workspace_bytes,
                  hipStream_t stream);

/*
 * The gradients of that product, straight through its rounding.
 * roi_linear_i8_grad_weight: grad_w[r, c] = sum_t grad_y[t, r] xs[t] xq[t, c],
 * the dL/dW_masked that roi_mask_bwd takes, from the checkpoint (xq, xs).
 * roi_linear_i8_grad_input:  grad_x[t, c] = sum_r grad_y[t, r] ws[r] wq[r, c]
 * (wq dense).  The scaled int8 operand is rounded once to bf16 (the value that
 * roi_dequantize_rows gives in bf16, and what the bf16 matrix cores take);
 * products and sums are fp32, and the result is rounded to bf16.
 *  grad_y bf16 [tokens, rows] (read)
 *  grad_w bf16 [rows, cols], grad_x bf16 [tokens, cols] (overwritten)
 */
int64_t roi_linear_i8_grad_weight_workspace(int64_t tokens, int64_t rows, int64_t cols);
int roi_linear_i8_grad_weight(const uint16_t* grad_y, const int8_t* xq, const float* xs,
                              int64_t tokens, int64_t rows, int64_t cols, uint16_t* grad_w,
                              void* workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t roi_linear_i8_grad_input_workspace(int64_t tokens, int64_t rows, int64_t cols);
int roi_linear_i8_grad_input(const uint16_t* grad_y, const int8_t* wq, const float* ws,
                             int64_t tokens, int64_t rows, int64_t cols, uint16_t* grad_x,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * Operands in 8-bit floats, with one power-of-two scale for each block of 128
 * values: the layer's products with all operands in 8 bits (forward and both
 * gradients), and the moments of roi_adamw_grouped.
 *
 * Blocks run along a tensor's rows: 128 consecutive values of a row ("rows"), or
 * 128 of each of 128 rows ("square": a weight's, whose transposition has the
 * transposed scales).  The last ones may be shorter.  With a the largest finite
 * magnitude of a block, as fp32, and E its biased exponent, one more where the
 * fraction of a is over 3/4, less 8 (e4m3) or 15 (e5m2), at least 1:
 *   scale = 2^(E - 127), held as the byte E;
 *   q = x 2^(127 - E), rounded to the format's nearest, ties to even.
 * The product is exact (but for subnormal results), so the bytes are
 * reproducible, and no magnitude passes the format's largest (448 of e4m3,
 * 57344 of e5m2).  A NaN becomes one of the format's; an infinity stays one in
 * e5m2 and becomes a NaN in e4m3, which has none; neither changes its neighbours
 * or the scale.  A block of zeros has E = 1.
 *
 * Layout
 *  - q: bytes, rows q_stride bytes apart, a multiple of 16 and at least the row;
 *    what lies between a row's end and the next row is left alone.  Rows are read
 *    in whole pieces of up to 16 bytes, so that the bytes behind a row's end up
 *    to the next multiple of 16 are read, and not used.
 *  - scale: bytes E, a row of them for each row (or 128 rows) of the tensor, each
 *    of roi_block_scales(cols) bytes: whole 32-bit words, 127 behind the last
 *    block's.  Aligned to 4 bytes, so that a batch may be cut at any token whose
 *    q is 16-byte aligned.  The products take E from 1 to 254 (0 is 2^-127, 255 a
 *    NaN).
 */
typedef enum { ROI_E4M3 = 0, ROI_E5M2 = 1 } roi_f8;

/* Bytes of scales of a row of cols values: 4 ceil(cols / 512). */
int64_t roi_block_scales(int64_t cols);

/*
 * roi_quantize_blocks -- x to 8-bit floats, and on request its transposed copy.
 *  x        bf16 or fp32 [rows, cols] (read; dtype says which)
 *  square   0: blocks of rows; 1: square blocks
 *  format   ROI_E4M3 or ROI_E5M2
 *  q        [rows, cols], rows q_stride apart    (written)
 *  scale    [rows or ceil(rows / 128), roi_block_scales(cols)]   (written)
 *  qt       NULL, or [cols, rows], rows qt_stride apart: the transposed x with
 *           blocks of its own, along the rows of x (what a sum over x's rows
 *           takes); with square blocks the transposed q   (written)
 *  scale_t  with qt: [cols or ceil(cols / 128), roi_block_scales(rows)] (written)
 * rows and cols are below 2^31.
 */
int roi_quantize_blocks(const void* x, int dtype, int64_t rows, int64_t cols, int square,
                        int format, uint8_t* q, int64_t q_stride, uint8_t* scale, uint8_t* qt,
                        int64_t qt_stride, uint8_t* scale_t, hipStream_t stream);
/*
 * roi_dequantize_blocks -- x = q 2^(E - 127) in fp32 (exact), rounded to nearest
 * where x is bf16 (exact too, but for subnormals).  A value that was within 1/32
 * (e4m3) or 1/16 (e5m2) of 2^128 is rounded up to it and comes back as an infinity.
 * Arguments as above, q and scale read, x written.
 */
int roi_dequantize_blocks(const uint8_t* q, int64_t q_stride, const uint8_t* scale, int64_t rows,
                          int64_t cols, int square, int format, void* x, int dtype,
                          hipStream_t stream);

/*
 * roi_linear_f8 -- y[t, r] = sum_c x[t, c] w[r, c] (+ bias[r]) of x and w in
 * blocks, both with their blocks along the sum.  The gradients of the layer are
 * the same product of transposed copies (roi_quantize_blocks' qt):
 *   dL/dx [t, c]: xq = dL/dy quantized, wq = the weight's qt (square blocks);
 *   dL/dW [r, c]: xq = dL/dy's qt, wq = the qt of the forward's x (blocks of rows).
 * Products of 8-bit floats are exact; the matrix cores cut those of eight
 * neighbours in the sum below 2^-13 of the largest one's power of two and add
 * up in fp32 (in sums of normal values 1.5e-5 of the result), so y is bf16 only,
 * rounded to nearest after the bias is added in fp32.  A NaN in a row of xq or wq
 * makes that row (column) of y NaN.
 *  xq       [tokens, cols], rows x_stride apart, in x_format
 *  xs       scales of its blocks of rows [tokens, roi_block_scales(cols)]
 *  wq       e4m3 [rows, cols], rows w_stride apart
 *  ws       its scales: square blocks' with w_square 1, else those of rows
 *  bias     bf16 [rows] or NULL
 *  y        bf16 [tokens, rows]  (written)
 *  workspace as in the int8 layer's conventions; tokens, rows and cols too
 *  (tokens below 2^30, rows and cols below 2^22, the strides at most that; in a
 *  weight's gradient the sum's cols are tokens).
 */
int64_t roi_linear_f8_workspace(int64_t tokens, int64_t rows, int64_t cols);
int roi_linear_f8(const uint8_t* xq, int64_t x_stride, const uint8_t* xs, int x_format,
                  const uint8_t* wq, int64_t w_stride, const uint8_t* ws, int w_square,
                  const uint16_t* bias, int64_t tokens, int64_t rows, int64_t cols, uint16_t* y,
                  void* workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * roi_adamw_grouped -- one AdamW step of `count` separately allocated tensors
 * from their gradients: the formulas of roi_mask_bwd_adamw, for logits whose
 * gradient does not come from one call of the item sampler's backward (summed
 * over micro-batches, the categorical sampler's) and for other parameters.
 *
 * bits 32: exp_avg = m and exp_avg_sq = v, fp32 [numel]; v' past fp32's largest
 * number, as |grad| above 2^64 makes it, is an infinity.
 * bits 8: m and the root of v, each in e4m3 [numel] with a scale byte for each
 * 128 consecutive values (the format above, a tensor being one row), for all finite
 * gradients:
 *   m = exp_avg 2^(avg_scale - 127), v = (exp_avg_sq 2^(sq_scale - 127))^2.
 * param's step is taken in fp32.  m' and sqrt(v') are stored with new scales as 64
 * bits give them, rounded up or down with the chance that their distance says, so
 * that they are kept in the mean (rounding to nearest would hold v where a step
 * changes its root by less than half of an e4m3 step, 3 to 6 %).  The chance's bits
 * are those of the noise word x of global element e = elem_offset + i (conventions
 * above): with t = |value| 2^(127 - E) and u the spacing of e4m3 values at t (2^-9 below
 * 2^-6), the stored value is floor(t / u + b) u, b = (x >> 12) 2^-20 for the
 * root and (x mod 2^12) 2^-12 for m.  A root above 0 is stored as 2^-9 at least:
 * m is not divided by eps alone.  A NaN or an infinity is stored as NaN and
 * changes no other element.  Use a (seed, step) of its own for each step; the
 * sampler's seed would tie the rounding to the sampler's noise.
 *
 *  param      fp32 [numel]  (read, overwritten)
 *  grad       fp32 or bf16 [numel] (read; grad_dtype says which for all tensors)
 *  exp_avg, exp_avg_sq  as above (read, overwritten)
 *  avg_scale, sq_scale  bits 8: [roi_block_scales(numel)] bytes each, 4-byte
 *             aligned (read, overwritten; those behind the last block's are
 *             left alone); bits 32: not looked at
 *  numel      >= 0, below 2^40 (a tensor of none is skipped)
 *  elem_offset % 4 == 0; only bits 8 use it, as they do seed and step
 *  opt        as in roi_mask_bwd_adamw, in 64 bits: each of beta and 1 - beta is
 *             rounded to fp32 once; eps is at least 2^-126.  Second moments below
 *             2^-120, and first moments of a block with none above 2^-110, may be
 *             those of fp32, or 0.  It is read during the call, as `tensors` are: a
 *             captured call replays with the settings, seed and step it was given
 * No output may overlap another tensor's or an input.  State starts as zeros
 * (the scale bytes may be zeros too).
 */
typedef struct {
    double lr;
    double beta1, beta2;
    double eps;
    double weight_decay;
    int64_t t;
} roi_step_params;

typedef struct {
    float* param;
    const void* grad;
    void* exp_avg;
    void* exp_avg_sq;
    uint8_t* avg_scale;
    uint8_t* sq_scale;
    int64_t numel;
    uint64_t elem_offset;
} roi_step_tensor;

int roi_adamw_grouped(const roi_step_tensor* tensors, int count, int grad_dtype, int bits,
                      uint64_t seed, uint64_t step, const roi_step_params* opt,
                      hipStream_t stream);

/*
 * roi_gumbel_noise -- the noise of `count` consecutive elements starting at
 * global index elem_offset (elem_offset % 4 == 0): the raw Philox words
 * and/or g = -L(-L(u)) (Algorithm 1).  Either output may be NULL, not both.
 *  words  uint32 [count] or NULL; gumbel fp32 [count] or NULL
 */
int roi_gumbel_noise(uint64_t seed, uint64_t step, uint64_t elem_offset, int64_t count,
                     uint32_t* words, float* gumbel, hipStream_t stream);

/*
 * roi_gumbel_from_words -- g = -L(-L(u(x))) for caller-given 32-bit words x
 * (Algorithm 1 applied to explicit uniforms; exposes the deterministic noise
 * transform on its own).  words uint32 [count] (read), gumbel fp32 [count]
 * (written).
 */
int roi_gumbel_from_words(const uint32_t* words, int64_t count, float* gumbel,
                          hipStream_t stream);

/*
 * roi_fast_noise_from_words -- the noise in log2 units from the hardware
 * logarithm, K(x) = -log2(-log2 u(x)) = g log2(e) + log2(ln 2) up to a few
 * ulp: the form the straight-through forwards use for their key comparisons,
 * falling back to the exact keys whenever two keys are closer than the proven
 * bound of this form's error (no relaxation uses it).  words uint32 [count]
 * (read), out fp32 [count] (written).
 */
int roi_fast_noise_from_words(const uint32_t* words, int64_t count, float* out, hipStream_t stream);

/*
 * roi_anneal -- §4.2.3 exponential annealing, host-side:
 * v_t = max{ v_end, v_init (v_end / v_init)^(t / t_anneal) }, evaluated in
 * fp64 and rounded to fp32.  Requires v_init > 0, v_end > 0, t >= 0,
 * t_anneal > 0; returns NaN otherwise.
 */
float roi_anneal(float v_init, float v_end, int64_t t, int64_t t_anneal);

/*
 * roi_stream_copy -- not part of the method: a plain copy of nbytes from src
 * to dst (device pointers, 16-byte aligned, not overlapping; nbytes a
 * multiple of 16), with the sampler kernels' access pattern: 16 bytes per
 * lane, non-temporal loads and stores, one pass of a one-shot grid.  The
 * benchmark times it as the same GPU's achievable streaming bandwidth.
 * Asynchronous on stream; ROI_E_INVAL for bad arguments before any launch.
 */
int roi_stream_copy(const void* src, void* dst, int64_t nbytes, hipStream_t stream);

/* Static description of a status code. */
const char* roi_status_string(int status);
/* Thread-local detail of the last failed call on this thread ("" if none). */
const char* roi_last_error(void);
/* ABI version, currently 1. */
int roi_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ROI_H */
