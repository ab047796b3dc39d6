// linear_i8.hip -- gfx950 kernels of the int8 product
// y[t, r] = xs[t] ws[r] sum_c xq[t, c] wq[r, c] (+ bias[r]), the weight dense
// or 2:4-compressed.
//
// The int8 matrix instructions take the weight's rows as their first operand
// and the tokens' as their second, so that a lane of the result holds four
// consecutive rows r of one token: a vector store of y.  Layouts, as measured
// on gfx950 (lane l, g = l / 16):
//   v_mfma_i32_16x16x64_i8: operand row l % 16, sum indices 16 g .. 16 g + 15;
//     result rows 4 g .. 4 g + 3 of column l % 16.
//   v_smfmac_i32_16x16x128_i8: the first operand's lane holds the 16 kept values
//     of the dense columns 32 g .. 32 g + 31 and its index operand their eight
//     4-bit fields, which is one metadata word; the second's lane holds dense
//     columns 16 g .. 16 g + 15 and 64 + 16 g .. 64 + 16 g + 15; result as above.
#include <hip/hip_runtime.h>

#include "host.hpp"
#include "mm.hpp"
#include "roi.h"

namespace roi {
namespace {

struct LinearArgs {
    const int8_t* x;
    const float* xs;
    const int8_t* w;
    const uint32_t* meta;
    const float* ws;
    const uint16_t* bias;
    void* y;
    int* partial; // int32 [splits, tokens, rows]
    int64_t tokens, rows, cols;
    uint32_t tm, tn, splits; // tiles along the rows and the tokens, parts of the sum
    int64_t steps;
};

// Four results of token t, rows r .. r + 3, from their exact sums.  The scale
// of the weight comes first: sum ws stays far from overflow for any weight.
template <typename Out>
__device__ __forceinline__ void finish4(const LinearArgs& a, int64_t t, int64_t r, i32x4 sum)
{
    Out* y = static_cast<Out*>(a.y) + t * a.rows + r;
    const float xs = a.xs[t];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t ri = r + i < a.rows ? r + i : a.rows - 1;
        v[i] = (float)sum[i] * a.ws[ri] * xs;
        if (a.bias) v[i] += bf16_bits_to_float(a.bias[ri]);
    }
    if (r + 4 <= a.rows) {
        if constexpr (sizeof(Out) == 2)
            store_any(y, Pair{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])});
        else
            store_any(y, Quad{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                              __float_as_uint(v[3])});
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < a.rows) {
                if constexpr (sizeof(Out) == 2)
                    y[i] = (uint16_t)bf16x2_rne(v[i], 0.0f);
                else
                    y[i] = v[i];
            }
    }
}

// ---------------------------------------------------------------- few tokens
// A block owns 16 weight rows and up to 16 kTok tokens; its waves share out the
// sum and add up their parts in LDS.  The weight is read once, straight into
// the matrix instructions' operands: nothing of it is used twice.  Bound by the
// weight's bytes.
constexpr int kFewWaves = 8;

// Operand chunk `k` .. k + 15 of a row of `len` bytes; kGuard: it may pass the
// row's end, where the values are zero.
template <bool kGuard>
__device__ __forceinline__ i32x4 chunk16(const int8_t* row, int64_t k, int64_t len)
{
    const uint8_t* p = reinterpret_cast<const uint8_t*>(row);
    const Quad v = kGuard ? load_row<Quad>(p, k, len) : load_any<Quad>(p + k);
    return i32x4{(int)v.w[0], (int)v.w[1], (int)v.w[2], (int)v.w[3]};
}

// One step of the sum: 128 columns of a dense weight, 256 of a 2:4 one.  A lane
// reads 32 consecutive bytes of its row, as two operands; the sum's order
// within the step is free, as long as both operands follow it.
template <int kTok, bool kPacked, bool kGuard>
__device__ __forceinline__ void few_step(const int8_t* wrow, const uint32_t* mrow,
                                         const int8_t* const (&xrow)[kTok], int64_t k, int64_t cols,
                                         int g, i32x4 (&acc)[kTok])
{
    if constexpr (!kPacked) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t c = k + 32 * g + 16 * h;
            const i32x4 w = chunk16<kGuard>(wrow, c, cols);
#pragma unroll
            for (int j = 0; j < kTok; ++j)
                acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                    w, chunk16<kGuard>(xrow[j], c, cols), acc[j], 0, 0, 0);
        }
    } else {
        // instruction h: operand lane g holds the dense columns 64 g + 32 h ..
        // + 31 of the step, so the second operand's lane g holds 16 columns at
        // 64 (g / 2) + 32 h + 16 (g % 2) and 16 at 128 further on
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t c = k + 64 * g + 32 * h;
            const i32x4 w = chunk16<kGuard>(wrow, c / 2, cols / 2);
            const int idx = !kGuard || c < cols ? (int)mrow[c / 32] : 0x44444444;
            const int64_t b = k + 64 * (g / 2) + 32 * h + 16 * (g % 2);
#pragma unroll
            for (int j = 0; j < kTok; ++j) {
                const i32x4 lo = chunk16<kGuard>(xrow[j], b, cols);
                const i32x4 hi = chunk16<kGuard>(xrow[j], b + 128, cols);
                const i32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                acc[j] = __builtin_amdgcn_smfmac_i32_16x16x128_i8(w, x, acc[j], idx, 0, 0);
            }
        }
    }
}

template <int kTok, bool kPacked, typename Out>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(LinearArgs a)
{
    constexpr int kStep = kPacked ? 256 : 128;
    __shared__ i32x4 part[kFewWaves][kTok][64];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r0 = (int64_t)(blockIdx.x % a.tm) * 16;
    const int64_t t0 = (int64_t)(blockIdx.x / a.tm) * (16 * kTok);
    // rows and tokens past the end repeat the last one; their results are dropped
    const int64_t r = r0 + (lane & 15) < a.rows ? r0 + (lane & 15) : a.rows - 1;
    const int8_t* wrow = a.w + r * (kPacked ? a.cols / 2 : a.cols);
    const uint32_t* mrow = kPacked ? a.meta + r * (a.cols / 32) : nullptr;
    const int8_t* xrow[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        const int64_t t = t0 + 16 * j + (lane & 15);
        xrow[j] = a.x + (t < a.tokens ? t : a.tokens - 1) * a.cols;
    }
    i32x4 acc[kTok] = {};
    const int64_t whole = a.cols / kStep;
    int64_t s = wave;
    for (; s + 3 * kFewWaves < whole; s += 4 * kFewWaves)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            few_step<kTok, kPacked, false>(wrow, mrow, xrow, (s + u * kFewWaves) * kStep, a.cols, g,
                                           acc);
    for (; s < whole; s += kFewWaves)
        few_step<kTok, kPacked, false>(wrow, mrow, xrow, s * kStep, a.cols, g, acc);
    if (whole * kStep < a.cols && wave == (int)(whole % kFewWaves))
        few_step<kTok, kPacked, true>(wrow, mrow, xrow, whole * kStep, a.cols, g, acc);
#pragma unroll
    for (int j = 0; j < kTok; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    for (int j = wave; j < kTok; j += kFewWaves) {
        i32x4 sum = {};
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) sum += part[v][j][lane];
        const int64_t t = t0 + 16 * j + (lane & 15), ro = r0 + 4 * g;
        if (t < a.tokens && ro < a.rows) finish4<Out>(a, t, ro, sum);
    }
}

// --------------------------------------------------------------- many tokens
// A block of 4 waves makes a 128 x 128 tile, each wave 64 x 64, over steps of
// 128 columns.  Two LDS buffers: the next step's tiles load while this one's
// are multiplied.
constexpr int kTile = 128;
constexpr int kThreads = 256;
constexpr int kTileBytes = kTile * kRowBytes;

// The 128-byte k-rows row0 .. row0 + 127 of an operand of `n` rows of `len`
// bytes, from byte k on, into LDS.  kWhole: rows are whole 16-byte chunks.
template <bool kWhole>
__device__ __forceinline__ void stage(const int8_t* p, int64_t row0, int64_t n, int64_t len,
                                      int64_t k, ROI_LDS uint8_t* dst)
{
    const uint8_t* base = reinterpret_cast<const uint8_t*>(p) + row0 * len;
    const int64_t left = n - row0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < kTileBytes / (16 * kThreads); ++i) {
        const int place = i * kThreads + threadIdx.x;
        const int row = place / 8, chunk = (place % 8) ^ (row & 7);
        const int64_t rr = row < left ? row : left - 1; // rows past the end repeat the last
        const int64_t b = k + 16 * chunk;
        if constexpr (kWhole) {
            load_to_lds(buffer_at(base), b < len ? (uint32_t)(rr * len + b) : kNowhere,
                        dst + (i * kThreads + wave * 64) * 16);
        } else {
            lds_write(dst + place * 16, load_row<Quad>(base + rr * len, b, len));
        }
    }
}

template <bool kWhole, typename Out>
__global__ __launch_bounds__(kThreads) void linear_tile_kernel(LinearArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0][0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    uint32_t tm, tn;
    tile_at(xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, 8, tm, tn);
    const int64_t r0 = (int64_t)tm * kTile, t0 = (int64_t)tn * kTile;

    i32x4 acc[4][4] = {};
    if (a.steps > 0) {
        stage<kWhole>(a.w, r0, a.rows, a.cols, 0, base);
        stage<kWhole>(a.x, t0, a.tokens, a.cols, 0, base + kTileBytes);
    }
    __syncthreads();
    for (int64_t s = 0; s < a.steps; ++s) {
        ROI_LDS uint8_t* cur = base + (s & 1) * 2 * kTileBytes;
        ROI_LDS uint8_t* nxt = base + (~s & 1) * 2 * kTileBytes;
        if (s + 1 < a.steps) {
            stage<kWhole>(a.w, r0, a.rows, a.cols, (s + 1) * kRowBytes, nxt);
            stage<kWhole>(a.x, t0, a.tokens, a.cols, (s + 1) * kRowBytes, nxt + kTileBytes);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int place = ((4 * h + g) ^ (lane & 7)) * 16;
            i32x4 w[4], x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = lds_read<i32x4>(cur + (wm + 16 * i + (lane & 15)) * kRowBytes + place);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = lds_read<i32x4>(cur + kTileBytes +
                                       (wn + 16 * i + (lane & 15)) * kRowBytes + place);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] =
                        __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t t = t0 + wn + 16 * j + (lane & 15);
        if (t >= a.tokens) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + wm + 16 * i + 4 * g;
            if (r < a.rows) finish4<Out>(a, t, r, acc[i][j]);
        }
    }
}

// Blocks of one launch: fewer than 2^32 threads.
bool fits(int64_t blocks, int threads) { return blocks <= (int64_t)(0xFFFFFFFFu / (uint32_t)threads); }

template <typename Out>
int launch(LinearArgs a, hipStream_t stream)
{
    if (a.tokens <= 64 || a.meta) {
        const int tok = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
        const int64_t tm = (a.rows + 15) / 16, tn = (a.tokens + 16 * tok - 1) / (16 * tok);
        if (!fits(tm * tn, 64 * kFewWaves))
            return fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
        a.tm = (uint32_t)tm;
        const dim3 grid((unsigned)(tm * tn)), block(64 * kFewWaves);
        auto go = [&](auto dense, auto packed) {
            hipLaunchKernelGGL(a.meta ? packed : dense, grid, block, 0, stream, a);
        };
        if (tok == 1)
            go(linear_few_kernel<1, false, Out>, linear_few_kernel<1, true, Out>);
        else if (tok == 2)
            go(linear_few_kernel<2, false, Out>, linear_few_kernel<2, true, Out>);
        else
            go(linear_few_kernel<4, false, Out>, linear_few_kernel<4, true, Out>);
        return launch_status("roi_linear_i8");
    }
    const Cut c = cut_product(a.rows, a.tokens, a.cols, kRowBytes);
    if (!fits(c.tm * c.tn, kThreads))
        return fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
    a.tm = (uint32_t)c.tm;
    a.tn = (uint32_t)c.tn;
    a.splits = 1;
    a.steps = c.steps;
    const dim3 grid((unsigned)(c.tm * c.tn));
    if (a.cols % 16 == 0)
        hipLaunchKernelGGL((linear_tile_kernel<true, Out>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((linear_tile_kernel<false, Out>), grid, dim3(kThreads), 0, stream, a);
    return launch_status("roi_linear_i8");
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_i8_workspace(int64_t tokens, int64_t rows, int64_t cols, int packed)
{
    if (check_linear_sizes(tokens, rows, cols)) return -1;
    ok();
    return 0;
}

extern "C" int roi_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq,
                             const uint32_t* meta, const float* ws, const uint16_t* bias,
                             int64_t tokens, int64_t rows, int64_t cols, void* y, int dtype,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    bool todo;
    if (int st = validate_linear_i8(xq, xs, wq, meta, ws, bias, tokens, rows, cols, y, dtype,
                                    workspace, workspace_bytes, 0, &todo))
        return st;
    if (!todo) return ok();
    LinearArgs a{xq, xs, wq, meta, ws, bias, y, static_cast<int*>(workspace), tokens, rows, cols,
                 0, 0, 1, 0};
    return dtype == ROI_BF16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}
