// linear_f8.hip -- gfx950 kernels of the product of operands in 8-bit floats,
// y[t, r] = sum_b 2^(xs[t, b] + ws[r, b] - 254) sum_{c in block b} xq[t, c] wq[r, c].
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes the sum of one block of 128 and applies
// both scales to it.  The weight's rows are its first operand and the tokens' its
// second, so that a lane of the result holds four consecutive rows of one token.
// Layout, as measured on gfx950 (lane l, g = l / 16): operand row l % 16, 32 of
// the 128 values, in any order that is the same in both operands; result rows
// 4 g .. 4 g + 3 of column l % 16.
#include <hip/hip_runtime.h>

#include "f8.hpp"
#include "host.hpp"
#include "mm.hpp"
#include "roi.h"

namespace roi {
namespace {

struct LinearF8Args {
    const uint8_t* x;
    const uint8_t* xs;
    const uint8_t* w;
    const uint8_t* ws;
    const uint16_t* bias;
    uint16_t* y;
    int64_t x_stride, w_stride;
    int tokens, rows, cols;
    int scales;  // bytes of a row of scales
    int w_shift; // a row r of the weight has scales row r >> w_shift
};

template <int kFormat>
__device__ __forceinline__ f32x4 multiply_block(i32x8 w, i32x8 x, f32x4 sum, int ws, int xs)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, sum, 0, kFormat, 0, ws, 0, xs);
}

// Rows r .. r + 3 of token t.
__device__ __forceinline__ void finish_f8(const LinearF8Args& a, int64_t t, int r, f32x4 v)
{
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < a.rows) v[i] += bf16_bits_to_float(a.bias[r + i]);
    }
    uint16_t* y = a.y + t * a.rows + r;
    if (r + 4 <= a.rows) {
        store_any(y, Pair{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])});
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < a.rows) y[i] = (uint16_t)bf16x2_rne(v[i], 0.0f);
    }
}

// 32 rows x 32 tokens a wave, operands straight from memory.
template <int kFormat>
__global__ __launch_bounds__(256) void linear_f8_kernel(LinearF8Args a, uint32_t tiles_r, int64_t tiles)
{
    const int lane = threadIdx.x & 63, in = lane & 15, g = lane >> 4;
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int r0 = (int)(tile % tiles_r) * 32;
    const int64_t t0 = tile / tiles_r * 32;
    const uint8_t *w[2], *x[2], *ws[2], *xs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = least(r0 + 16 * i + in, a.rows - 1), t = least((int)t0 + 16 * i + in, a.tokens - 1);
        w[i] = a.w + r * a.w_stride;
        ws[i] = a.ws + (int64_t)(r >> a.w_shift) * a.scales;
        x[i] = a.x + t * a.x_stride;
        xs[i] = a.xs + (int64_t)t * a.scales;
    }
    f32x4 acc[2][2] = {};
    for (int k = 0; k < a.cols; k += 128) {
        i32x8 fw[2], fx[2];
        int sw[2], sx[2];
        auto load = [&](const uint8_t* row) {
            const Quad lo = load_row<Quad>(row, k + 32 * g, a.cols);
            const Quad hi = load_row<Quad>(row, k + 32 * g + 16, a.cols);
            return i32x8{(int)lo.w[0], (int)lo.w[1], (int)lo.w[2], (int)lo.w[3],
                         (int)hi.w[0], (int)hi.w[1], (int)hi.w[2], (int)hi.w[3]};
        };
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fw[i] = load(w[i]);
            fx[i] = load(x[i]);
            sw[i] = ws[i][k / 128];
            sx[i] = xs[i][k / 128];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = multiply_block<kFormat>(fw[i], fx[j], acc[i][j], sw[i], sx[j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t t = t0 + 16 * j + in;
            const int r = r0 + 16 * i + 4 * g;
            if (t < a.tokens && r < a.rows) finish_f8(a, t, r, acc[i][j]);
        }
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_f8_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    ok();
    return 0;
}

extern "C" int roi_linear_f8(const uint8_t* xq, int64_t x_stride, const uint8_t* xs, int x_format,
                             const uint8_t* wq, int64_t w_stride, const uint8_t* ws, int w_square,
                             const uint16_t* bias, int64_t tokens, int64_t rows, int64_t cols,
                             uint16_t* y, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    if (int st = validate_linear_f8(xq, x_stride, xs, x_format, wq, w_stride, ws, w_square != 0, bias,
                                    tokens, rows, cols, y, workspace, workspace_bytes, 0, &todo))
        return st;
    if (!todo) return ok();
    const LinearF8Args a{xq, xs, wq, ws, bias, y, x_stride, w_stride, (int)tokens, (int)rows, (int)cols,
                         (int)roi_block_scales(cols), w_square ? 7 : 0};
    const int64_t tiles_r = (rows + 31) / 32, tiles = tiles_r * ((tokens + 31) / 32);
    if ((tiles + 3) / 4 > 0xFFFFFF) return fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
    const dim3 grid((unsigned)((tiles + 3) / 4));
    if (x_format == ROI_E4M3)
        hipLaunchKernelGGL((linear_f8_kernel<ROI_E4M3>), grid, dim3(256), 0, stream, a, (uint32_t)tiles_r, tiles);
    else
        hipLaunchKernelGGL((linear_f8_kernel<ROI_E5M2>), grid, dim3(256), 0, stream, a, (uint32_t)tiles_r, tiles);
    return launch_status("roi_linear_f8");
}
