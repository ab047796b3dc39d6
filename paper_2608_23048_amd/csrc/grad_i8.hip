// grad_i8.hip -- gfx950 kernels of the two gradients of the int8 product:
//   grad_w[r, c] = sum_t grad_y[t, r] xs[t] xq[t, c]
//   grad_x[t, c] = sum_r grad_y[t, r] ws[r] wq[r, c]
// Both are out[d, c] = sum_k dy(d, k) s[k] q[k, c] with q int8 [K, cols], one
// scale a row, and dy bf16 with its sum index k in rows (the weight gradient:
// dy is [K, D]) or contiguous (the input gradient: dy is [D, K]).
//
// s q is formed in fp32 and rounded once to bf16 on its way to LDS (the other
// operand and the result are bf16, and so are the matrix instructions); the
// products and sums are fp32.  The int8 operand is the matrix instruction's
// first, so that a lane of the result holds four consecutive c of one d: a
// vector store.  Layouts, as measured on gfx950 (lane l, g = l / 16):
//   v_mfma_f32_16x16x32_bf16: operand row l % 16, sum indices 8 g .. 8 g + 7;
//     result rows 4 g .. 4 g + 3 of column l % 16;
//   ds_read_b64_tr_b16: the 16 lanes of a group read a 4 x 16 block, lane i the
//     four values at row i / 4, columns 4 (i % 4) ..; lane i gets column i.
#include <hip/hip_runtime.h>

#include "host.hpp"
#include "mm.hpp"
#include "roi.h"

namespace roi {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 128;   // of out, in d and in c
constexpr int kThreads = 256;
constexpr int kSum = 64;     // sum indices a step
constexpr int kTileBytes = kTile * kRowBytes;
static_assert(kTileBytes == kSum * kTile * 2, "both layouts of dy take the same LDS");

struct Word {
    uint32_t w[1];
};

struct GradArgs {
    const uint16_t* dy;
    const int8_t* q;
    const float* scale;
    uint16_t* out;
    float* partial; // fp32 [splits, D, cols]
    int64_t K, D, cols;
    uint32_t td, tc, splits;
    int64_t steps;
};

// dy's tile of the step at sum index k0 into LDS.  kSumRows: [64 k][128 d], the
// 16-byte chunk j of row k at place j ^ 2 (k & 3), so that the four rows that a
// group of 16 lanes reads together lie in different banks.  Otherwise [128 d]
// k-rows (mm.hpp).  What lies past K or D is zero or repeats the last row.
template <bool kSumRows, bool kWhole>
__device__ __forceinline__ void stage_dy(const GradArgs& a, int64_t k0, int64_t d0,
                                         ROI_LDS uint8_t* dst)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t width = kSumRows ? a.D : a.K; // of a row of dy, in elements
    const uint8_t* base = reinterpret_cast<const uint8_t*>(a.dy) +
                          2 * (kSumRows ? k0 * width + d0 : d0 * width + k0);
#pragma unroll
    for (int i = 0; i < kTileBytes / (16 * kThreads); ++i) {
        const int place = i * kThreads + threadIdx.x;
        int row, chunk;
        if constexpr (kSumRows) {
            row = place / (kTile / 8);
            chunk = (place % (kTile / 8)) ^ (2 * (row & 3));
        } else {
            row = place / 8;
            chunk = (place % 8) ^ (row & 7);
        }
        const int64_t rows_left = kSumRows ? a.K - k0 : a.D - d0;
        const int64_t at = (kSumRows ? d0 : k0) + 8 * chunk; // first element's index in its row
        // a row past the end: zeros where it is summed over, else any row
        const int64_t rr = row < rows_left ? row : rows_left - 1;
        const bool live = (!kSumRows || row < rows_left) && at < width;
        if constexpr (kWhole) {
            load_to_lds(buffer_at(base), live ? (uint32_t)(2 * (rr * width + 8 * chunk)) : kNowhere,
                        dst + (i * kThreads + wave * 64) * 16);
        } else {
            const uint8_t* p = base + 2 * (rr * width - (kSumRows ? d0 : k0));
            lds_write(dst + place * 16, live ? load_row<Quad>(p, 2 * at, 2 * width) : Quad{});
        }
    }
}

// The int8 tile of a step: thread `item` takes eight sum indices of four
// columns, and writes each column's eight values as one 16-byte chunk of that
// column's k-row.  Chunk j of row c lies at place j ^ ((c ^ c / 4) & 7): any
// eight lanes that write (c = 4 lane + i) or read (consecutive c) meet eight
// different places.
__device__ __forceinline__ int q_place(int c, int chunk)
{
    return c * kRowBytes + (chunk ^ ((c ^ (c >> 2)) & 7)) * 16;
}

struct QTile {
    uint32_t v[8];
    float s[8];
};

template <bool kWhole>
__device__ __forceinline__ QTile load_q(const GradArgs& a, int64_t k0, int64_t c0)
{
    const int oct = threadIdx.x / (kTile / 4), group = threadIdx.x % (kTile / 4);
    const int64_t c = c0 + 4 * group;
    QTile t;
    const uint8_t* base = reinterpret_cast<const uint8_t*>(a.q) + k0 * a.cols + c0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = 8 * oct + j;
        const bool live = k0 + row < a.K && c < a.cols;
        t.s[j] = live ? a.scale[k0 + row] : 0.0f;
        if constexpr (kWhole)
            t.v[j] = __builtin_amdgcn_raw_buffer_load_b32(
                buffer_at(base), live ? (uint32_t)(row * a.cols + 4 * group) : kNowhere, 0, 0);
        else
            t.v[j] = live ? load_row<Word>(base + row * a.cols - c0, c, a.cols).w[0] : 0;
    }
    return t;
}

__device__ __forceinline__ void write_q(const QTile& t, ROI_LDS uint8_t* dst)
{
    const int oct = threadIdx.x / (kTile / 4), group = threadIdx.x % (kTile / 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float)(int8_t)(t.v[j] >> (8 * i)) * t.s[j];
        lds_write(dst + q_place(4 * group + i, oct),
                  Quad{bf16x2_rne(f[0], f[1]), bf16x2_rne(f[2], f[3]), bf16x2_rne(f[4], f[5]),
                       bf16x2_rne(f[6], f[7])});
    }
}

__device__ __forceinline__ void store4(const GradArgs& a, int64_t d, int64_t c, f32x4 v)
{
    uint16_t* p = a.out + d * a.cols + c;
    if (c + 4 <= a.cols) {
        store_any(p, Pair{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])});
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < a.cols) p[i] = (uint16_t)bf16x2_rne(v[i], 0.0f);
    }
}

template <bool kSumRows, bool kWhole>
__global__ __launch_bounds__(kThreads) void grad_tile_kernel(GradArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0][0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = (wave >> 1) * 64, wd = (wave & 1) * 64;
    uint32_t td, tc;
    tile_at(xcd_order(blockIdx.x, a.td * a.tc), a.td, a.tc, 8, td, tc);
    const int64_t d0 = (int64_t)td * kTile, c0 = (int64_t)tc * kTile;

    f32x4 acc[4][4] = {};
    if (a.steps > 0) {
        stage_dy<kSumRows, kWhole>(a, 0, d0, base + kTileBytes);
        write_q(load_q<kWhole>(a, 0, c0), base);
    }
    __syncthreads();
    for (int64_t s = 0; s < a.steps; ++s) {
        ROI_LDS uint8_t* cur = base + (s & 1) * 2 * kTileBytes;
        ROI_LDS uint8_t* nxt = base + (~s & 1) * 2 * kTileBytes;
        const bool more = s + 1 < a.steps;
        QTile next{};
        if (more) {
            stage_dy<kSumRows, kWhole>(a, (s + 1) * kSum, d0, nxt + kTileBytes);
            next = load_q<kWhole>(a, (s + 1) * kSum, c0);
        }
        ROI_LDS uint8_t* dyt = cur + kTileBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 q[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[i] = lds_read<bf16x8>(cur + q_place(wc + 16 * i + (lane & 15), 4 * h + g));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kSumRows) {
                    typedef short i16x8 __attribute__((ext_vector_type(8)));
                    const int row = 32 * h + 8 * g + ((lane & 15) >> 2);
                    const int chunk = (wd + 16 * j) / 8 + ((lane & 3) >> 1);
                    ROI_LDS uint8_t* p = dyt + row * (2 * kTile) +
                                         (chunk ^ (2 * (row & 3))) * 16 + (lane & 1) * 8;
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ROI_LDS i16x4*)p);
                    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (ROI_LDS i16x4*)(p + 4 * (2 * kTile)));
                    const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    y[j] = __builtin_bit_cast(bf16x8, both);
                } else {
                    y[j] = lds_read<bf16x8>(dyt + (wd + 16 * j + (lane & 15)) * kRowBytes +
                                            ((4 * h + g) ^ (lane & 7)) * 16);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[i], y[j], acc[i][j], 0, 0, 0);
        }
        if (more) write_q(next, nxt);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t d = d0 + wd + 16 * j + (lane & 15);
        if (d >= a.D) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + wc + 16 * i + 4 * g;
            if (c < a.cols) store4(a, d, c, acc[i][j]);
        }
    }
}

template <bool kSumRows>
int launch(GradArgs a, const char* what, hipStream_t stream)
{
    const Cut c = cut_product(a.D, a.cols, a.K, kSum);
    if (c.tm * c.tn > (int64_t)(0xFFFFFFFFu / kThreads))
        return fail(ROI_E_UNSUPPORTED, "the gradient has too many elements for one call");
    a.td = (uint32_t)c.tm;
    a.tc = (uint32_t)c.tn;
    a.splits = 1;
    a.steps = c.steps;
    const dim3 grid((unsigned)(c.tm * c.tn));
    // 16-byte chunks of dy's rows and 4-byte words of q's that end with the row
    const bool whole = (kSumRows ? a.D : a.K) % 8 == 0 && a.cols % 4 == 0;
    if (whole)
        hipLaunchKernelGGL((grad_tile_kernel<kSumRows, true>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((grad_tile_kernel<kSumRows, false>), grid, dim3(kThreads), 0, stream, a);
    return launch_status(what);
}

int64_t workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    if (check_linear_sizes(tokens, rows, cols)) return -1;
    ok();
    return 0;
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_i8_grad_weight_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    return workspace(tokens, rows, cols);
}

extern "C" int64_t roi_linear_i8_grad_input_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    return workspace(tokens, rows, cols);
}

extern "C" int roi_linear_i8_grad_weight(const uint16_t* grad_y, const int8_t* xq, const float* xs,
                                         int64_t tokens, int64_t rows, int64_t cols,
                                         uint16_t* grad_w, void* workspace, int64_t workspace_bytes,
                                         hipStream_t stream)
{
    bool todo;
    if (int st = validate_grad_i8(grad_y, xq, xs, tokens, tokens, rows, cols, grad_w, rows,
                                  workspace, workspace_bytes, 0, &todo))
        return st;
    if (!todo) return ok();
    const GradArgs a{grad_y, xq, xs, grad_w, static_cast<float*>(workspace), tokens, rows, cols,
                     0, 0, 1, 0};
    return launch<true>(a, "roi_linear_i8_grad_weight", stream);
}

extern "C" int roi_linear_i8_grad_input(const uint16_t* grad_y, const int8_t* wq, const float* ws,
                                        int64_t tokens, int64_t rows, int64_t cols,
                                        uint16_t* grad_x, void* workspace, int64_t workspace_bytes,
                                        hipStream_t stream)
{
    bool todo;
    if (int st = validate_grad_i8(grad_y, wq, ws, rows, tokens, rows, cols, grad_x, tokens,
                                  workspace, workspace_bytes, 0, &todo))
        return st;
    if (!todo) return ok();
    const GradArgs a{grad_y, wq, ws, grad_x, static_cast<float*>(workspace), rows, tokens, cols,
                     0, 0, 1, 0};
    return launch<false>(a, "roi_linear_i8_grad_input", stream);
}
