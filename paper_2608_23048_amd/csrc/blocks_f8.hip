// blocks_f8.hip -- gfx950 kernels of the operands in 8-bit floats:
// quantize_blocks and dequantize_blocks.
//
// E from the largest finite magnitude of 128 (or 128 x 128) values, q = x 2^(127 - E)
// rounded by the conversion instruction (to nearest, ties to even): some ten
// instructions a value.  Bound by HBM: a value is read once (2 or 4 bytes) and
// written once a copy (1 byte).
#include <hip/hip_runtime.h>

#include "f8.hpp"
#include "host.hpp"
#include "roi.h"

namespace roi {
namespace {

// Elements k .. k + 7 of a row of `cols`, zeros past its end.
template <typename T>
__device__ __forceinline__ void load_eight_f32(const T* row, int64_t k, int64_t cols, float (&f)[8])
{
    struct Eight {
        uint32_t w[2 * sizeof(T)];
    } e{};
    if (k + 8 <= cols) {
        e = load_any<Eight>(row + k);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols)
                e.w[i * sizeof(T) / 4] |= (uint32_t)row[k + i] << (8 * (i * sizeof(T) % 4));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2)
            f[i] = __uint_as_float(i & 1 ? e.w[i / 2] & 0xFFFF0000u : e.w[i / 2] << 16);
        else
            f[i] = __uint_as_float(e.w[i]);
    }
}

// Bytes k .. k + 7 of a row of `cols`.
__device__ __forceinline__ void store_eight(uint8_t* row, int64_t k, int64_t cols, uint32_t lo,
                                            uint32_t hi)
{
    if (k + 8 <= cols) {
        *reinterpret_cast<u32x2*>(row + k) = u32x2{lo, hi};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols) row[k + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i % 4)));
    }
}

struct QuantizeArgs {
    const void* x;
    uint8_t* q;
    uint8_t* scale;
    uint8_t* qt;
    uint8_t* scale_t;
    int64_t rows, cols, stride, stride_t;
};

// Blocks of rows: a wave takes kUnits times 512 consecutive values of a row (four
// blocks, one word of scales), eight values a lane.
template <typename T, int kFormat>
__global__ __launch_bounds__(256) void quantize_rows_f8_kernel(QuantizeArgs a, int64_t per_row)
{
    constexpr int kUnits = 4;
    const int lane = threadIdx.x & 63;
    const int64_t units = a.rows * per_row;
    for (int64_t u = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kUnits; u < units;
         u += (int64_t)gridDim.x * 4 * kUnits) {
        float f[kUnits][8];
        int64_t r = u / per_row, c = u - r * per_row;
        const int64_t r0 = r, c0 = c;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (u + i < units)
                load_eight_f32(static_cast<const T*>(a.x) + r * a.cols, c * 512 + lane * 8, a.cols,
                               f[i]);
            if (++c == per_row) {
                c = 0;
                ++r;
            }
        }
        r = r0;
        c = c0;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (u + i < units) {
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = most(m, finite_bits(f[i][e]));
                const int byte = scale_byte<kFormat>(most_of_16(m));
                const float inv = inverse_scale(byte);
                const int64_t k = c * 512 + lane * 8;
                store_eight(a.q + r * a.stride, k, a.cols,
                            to_f8x4<kFormat>(f[i][0] * inv, f[i][1] * inv, f[i][2] * inv, f[i][3] * inv),
                            to_f8x4<kFormat>(f[i][4] * inv, f[i][5] * inv, f[i][6] * inv, f[i][7] * inv));
                uint32_t word = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    word |= (c * 512 + b * kF8Block < a.cols
                                 ? (uint32_t)__builtin_amdgcn_readlane(byte, 16 * b)
                                 : (uint32_t)kNoScale)
                            << (8 * b);
                if (lane == 0) reinterpret_cast<uint32_t*>(a.scale)[r * per_row + c] = word;
            }
            if (++c == per_row) {
                c = 0;
                ++r;
            }
        }
    }
}

// A block takes 128 x 128 values; thread (g, c) of 16 x 16 those of rows 8 g .. 8 g + 7
// and columns 8 c .. 8 c + 7.  The transposed bytes pass LDS: eight rows of a
// column are a piece of 8 bytes, piece g of column k at place g ^ (k / 8), so that
// the 16 lanes of equal g cover all banks.
template <typename T, int kFormat, bool kSquare>
__global__ __launch_bounds__(256) void quantize_tile_f8_kernel(QuantizeArgs a, int64_t tiles_c,
                                                               int64_t tiles)
{
    __shared__ __attribute__((aligned(16))) uint8_t out[128 * 128];
    __shared__ uint32_t part[4][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = threadIdx.x / 16, c = threadIdx.x % 16;
    const int64_t scales = (a.cols + 511) / 512 * 4, scales_t = (a.rows + 511) / 512 * 4;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t tr = tile / tiles_c, tc = tile - tr * tiles_c;
        const int64_t r0 = tr * 128 + 8 * g, k0 = tc * 128 + 8 * c;
        float f[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i < a.rows) {
                load_eight_f32(static_cast<const T*>(a.x) + (r0 + i) * a.cols, k0, a.cols, f[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[i][e] = 0.0f;
            }
        }
        uint32_t row_most[8], col_most[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row_most[i] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = finite_bits(f[i][e]);
                row_most[i] = most(row_most[i], b);
                col_most[e] = most(col_most[e], b);
            }
        }
        int row_byte[8], col_byte[8];
        if constexpr (kSquare) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = most(m, col_most[e]);
            m = most_of_32(m);
            m = most(m, (uint32_t)__shfl_xor((int)m, 32));
            if (lane == 0) part[wave][0] = m;
            __syncthreads();
            m = most(most(part[0][0], part[1][0]), most(part[2][0], part[3][0]));
            const int byte = scale_byte<kFormat>(m);
#pragma unroll
            for (int i = 0; i < 8; ++i) row_byte[i] = col_byte[i] = byte;
            if (threadIdx.x == 0) {
                a.scale[tr * scales + tc] = (uint8_t)byte;
                if (a.qt) a.scale_t[tc * scales_t + tr] = (uint8_t)byte;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                row_byte[i] = scale_byte<kFormat>(most_of_16(row_most[i]));
                if (c == 0 && r0 + i < a.rows) a.scale[(r0 + i) * scales + tc] = (uint8_t)row_byte[i];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t m = most(col_most[e], (uint32_t)__shfl_xor((int)col_most[e], 16));
                m = most(m, (uint32_t)__shfl_xor((int)m, 32));
                if (lane < 16) part[wave][8 * c + e] = m;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 8 * c + e;
                col_byte[e] = scale_byte<kFormat>(
                    most(most(part[0][k], part[1][k]), most(part[2][k], part[3][k])));
                if (g == 0 && k0 + e < a.cols) a.scale_t[(k0 + e) * scales_t + tr] = (uint8_t)col_byte[e];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float inv = inverse_scale(row_byte[i]);
            if (r0 + i < a.rows)
                store_eight(a.q + (r0 + i) * a.stride, k0, a.cols,
                            to_f8x4<kFormat>(f[i][0] * inv, f[i][1] * inv, f[i][2] * inv, f[i][3] * inv),
                            to_f8x4<kFormat>(f[i][4] * inv, f[i][5] * inv, f[i][6] * inv, f[i][7] * inv));
        }
        if (a.qt) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float inv = inverse_scale(col_byte[e]);
                const u32x2 v = {
                    to_f8x4<kFormat>(f[0][e] * inv, f[1][e] * inv, f[2][e] * inv, f[3][e] * inv),
                    to_f8x4<kFormat>(f[4][e] * inv, f[5][e] * inv, f[6][e] * inv, f[7][e] * inv)};
                *reinterpret_cast<u32x2*>(out + (8 * c + e) * 128 + ((g ^ c) * 8)) = v;
            }
            __syncthreads();
            // eight lanes a column, 16 rows each: pieces 2 p and 2 p + 1
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int k = n * 32 + threadIdx.x / 8, p = threadIdx.x % 8, by = k / 8;
                const u32x4 v = *reinterpret_cast<const u32x4*>(out + k * 128 + (p ^ (by >> 1)) * 16);
                const u32x4 w = by & 1 ? u32x4{v.z, v.w, v.x, v.y} : v;
                const int64_t col = tc * 128 + k, r = tr * 128 + 16 * p;
                if (col < a.cols) {
                    uint8_t* to = a.qt + col * a.stride_t;
                    if (r + 16 <= a.rows) {
                        *reinterpret_cast<u32x4*>(to + r) = w;
                    } else {
                        for (int i = 0; i < 16; ++i)
                            if (r + i < a.rows)
                                to[r + i] = (uint8_t)((i < 8 ? (i < 4 ? w.x : w.y) : (i < 12 ? w.z : w.w)) >>
                                                      (8 * (i % 4)));
                    }
                }
            }
        }
        // the bytes behind the last block's
        const int64_t last_c = (a.cols + 127) / 128, last_r = (a.rows + 127) / 128;
        if (tc == last_c - 1 && last_c < scales) {
            const int64_t first = kSquare ? tr : tr * 128, end = kSquare ? tr + 1 : a.rows;
            for (int64_t r = first + threadIdx.x; r < end && r < first + 128; r += 256)
                for (int64_t k = last_c; k < scales; ++k) a.scale[r * scales + k] = (uint8_t)kNoScale;
        }
        if (a.qt && tr == last_r - 1 && last_r < scales_t) {
            const int64_t first = kSquare ? tc : tc * 128, end = kSquare ? tc + 1 : a.cols;
            for (int64_t k = first + threadIdx.x; k < end && k < first + 128; k += 256)
                for (int64_t r = last_r; r < scales_t; ++r) a.scale_t[k * scales_t + r] = (uint8_t)kNoScale;
        }
        __syncthreads(); // the next tile's shared values
    }
}

// One wave per 512 values of a row, eight a lane.
template <typename T, int kFormat>
__global__ __launch_bounds__(256) void dequantize_f8_kernel(const uint8_t* q, int64_t stride,
                                                            const uint8_t* scale, T* x, int64_t rows,
                                                            int64_t cols, int64_t per_row, int shift)
{
    const int lane = threadIdx.x & 63;
    const int64_t units = rows * per_row;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units;
         u += (int64_t)gridDim.x * 4) {
        const int64_t r = u / per_row, c = u - r * per_row, k = c * 512 + lane * 8;
        if (k >= cols) continue;
        const Pair v = k + 8 <= cols ? load_any<Pair>(q + r * stride + k)
                                     : load_row<Pair>(q + r * stride, k, cols);
        const float s = scale_value(scale[(r >> shift) * (per_row * 4) + k / kF8Block]);
        float f[8];
        float(&lo)[4] = *reinterpret_cast<float(*)[4]>(f);
        float(&hi)[4] = *reinterpret_cast<float(*)[4]>(f + 4);
        from_f8x4<kFormat>(v.w[0], lo);
        from_f8x4<kFormat>(v.w[1], hi);
        struct Eight {
            uint32_t w[2 * sizeof(T)];
        } o;
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) {
            if constexpr (sizeof(T) == 2)
                o.w[i] = bf16x2_rne(f[2 * i] * s, f[2 * i + 1] * s);
            else
                o.w[i] = __float_as_uint(f[i] * s);
        }
        T* out = x + r * cols + k;
        if (k + 8 <= cols) {
            store_any(out, o);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < cols)
                    out[i] = sizeof(T) == 2 ? (T)(o.w[i / 2] >> (16 * (i % 2))) : (T)o.w[i % (2 * sizeof(T))];
        }
    }
}

constexpr int64_t kMostBlocks = 0xFFFFFF; // of 256 threads: a launch has fewer than 2^32

template <typename T, int kFormat>
void quantize_f8(const QuantizeArgs& a, bool square, hipStream_t stream)
{
    if (!square && !a.qt) {
        const int64_t per_row = (a.cols + 511) / 512;
        const int64_t blocks = (a.rows * per_row + 15) / 16;
        hipLaunchKernelGGL((quantize_rows_f8_kernel<T, kFormat>),
                           dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0,
                           stream, a, per_row);
        return;
    }
    const int64_t tiles_c = (a.cols + 127) / 128, tiles = (a.rows + 127) / 128 * tiles_c;
    const dim3 grid((unsigned)(tiles < kMostBlocks ? tiles : kMostBlocks));
    if (square)
        hipLaunchKernelGGL((quantize_tile_f8_kernel<T, kFormat, true>), grid, dim3(256), 0, stream, a,
                           tiles_c, tiles);
    else
        hipLaunchKernelGGL((quantize_tile_f8_kernel<T, kFormat, false>), grid, dim3(256), 0, stream, a,
                           tiles_c, tiles);
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_block_scales(int64_t cols) { return cols > 0 ? (cols + 511) / 512 * 4 : 0; }

extern "C" int roi_quantize_blocks(const void* x, int dtype, int64_t rows, int64_t cols, int square,
                                   int format, uint8_t* q, int64_t q_stride, uint8_t* scale,
                                   uint8_t* qt, int64_t qt_stride, uint8_t* scale_t,
                                   hipStream_t stream)
{
    bool todo;
    if (int st = validate_quantize_f8(x, dtype, rows, cols, square != 0, format, q, q_stride, scale, qt,
                                      qt_stride, scale_t, &todo))
        return st;
    if (!todo) return ok();
    const QuantizeArgs a{x, q, scale, qt, scale_t, rows, cols, q_stride, qt_stride};
    if (dtype == ROI_BF16)
        format == ROI_E4M3 ? quantize_f8<uint16_t, ROI_E4M3>(a, square != 0, stream)
                           : quantize_f8<uint16_t, ROI_E5M2>(a, square != 0, stream);
    else
        format == ROI_E4M3 ? quantize_f8<uint32_t, ROI_E4M3>(a, square != 0, stream)
                           : quantize_f8<uint32_t, ROI_E5M2>(a, square != 0, stream);
    return launch_status("roi_quantize_blocks");
}

extern "C" int roi_dequantize_blocks(const uint8_t* q, int64_t q_stride, const uint8_t* scale,
                                     int64_t rows, int64_t cols, int square, int format, void* x,
                                     int dtype, hipStream_t stream)
{
    bool todo;
    if (int st = validate_dequantize_f8(q, q_stride, scale, rows, cols, square != 0, format, x, dtype,
                                        &todo))
        return st;
    if (!todo) return ok();
    const int64_t per_row = (cols + 511) / 512;
    const int64_t blocks = (rows * per_row + 3) / 4;
    const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks));
    const int shift = square ? 7 : 0;
    auto go = [&](auto kernel, auto* out) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, q, q_stride, scale, out, rows, cols,
                           per_row, shift);
    };
    if (dtype == ROI_BF16)
        format == ROI_E4M3 ? go(dequantize_f8_kernel<uint16_t, ROI_E4M3>, static_cast<uint16_t*>(x))
                           : go(dequantize_f8_kernel<uint16_t, ROI_E5M2>, static_cast<uint16_t*>(x));
    else
        format == ROI_E4M3 ? go(dequantize_f8_kernel<uint32_t, ROI_E4M3>, static_cast<uint32_t*>(x))
                           : go(dequantize_f8_kernel<uint32_t, ROI_E5M2>, static_cast<uint32_t*>(x));
    return launch_status("roi_dequantize_blocks");
}
