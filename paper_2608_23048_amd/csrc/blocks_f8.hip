// blocks_f8.hip -- gfx950 kernels of the operands in 8-bit floats:
// quantize_blocks and dequantize_blocks.
//
// E from the largest finite magnitude of 128 (or 128 x 128) values, q = x 2^(127 - E)
// rounded by the conversion instruction (to nearest, ties to even): some ten
// instructions a value.  Bound by HBM: a value is read once (2 or 4 bytes) and
// written once a copy (1 byte).  8192 x 18944 in bf16: blocks of rows 70 to 89 us (6.6
// to 5.2 TB/s), restored in 66, with the transposed copy 129 to 136, square 118 to 129.
#include <hip/hip_runtime.h>

#include "f8.hpp"
#include "host.hpp"
#include "roi.h"

namespace roi {
namespace {

// kN consecutive elements of a row, as loaded: bf16 two to a word.
template <typename T, int kN>
struct Held {
    uint32_t w[kN * sizeof(T) / 4];

    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 2)
            return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else
            return __uint_as_float(w[i]);
    }
};
// Elements k .. of a row of `cols`, zeros past its end.
template <bool kStream, typename T, int kN>
__device__ __forceinline__ Held<T, kN> load_held(const T* row, int64_t k, int64_t cols)
{
    using H = Held<T, kN>;
    if (k + kN <= cols) return kStream ? stream_load_any<H>(row + k) : load_any<H>(row + k);
    H h{};
#pragma unroll
    for (int i = 0; i < kN; ++i)
        if (k + i < cols) h.w[i * sizeof(T) / 4] |= (uint32_t)row[k + i] << (8 * (i * sizeof(T) % 4));
    return h;
}

// The largest magnitudes of two values in the halves of a word (bf16), or of one
// (fp32); infinities and NaN are above every number.
template <typename T>
__device__ __forceinline__ uint32_t magnitudes(uint32_t w)
{
    return w & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu);
}
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 2) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                      __builtin_bit_cast(u16x2, b)));
    } else {
        return most(a, b);
    }
}
// fp32 bits of the larger of what larger() gives.
template <typename T>
__device__ __forceinline__ uint32_t larger_half(uint32_t m)
{
    return sizeof(T) == 2 ? most(m << 16, m & 0xFFFF0000u) : m;
}
// The largest finite magnitude: what larger() passes over where one is not finite.
template <typename T, int kN>
__device__ __forceinline__ uint32_t largest_finite(const Held<T, kN>& h)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) m = most(m, finite_bits(h.get(i)));
    return m;
}

// Bytes k .. k + 7 (one word: .. k + 3) of a row of `cols`; kPast: past the caches.
template <bool kPast>
__device__ __forceinline__ void store_bytes(uint8_t* row, int64_t k, int64_t cols, uint32_t lo)
{
    if (k + 4 <= cols) {
        if (kPast)
            stream_store(lo, reinterpret_cast<uint32_t*>(row + k));
        else
            *reinterpret_cast<uint32_t*>(row + k) = lo;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < cols) row[k + i] = (uint8_t)(lo >> (8 * i));
    }
}
template <bool kPast>
__device__ __forceinline__ void store_bytes(uint8_t* row, int64_t k, int64_t cols, uint32_t lo,
                                            uint32_t hi)
{
    if (k + 8 <= cols) {
        if (kPast)
            stream_store(u32x2{lo, hi}, reinterpret_cast<u32x2*>(row + k));
        else
            *reinterpret_cast<u32x2*>(row + k) = u32x2{lo, hi};
    } else {
        store_bytes<kPast>(row, k, cols, lo);
        if (k + 4 < cols) store_bytes<kPast>(row, k + 4, cols, hi);
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

// Blocks of rows: a wave takes kOfWave times 512 consecutive values of a row (four
// blocks, one word of scales), 16 bytes a lane and load.  Its results are read soon
// (past the caches, 8192 x 18944 and its restoring take 149 us instead of 143.5).
template <typename T, int kFormat, bool kStream, int kOfWave>
__global__ __launch_bounds__(256) void quantize_rows_f8_kernel(QuantizeArgs a, int64_t per_row)
{
    constexpr int kN = 16 / sizeof(T), kLoads = 512 / (64 * kN);
    const int lane = threadIdx.x & 63;
    const int64_t units = a.rows * per_row;
    for (int64_t u = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kOfWave; u < units;
         u += (int64_t)gridDim.x * 4 * kOfWave) {
        Held<T, kN> h[kOfWave][kLoads];
        int64_t r = u / per_row, c = u - r * per_row;
        const int64_t r0 = r, c0 = c;
#pragma unroll
        for (int i = 0; i < kOfWave; ++i) {
            if (u + i < units) {
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    const int64_t k = c * 512 + (l * 64 + lane) * kN;
                    h[i][l] = load_held<kStream, T, kN>(static_cast<const T*>(a.x) + r * a.cols, k, a.cols);
                }
            }
            if (++c == per_row) {
                c = 0;
                ++r;
            }
        }
        r = r0;
        c = c0;
#pragma unroll
        for (int i = 0; i < kOfWave; ++i) {
            if (u + i < units) {
                uint32_t word = 0;
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    uint32_t m = magnitudes<T>(h[i][l].w[0]);
#pragma unroll
                    for (int e = 1; e < 4; ++e) m = larger<T>(m, magnitudes<T>(h[i][l].w[e]));
                    auto of_block = [](uint32_t v) { return kN == 8 ? most_of_16(v) : most_of_32(v); };
                    m = of_block(larger_half<T>(m));
                    if (__builtin_amdgcn_ballot_w64(m >= kInfinity)) m = of_block(largest_finite(h[i][l]));
                    const int byte = scale_byte<kFormat>(m);
                    const float inv = inverse_scale(byte);
                    const int64_t k = c * 512 + (l * 64 + lane) * kN;
                    uint32_t q[kN / 4];
#pragma unroll
                    for (int e = 0; e < kN; e += 4)
                        q[e / 4] = to_f8x4<kFormat>(h[i][l].get(e) * inv, h[i][l].get(e + 1) * inv,
                                                    h[i][l].get(e + 2) * inv, h[i][l].get(e + 3) * inv);
                    if constexpr (kN == 8)
                        store_bytes<false>(a.q + r * a.stride, k, a.cols, q[0], q[1]);
                    else
                        store_bytes<false>(a.q + r * a.stride, k, a.cols, q[0]);
                    constexpr int kBlocks = kN / 2; // of this load
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) {
                        const int at = l * kBlocks + b;
                        word |= (c * 512 + at * kF8Block < a.cols
                                     ? (uint32_t)__builtin_amdgcn_readlane(byte, 64 / kBlocks * b)
                                     : (uint32_t)kNoScale)
                                << (8 * at);
                    }
                }
                if (lane == 0) reinterpret_cast<uint32_t*>(a.scale)[r * per_row + c] = word;
            }
            if (++c == per_row) {
                c = 0;
                ++r;
            }
        }
    }
}

// A block takes 128 x 128 values; thread (g, c) of 32 x 16 those of rows 4 g .. 4 g + 3
// and columns 8 c .. 8 c + 7: few enough registers for four blocks on a compute unit
// (with twice the rows a thread, and two blocks, 8192 x 18944 took 157 us).  The
// transposed bytes pass LDS: eight rows of a column are a piece of 8 bytes, piece p of
// column k at place p ^ (k / 8), so that a wave's writes cover all banks evenly.  Both
// copies are stored past the caches: 18944 x 3584 in square blocks takes 52.7 us so and
// 55.1 through them, 8192 x 3584 in blocks of rows 25 and 27 to 30.
template <typename T, int kFormat, bool kSquare, bool kStream>
__global__ __launch_bounds__(512) void quantize_tile_f8_kernel(QuantizeArgs a, int64_t tiles_c,
                                                               int64_t tiles)
{
    constexpr int kWords = 2 * sizeof(T);
    __shared__ __attribute__((aligned(16))) uint8_t out[128 * 128];
    __shared__ uint32_t part[8][128];
    __shared__ __attribute__((aligned(8))) uint8_t of_column[128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = threadIdx.x / 16, c = threadIdx.x % 16;
    const int64_t scales = (a.cols + 511) / 512 * 4, scales_t = (a.rows + 511) / 512 * 4;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t tr = tile / tiles_c, tc = tile - tr * tiles_c;
        const int64_t r0 = tr * 128 + 4 * g, k0 = tc * 128 + 8 * c;
        Held<T, 8> h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            h[i] = r0 + i < a.rows ? load_held<kStream, T, 8>(static_cast<const T*>(a.x) + (r0 + i) * a.cols, k0, a.cols)
                                   : Held<T, 8>{};
        uint32_t row_most[4], col_most[kWords];
#pragma unroll
        for (int e = 0; e < kWords; ++e) col_most[e] = 0;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < kWords; ++e) {
                const uint32_t b = magnitudes<T>(h[i].w[e]);
                m = larger<T>(m, b);
                col_most[e] = larger<T>(col_most[e], b);
            }
            row_most[i] = larger_half<T>(m);
            any = most(any, row_most[i]);
        }
        uint32_t col[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            col[e] = sizeof(T) == 2 ? (e & 1 ? col_most[e / 2] & 0xFFFF0000u : col_most[e / 2] << 16)
                                    : col_most[e % kWords];
        if (__builtin_amdgcn_ballot_w64(any >= kInfinity)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) row_most[i] = largest_finite(h[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                col[e] = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) col[e] = most(col[e], finite_bits(h[i].get(e)));
            }
        }
        int row_byte[4], col_byte[8];
        if constexpr (kSquare) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = most(m, row_most[i]);
            m = most_with_32(most_of_32(m));
            if (lane == 0) part[wave][0] = m;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < 8; ++v) m = most(m, part[v][0]);
            const int byte = scale_byte<kFormat>(m);
#pragma unroll
            for (int i = 0; i < 4; ++i) row_byte[i] = byte;
#pragma unroll
            for (int e = 0; e < 8; ++e) col_byte[e] = byte;
            if (threadIdx.x == 0) {
                a.scale[tr * scales + tc] = (uint8_t)byte;
                if (a.qt) a.scale_t[tc * scales_t + tr] = (uint8_t)byte;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = most_with_32(most_with_16(col[e]));
                if (lane < 16) part[wave][8 * c + e] = m;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                row_byte[i] = scale_byte<kFormat>(most_of_16(row_most[i]));
                if (c == 0 && r0 + i < a.rows) a.scale[(r0 + i) * scales + tc] = (uint8_t)row_byte[i];
            }
            __syncthreads();
            // a column's by one thread: all of a column's threads reading the eight waves'
            // took 8192 x 18944 from 113 us to 147
            if (threadIdx.x < 128) {
                uint32_t m = 0;
#pragma unroll
                for (int v = 0; v < 8; ++v) m = most(m, part[v][threadIdx.x]);
                const int byte = scale_byte<kFormat>(m);
                of_column[threadIdx.x] = (uint8_t)byte;
                const int64_t k = tc * 128 + threadIdx.x;
                if (k < a.cols) a.scale_t[k * scales_t + tr] = (uint8_t)byte;
            }
            __syncthreads();
            const u32x2 bytes = *reinterpret_cast<const u32x2*>(of_column + 8 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e) col_byte[e] = (e < 4 ? bytes.x : bytes.y) >> (8 * (e % 4)) & 255;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float inv = inverse_scale(row_byte[i]);
            if (r0 + i < a.rows)
                store_bytes<true>(a.q + (r0 + i) * a.stride, k0, a.cols,
                            to_f8x4<kFormat>(h[i].get(0) * inv, h[i].get(1) * inv, h[i].get(2) * inv, h[i].get(3) * inv),
                            to_f8x4<kFormat>(h[i].get(4) * inv, h[i].get(5) * inv, h[i].get(6) * inv, h[i].get(7) * inv));
        }
        if (a.qt) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float inv = inverse_scale(col_byte[e]);
                *reinterpret_cast<uint32_t*>(out + (8 * c + e) * 128 + (g / 2 ^ c) * 8 + g % 2 * 4) =
                    to_f8x4<kFormat>(h[0].get(e) * inv, h[1].get(e) * inv, h[2].get(e) * inv, h[3].get(e) * inv);
            }
            __syncthreads();
            // eight lanes a column, 16 rows each: pieces 2 p and 2 p + 1
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int k = n * 64 + threadIdx.x / 8, p = threadIdx.x % 8, by = k / 8;
                const u32x4 v = *reinterpret_cast<const u32x4*>(out + k * 128 + (p ^ (by >> 1)) * 16);
                const u32x4 w = by & 1 ? u32x4{v.z, v.w, v.x, v.y} : v;
                const int64_t col_at = tc * 128 + k, r = tr * 128 + 16 * p;
                if (col_at < a.cols) {
                    uint8_t* to = a.qt + col_at * a.stride_t;
                    if (r + 16 <= a.rows) {
                        stream_store(w, reinterpret_cast<u32x4*>(to + r));
                    } else {
                        store_bytes<true>(to, r, a.rows, w.x, w.y);
                        store_bytes<true>(to, r + 8, a.rows, w.z, w.w);
                    }
                }
            }
        }
        // the bytes behind the last block's
        const int64_t last_c = (a.cols + 127) / 128, last_r = (a.rows + 127) / 128;
        if (tc == last_c - 1 && last_c < scales) {
            const int64_t first = kSquare ? tr : tr * 128, end = kSquare ? tr + 1 : a.rows;
            for (int64_t r = first + threadIdx.x; r < end && r < first + 128; r += 512)
                for (int64_t k = last_c; k < scales; ++k) a.scale[r * scales + k] = (uint8_t)kNoScale;
        }
        if (a.qt && tr == last_r - 1 && last_r < scales_t) {
            const int64_t first = kSquare ? tc : tc * 128, end = kSquare ? tc + 1 : a.cols;
            for (int64_t k = first + threadIdx.x; k < end && k < first + 128; k += 512)
                for (int64_t r = last_r; r < scales_t; ++r) a.scale_t[k * scales_t + r] = (uint8_t)kNoScale;
        }
        __syncthreads(); // the next tile's shared values
    }
}

// One wave per kPieces times 1024 bytes of a row of x, which it stores 1024 consecutive
// bytes at a time, past the caches: a lane's piece of q makes 16.  Pieces are read
// whole, past a row's end too.
template <typename T, int kFormat, int kPieces>
__global__ __launch_bounds__(256) void dequantize_f8_kernel(const uint8_t* q, int64_t stride,
                                                            const uint8_t* scale, T* x, int64_t rows,
                                                            int64_t cols, int64_t per_row, int shift)
{
    constexpr int kN = 16 / sizeof(T);
    struct Piece {
        uint32_t w[kN / 4];
    };
    const int lane = threadIdx.x & 63;
    const int64_t units = rows * per_row, scales = (cols + 511) / 512 * 4;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units;
         u += (int64_t)gridDim.x * 4) {
        const int64_t r = u / per_row, k0 = (u - r * per_row) * (64 * kN * kPieces) + lane * kN;
        const uint8_t* in = q + r * stride;
        const uint8_t* of_row = scale + (r >> shift) * scales;
        Piece v[kPieces];
        float s[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int64_t k = k0 + j * 64 * kN;
            v[j] = k < cols ? load_any<Piece>(in + k) : Piece{};
            s[j] = k < cols ? scale_value(of_row[k / kF8Block]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int64_t k = k0 + j * 64 * kN;
            float f[kN];
#pragma unroll
            for (int i = 0; i < kN / 4; ++i) from_f8x4<kFormat>(v[j].w[i], *reinterpret_cast<float(*)[4]>(f + 4 * i));
            Quad o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2)
                    o.w[i] = bf16x2_rne(f[2 * i] * s[j], f[2 * i + 1] * s[j]);
                else
                    o.w[i] = __float_as_uint(f[i] * s[j]);
            }
            T* out = x + r * cols + k;
            if (k + kN <= cols) {
                stream_store_any(out, o);
            } else {
#pragma unroll
                for (int i = 0; i < kN; ++i)
                    if (k + i < cols)
                        out[i] = sizeof(T) == 2 ? (T)(o.w[i / 2] >> (16 * (i % 2))) : (T)o.w[i % 4];
            }
        }
    }
}

constexpr int64_t kMostBlocks = 0x7FFFFF; // of up to 512 threads: a launch has fewer than 2^32

// Past the caches where x is larger than the 256 MB behind all L2s: 8192 x 18944 (310 MB)
// takes 132 us so with its transposed copy and 137 through them, 8192 x 3584, which
// what made it left there, 30 and 26.
constexpr int64_t kCached = (int64_t)1 << 28;

// A wave of blocks of rows takes one unit where all are on the chip at once (1024 x 3584
// in bf16: 4.0 us, with two 4.2, with four 4.6; 333 x 896: 2.6, 3.3, 4.6), else two
// (8192 x 3584: 15.8 us, with one 16.4, with four 16.7), in bf16 from memory four
// (8192 x 18944: 71.7, with two 74, with one 83; fp32: 120, 117, 119).
template <typename T, int kFormat, bool kStream>
void quantize_f8_as(const QuantizeArgs& a, bool square, hipStream_t stream)
{
    if (!square && !a.qt) {
        const int64_t per_row = (a.cols + 511) / 512, units = a.rows * per_row;
        auto go = [&](auto kernel, int64_t of_block) {
            const int64_t blocks = (units + of_block - 1) / of_block;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)),
                               dim3(256), 0, stream, a, per_row);
        };
        constexpr int kMany = kStream && sizeof(T) == 2 ? 4 : 2;
        if constexpr (!kStream) { // else they are 131072 and more
            if (units <= kUnits * 32) return go(quantize_rows_f8_kernel<T, kFormat, kStream, 1>, 4);
        }
        return go(quantize_rows_f8_kernel<T, kFormat, kStream, kMany>, 4 * kMany);
    }
    const int64_t tiles_c = (a.cols + 127) / 128, tiles = (a.rows + 127) / 128 * tiles_c;
    const dim3 grid((unsigned)(tiles < kMostBlocks ? tiles : kMostBlocks));
    if (square)
        hipLaunchKernelGGL((quantize_tile_f8_kernel<T, kFormat, true, kStream>), grid, dim3(512), 0,
                           stream, a, tiles_c, tiles);
    else
        hipLaunchKernelGGL((quantize_tile_f8_kernel<T, kFormat, false, kStream>), grid, dim3(512), 0,
                           stream, a, tiles_c, tiles);
}
template <typename T, int kFormat>
void quantize_f8(const QuantizeArgs& a, bool square, hipStream_t stream)
{
    if (a.rows * a.cols > kCached / (int64_t)sizeof(T))
        quantize_f8_as<T, kFormat, true>(a, square, stream);
    else
        quantize_f8_as<T, kFormat, false>(a, square, stream);
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
    const int shift = square ? 7 : 0;
    auto go = [&](auto* out, auto one, auto more, int pieces) {
        // a piece a wave where these are few (fp32, 2048 x 3584: 6.1 us, with four 7.4; 16 x
        // 18944: 2.4, 3.0), else 1024 values (2048 x 18944 in bf16: 18.6 us, with one 19.4)
        const int64_t of_piece = 1024 / (int64_t)sizeof(*out);
        const bool few = rows * ((cols + of_piece - 1) / of_piece) <= kUnits * 128;
        const int64_t of_wave = few ? of_piece : of_piece * pieces;
        const int64_t per_row = (cols + of_wave - 1) / of_wave, blocks = (rows * per_row + 3) / 4;
        const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks));
        hipLaunchKernelGGL(few ? one : more, grid, dim3(256), 0, stream, q, q_stride, scale, out, rows,
                           cols, per_row, shift);
    };
    auto to_bf16 = [&](auto one, auto more) { go(static_cast<uint16_t*>(x), one, more, 2); };
    auto to_fp32 = [&](auto one, auto more) { go(static_cast<uint32_t*>(x), one, more, 4); };
    if (dtype == ROI_BF16)
        format == ROI_E4M3
            ? to_bf16(dequantize_f8_kernel<uint16_t, ROI_E4M3, 1>, dequantize_f8_kernel<uint16_t, ROI_E4M3, 2>)
            : to_bf16(dequantize_f8_kernel<uint16_t, ROI_E5M2, 1>, dequantize_f8_kernel<uint16_t, ROI_E5M2, 2>);
    else
        format == ROI_E4M3
            ? to_fp32(dequantize_f8_kernel<uint32_t, ROI_E4M3, 1>, dequantize_f8_kernel<uint32_t, ROI_E4M3, 4>)
            : to_fp32(dequantize_f8_kernel<uint32_t, ROI_E5M2, 1>, dequantize_f8_kernel<uint32_t, ROI_E5M2, 4>);
    return launch_status("roi_dequantize_blocks");
}
