// rows_i8.hip -- gfx950 kernels of the int8 rows: quantize_rows and
// dequantize_rows.
//
// scale = fl(amax / 127), at least 2^-126 and at most the largest whose 127-fold is
// finite, inv = fl(127 fl(1 / amax)) (2^126 at that floor), q = rint(fl(x inv)): the
// two divisions are one per row and IEEE, the per-element work is a product, a
// rounding and a pack.  Both kernels are bound
// by HBM: 3 bytes an element from bf16 (5 from fp32), once each.  The row is
// read once: it stays in the registers of the waves that own it between the
// maximum and the rounding.
#include <hip/hip_runtime.h>

#include "host.hpp"
#include "rows.hpp"
#include "roi.h"

namespace roi {
namespace {

constexpr float kScaleFloor = 0x1p-126f;
// The largest fp32 value whose 127-fold rounds to a finite one: fl(amax / 127) of
// amax = FLT_MAX, the one row it is for, lies one step above.
constexpr float kScaleTop = 0x1.020406p+121f;
constexpr uint32_t kInfBits = 0x7F800000u;

// Eight consecutive elements of a row, as loaded.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    uint32_t w[4];
    __device__ __forceinline__ float get(int i) const
    {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(int i, uint16_t v)
    {
        w[i / 2] = i & 1 ? (w[i / 2] & 0xFFFFu) | ((uint32_t)v << 16)
                         : (w[i / 2] & 0xFFFF0000u) | v;
    }
};
template <>
struct Eight<uint32_t> {
    uint32_t w[8];
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void set(int i, uint32_t v) { w[i] = v; }
};

// Elements 8 c .. 8 c + 7 of a row of `cols`, zeros past its end.
template <bool kStream, typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* row, int64_t c, int64_t cols)
{
    Eight<T> e{};
    const int64_t k = 8 * c;
    if (k + 8 <= cols) {
        e = kStream ? stream_load_any<Eight<T>>(row + k) : load_any<Eight<T>>(row + k);
    } else if (k < cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols) e.set(i, row[k + i]);
    }
    return e;
}

// The largest magnitude as fp32 bits: magnitudes of floats order as integers,
// infinities and NaN above every number.
template <typename T>
__device__ __forceinline__ uint32_t max_bits(const Eight<T>& e, uint32_t m)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(e.get(i)) & 0x7FFFFFFFu;
        m = b > m ? b : m;
    }
    return m;
}

// rint(fl(x inv)) of four elements, a byte each.  Adding 1.5 2^23 rounds the
// product to an integer, ties to even, and leaves it in the sum's low bits.
template <typename T>
__device__ __forceinline__ uint32_t quantize4(const Eight<T>& e, int first, float inv)
{
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(e.get(first + i) * inv + 0x1.8p23f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0C0C0400),
                                 __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400), 0x05040100);
}

template <typename T>
__device__ __forceinline__ void store_quantized(const Eight<T>& e, float inv, bool finite,
                                                int8_t* row, int64_t c, int64_t cols)
{
    Pair p{finite ? quantize4(e, 0, inv) : 0, finite ? quantize4(e, 4, inv) : 0};
    const int64_t k = 8 * c;
    if (k + 8 <= cols) {
        store_any(row + k, p);
    } else if (k < cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols) row[k + i] = (int8_t)(p.w[i / 4] >> (8 * (i % 4)));
    }
}

// A row over kWaves waves (a block holds 4 / kWaves rows when kWaves <= 4),
// each lane holding kChunks groups of eight in registers; kChunks == 0: a row
// longer than that, read twice.
template <typename T, int kWaves, int kChunks>
__global__ __launch_bounds__(kWaves > 4 ? 64 * kWaves : 256) void quantize_rows_kernel(
    const T* x, int8_t* q, float* scale, int64_t rows, int64_t cols)
{
    constexpr int kRowsPerBlock = kWaves > 4 ? 1 : 4 / kWaves;
    constexpr int kLanes = 64 * kWaves;
    __shared__ uint32_t part[kWaves > 4 ? kWaves : 4];
    const int wave = threadIdx.x >> 6;
    const int lane = threadIdx.x % kLanes;
    const int64_t r = (int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x / kLanes;
    const bool live = r < rows;
    const T* row = x + (live ? r : 0) * cols;
    int8_t* out = q + (live ? r : 0) * cols;
    const int64_t chunks = live ? (cols + 7) / 8 : 0;

    // past the caches for the widest rows: 8192 x 18944 takes 79 us so and 84
    // through them, 8192 x 896 6.5 and 6.2
    constexpr bool kStream = kWaves == 16 && kChunks > 0;
    constexpr int kHeld = kChunks > 0 ? kChunks : 1;
    Eight<T> held[kHeld];
    uint32_t m = 0;
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int64_t c = lane + (int64_t)j * kLanes;
            held[j] = c < chunks ? load_eight<kStream>(row, c, cols) : Eight<T>{};
        }
#pragma unroll
        for (int j = 0; j < kChunks; ++j) m = max_bits(held[j], m);
    } else {
        for (int64_t c = lane; c < chunks; c += kLanes) m = max_bits(load_eight<kStream>(row, c, cols), m);
    }
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)m, d);
        m = o > m ? o : m;
    }
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) part[wave] = m;
        __syncthreads();
        const int first = wave - wave % kWaves;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) m = part[first + j] > m ? part[first + j] : m;
    }
    if (!live) return;

    const float amax = __uint_as_float(m);
    const bool finite = m < kInfBits;
    const float s = amax / 127.0f;
    const bool low = !(s > kScaleFloor);
    const float inv = low ? 0x1p126f : 127.0f * (1.0f / amax);
    if (lane == 0)
        scale[r] = finite ? (low ? kScaleFloor : s < kScaleTop ? s : kScaleTop)
                          : __uint_as_float(0x7FC00000u);
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int64_t c = lane + (int64_t)j * kLanes;
            if (c < chunks) store_quantized(held[j], inv, finite, out, c, cols);
        }
    } else {
        for (int64_t c = lane; c < chunks; c += kLanes)
            store_quantized(load_eight<kStream>(row, c, cols), inv, finite, out, c, cols);
    }
}

// One wave per 1024 elements of a row; a lane's pieces make 16 bytes of x, so that
// a wave stores 1024 consecutive bytes at a time (past the caches: x is wide and
// written once; 8192 x 18944 takes 67 us so and 86 through them).
template <typename T>
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const int8_t* q, const float* scale,
                                                              T* x, int64_t rows, int64_t cols,
                                                              int64_t per_row)
{
    constexpr int kN = 16 / sizeof(T);
    struct Piece {
        uint32_t w[kN / 4];
    };
    const int64_t waves = rows * per_row;
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < waves;
         w += (int64_t)gridDim.x * 4) {
        const int64_t r = w / per_row, k0 = (w % per_row) * 1024 + lane * kN;
        const float s = scale[r];
        const uint8_t* in = reinterpret_cast<const uint8_t*>(q) + r * cols;
        T* out = x + r * cols;
        Piece v[16 / kN];
#pragma unroll
        for (int j = 0; j < 16 / kN; ++j)
            v[j] = k0 + j * 64 * kN < cols ? load_row<Piece>(in, k0 + j * 64 * kN, cols) : Piece{};
#pragma unroll
        for (int j = 0; j < 16 / kN; ++j) {
            const int64_t k = k0 + j * 64 * kN;
            float f[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i)
                f[i] = (float)(int8_t)(v[j].w[i / 4] >> (8 * (i % 4))) * s;
            Quad o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2)
                    o.w[i] = bf16x2_rne(f[2 * i], f[2 * i + 1]);
                else
                    o.w[i] = __float_as_uint(f[i]);
            }
            if (k + kN <= cols) {
                stream_store_any(out + k, o);
            } else {
#pragma unroll
                for (int i = 0; i < kN; ++i)
                    if (k + i < cols)
                        out[k + i] = sizeof(T) == 2 ? (T)(o.w[i / 2] >> (16 * (i % 2))) : (T)o.w[i % 4];
            }
        }
    }
}

// Rows to rows of whole 16-byte pieces, one piece a lane, a wave within a row.
__host__ __device__ int64_t copy_waves(const RowsCopy& c) { return c.rows * ((c.row + 1023) / 1024); }
__global__ __launch_bounds__(256) void copy_rows_kernel(RowsCopy a, RowsCopy b)
{
    const int64_t first = copy_waves(a), waves = first + copy_waves(b);
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < waves;
         w += (int64_t)gridDim.x * 4) {
        const RowsCopy& c = w < first ? a : b;
        const int64_t in = w < first ? w : w - first, per_row = (c.row + 1023) / 1024;
        const int64_t r = in / per_row, k = (in % per_row) * 1024 + 16 * lane;
        if (k < c.row) {
            const Quad v = load_row<Quad>(static_cast<const uint8_t*>(c.from) + r * c.len, k, c.len);
            *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(c.to) + r * c.row + k) =
                u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
        }
    }
}

template <typename T, int kWaves, int kChunks>
void launch_quantize(const T* x, int8_t* q, float* scale, int64_t rows, int64_t cols,
                     hipStream_t stream)
{
    constexpr int kThreads = kWaves > 4 ? 64 * kWaves : 256;
    constexpr int kRowsPerBlock = kWaves > 4 ? 1 : 4 / kWaves;
    // a launch has fewer than 2^32 threads; longer inputs take several
    const int64_t most = (int64_t)(0xFFFFFFFFu / kThreads) * kRowsPerBlock;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        hipLaunchKernelGGL((quantize_rows_kernel<T, kWaves, kChunks>),
                           dim3((unsigned)((n + kRowsPerBlock - 1) / kRowsPerBlock)),
                           dim3(kThreads), 0, stream, x + r * cols, q + r * cols, scale + r, n,
                           cols);
    }
}

template <typename T>
void quantize(const T* x, int8_t* q, float* scale, int64_t rows, int64_t cols, hipStream_t stream)
{
    if (cols <= 64 * 8 * 2)
        launch_quantize<T, 1, 2>(x, q, scale, rows, cols, stream);
    else if (cols <= 64 * 8 * 4)
        launch_quantize<T, 1, 4>(x, q, scale, rows, cols, stream);
    else if (cols <= 256 * 8 * 4)
        launch_quantize<T, 4, 4>(x, q, scale, rows, cols, stream);
    else if (cols <= 512 * 8 * 3)
        launch_quantize<T, 8, 3>(x, q, scale, rows, cols, stream);
    else if (cols <= 1024 * 8 * 4)
        launch_quantize<T, 16, 4>(x, q, scale, rows, cols, stream);
    else
        launch_quantize<T, 16, 0>(x, q, scale, rows, cols, stream);
}

} // namespace

void launch_copy_rows(const RowsCopy& a, const RowsCopy& b, hipStream_t stream)
{
    const int64_t blocks = (copy_waves(a) + copy_waves(b) + 3) / 4;
    if (blocks == 0) return;
    hipLaunchKernelGGL(copy_rows_kernel, dim3((unsigned)(blocks < 0xFFFFFF ? blocks : 0xFFFFFF)),
                       dim3(256), 0, stream, a, b);
}

} // namespace roi

using namespace roi;

extern "C" int roi_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int8_t* q,
                                 float* scale, hipStream_t stream)
{
    bool todo;
    if (int st = validate_rows_i8(x, dtype, q, scale, rows, cols, false, &todo)) return st;
    if (!todo) return ok();
    if (dtype == ROI_BF16)
        quantize(static_cast<const uint16_t*>(x), q, scale, rows, cols, stream);
    else
        quantize(static_cast<const uint32_t*>(x), q, scale, rows, cols, stream);
    return launch_status("roi_quantize_rows");
}

extern "C" int roi_dequantize_rows(const int8_t* q, const float* scale, int64_t rows, int64_t cols,
                                   void* x, int dtype, hipStream_t stream)
{
    bool todo;
    if (int st = validate_rows_i8(x, dtype, q, scale, rows, cols, true, &todo)) return st;
    if (!todo) return ok();
    const int64_t per_row = (cols + 1023) / 1024;
    const int64_t blocks = (rows * per_row + 3) / 4; // below 2^31 * 2^21
    const dim3 grid((unsigned)(blocks < 0xFFFFFF ? blocks : 0xFFFFFF));
    if (dtype == ROI_BF16)
        hipLaunchKernelGGL((dequantize_rows_kernel<uint16_t>), grid, dim3(256), 0, stream, q, scale,
                           static_cast<uint16_t*>(x), rows, cols, per_row);
    else
        hipLaunchKernelGGL((dequantize_rows_kernel<uint32_t>), grid, dim3(256), 0, stream, q, scale,
                           static_cast<uint32_t*>(x), rows, cols, per_row);
    return launch_status("roi_dequantize_rows");
}
