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

#include <type_traits>

#include "host.hpp"
#include "mm.hpp"
#include "roi.h"

namespace roi {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kSum = 64; // sum indices a step

struct Word {
    uint32_t w[1];
};

struct GradArgs {
    const uint16_t* dy;
    const int8_t* q;
    const float* scale;
    uint16_t* out;
    float* partial; // fp32 [splits, D, cols]
    int K, D, cols;
    uint32_t td, tc, splits;
    int steps;
};

// dy's tile of a step in LDS.  kSumRows: [64 k][kTile d], the 16-byte chunk j of
// row k at place j ^ 2 (k & 3), so that the four rows that a group of 16 lanes
// reads together lie in different banks.  Otherwise [kTile d] k-rows (mm.hpp).
// What lies past K is zero; past D, zero or the last row again.
template <int kTile, bool kSumRows, bool kWhole>
struct DyTile {
    static constexpr int kThreads = Tile<kTile>::kThreads;
    static constexpr int kLoads = kTile * kRowBytes / (16 * kThreads);
    static constexpr int kAcrossRow = kSumRows ? kTile / 8 : 8; // chunks of a row
    const uint8_t* base; // of row 0, column d0 (kSumRows), or of row d0
    int K, D, d0;
    uint32_t at;  // byte offset of load 0 from base
    int from[4];  // where read() starts, by block of 16 columns (mod 4)

    __device__ __forceinline__ DyTile(const GradArgs& a, int d0_)
        : base(reinterpret_cast<const uint8_t*>(a.dy) + 2 * (kSumRows ? d0_ : (int64_t)d0_ * a.K)),
          K(a.K), D(a.D), d0(d0_)
    {
        at = 2 * ((uint32_t)row(0) * width() + 8 * chunk());
        if (kSumRows && 8 * chunk() >= D - d0) at = kNowhere;
        const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (kSumRows) {
                const int r = 8 * g + ((lane & 15) >> 2);
                from[j] = r * (2 * kTile) + (2 * (j ^ (r & 3)) + ((lane & 3) >> 1)) * 16 +
                          (lane & 1) * 8;
            } else {
                from[j] = (16 * j + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
            }
        }
    }
    // Row and chunk of this thread's load i (the chunk is the same for all: the
    // rows differ by a multiple of eight).
    __device__ __forceinline__ static int row(int i)
    {
        return (i * kThreads + (int)threadIdx.x) / kAcrossRow;
    }
    __device__ __forceinline__ static int chunk()
    {
        return (threadIdx.x % kAcrossRow) ^ (kSumRows ? 2 * (row(0) & 3) : row(0) & 7);
    }
    // Elements of a row of dy.
    __device__ __forceinline__ uint32_t width() const { return kSumRows ? D : K; }
    // Load i of the step at sum index k0.
    __device__ __forceinline__ void stage(int i, int k0, ROI_LDS uint8_t* dst) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint8_t* p = base + 2 * (kSumRows ? (int64_t)k0 * D : k0);
        const bool live = row(i) < (kSumRows ? K - k0 : D - d0) &&
                          (kSumRows || 8 * chunk() < K - k0);
        if constexpr (kWhole) {
            load_to_lds(buffer_at(p), live ? at : kNowhere, 2 * (i * kThreads / kAcrossRow) * width(),
                        dst + (i * kThreads + wave * 64) * 16);
        } else {
            Quad v{};
            if (live && at != kNowhere) {
                const int64_t k = (kSumRows ? d0 : k0) + 8 * chunk(); // within dy's row
                v = load_row<Quad>(p + 2 * ((int64_t)row(i) * width() - (kSumRows ? d0 : k0)), 2 * k,
                                   2 * (int64_t)width());
            }
            lds_write(dst + (i * kThreads + threadIdx.x) * 16, v);
        }
    }
    // The 16 columns d of block `block` (its number mod 4 is j), sum indices
    // 32 h + 8 g .. + 7.
    __device__ __forceinline__ bf16x8 read(const ROI_LDS uint8_t* src, int block, int j, int h) const
    {
        if constexpr (kSumRows) {
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            const ROI_LDS uint8_t* p = src + from[j] + block / 4 * 128 + h * 32 * (2 * kTile);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ROI_LDS i16x4*)p);
            const i16x4 hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((ROI_LDS i16x4*)(p + 4 * (2 * kTile)));
            const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, both);
        } else { // chunk 4 + g is 64 bytes away: the places' third bit flips
            return lds_read<bf16x8>(src + block / 4 * 64 * kRowBytes + 16 * j * kRowBytes +
                                    (from[0] ^ (64 * h)));
        }
    }
};

// The int8 tile of a step: an item is eight sum indices of four columns, whose
// values are scaled, rounded to bf16, and written as one 16-byte chunk of each
// column's k-row.  Chunk j of row c lies at place j ^ ((c ^ c / 4) & 7): any
// eight lanes that write (c = 4 lane + b) or read (consecutive c) meet eight
// different places.  A step's 64 scales are one load, lane k's the k-th.
template <int kTile, bool kWhole>
struct QTile {
    static constexpr int kItems = kTile * 2 / Tile<kTile>::kThreads;
    static_assert(kItems == 1, "one item a thread");
    static constexpr bool kOneOct = kTile / 4 == 64; // all of a wave's items have the same sum indices
    const uint8_t* base; // of row 0, column c0
    const float* scale;
    int K, left;         // columns from this thread's first on
    uint32_t cols;
    int to, from;        // where write() and read() start
    uint32_t v[8], s;

    __device__ __forceinline__ QTile(const GradArgs& a, int c0)
        : base(reinterpret_cast<const uint8_t*>(a.q) + c0), scale(a.scale), K(a.K),
          left(a.cols - c0 - 4 * group()), cols(a.cols)
    {
        const int lane = threadIdx.x & 63;
        to = place(4 * group(), oct());
        from = place(lane & 15, lane >> 4);
    }
    __device__ __forceinline__ static int oct()
    {
        const int o = threadIdx.x / (kTile / 4);
        return kOneOct ? __builtin_amdgcn_readfirstlane(o) : o;
    }
    __device__ __forceinline__ static int group() { return threadIdx.x % (kTile / 4); }
    __device__ __forceinline__ static int place(int c, int chunk)
    {
        return c * kRowBytes + (chunk ^ ((c ^ (c >> 2)) & 7)) * 16;
    }

    __device__ __forceinline__ void load(int k0)
    {
        const int lane = threadIdx.x & 63;
        s = __builtin_amdgcn_raw_buffer_load_b32(buffer_at(scale + k0),
                                                 lane < K - k0 ? 4 * lane : kNowhere, 0, 0);
        const uint8_t* p = base + (int64_t)k0 * cols;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // a row past the end is the last again, times a scale of zero
            const int row = least(8 * oct() + j, K - k0 - 1);
            if constexpr (kWhole && kOneOct)
                v[j] = __builtin_amdgcn_raw_buffer_load_b32(
                    buffer_at(p), left > 0 ? 4 * group() : kNowhere, row * (int)cols, 0);
            else if constexpr (kWhole)
                v[j] = __builtin_amdgcn_raw_buffer_load_b32(
                    buffer_at(p), left > 0 && row >= 0 ? row * cols + 4 * group() : kNowhere, 0, 0);
            else
                v[j] = left > 0 && row >= 0
                           ? load_row<Word>(p + (int64_t)row * cols + 4 * group(), 0, left).w[0]
                           : 0;
        }
    }
    // Column b.
    __device__ __forceinline__ void write(int b, ROI_LDS uint8_t* dst) const
    {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 8 * oct() + j;
            const int sk = kOneOct ? __builtin_amdgcn_readlane((int)s, k) : __shfl((int)s, k);
            f[j] = (float)(int8_t)(v[j] >> (8 * b)) * __uint_as_float(sk);
        }
        // the place of column b is that of column 0 with its low bits flipped by b
        lds_write(dst + (to ^ (16 * b)) + b * kRowBytes,
                  Quad{bf16x2_rne(f[0], f[1]), bf16x2_rne(f[2], f[3]), bf16x2_rne(f[4], f[5]),
                       bf16x2_rne(f[6], f[7])});
    }
    // The 16 columns of block `block` (its number is even or odd as i), sum
    // indices 32 h + 8 g .. + 7: chunk 4 h + g, and the place's third bit flips
    // with h and with each block.
    __device__ __forceinline__ bf16x8 read(const ROI_LDS uint8_t* src, int block, int i, int h) const
    {
        return lds_read<bf16x8>(src + block * 16 * kRowBytes + (from ^ (64 * ((i + h) & 1))));
    }
};

__device__ __forceinline__ void store4(const GradArgs& a, int64_t d, int c, f32x4 v)
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

template <int kTile, bool kSumRows, bool kWhole>
__global__ __launch_bounds__(Tile<kTile>::kThreads) void grad_tile_kernel(GradArgs a)
{
    constexpr int kTileBytes = kTile * kRowBytes;
    static_assert(kTileBytes == kSum * kTile * 2, "both layouts of dy take the same LDS");
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    static_assert(kJ == 4 && kI % 2 == 0, "DyTile::read and QTile::read");
    using Dy = DyTile<kTile, kSumRows, kWhole>;
    using Q = QTile<kTile, kWhole>;
    static_assert(Dy::kLoads <= kI && kI >= 4, "a part a row");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0][0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // first block of 16 of this wave along c and d
    const int bc = wave / Tile<kTile>::kAcross * kI, bd = wave % Tile<kTile>::kAcross * kJ;
    int td, tc;
    tile_at(xcd_order(blockIdx.x, a.td * a.tc), a.td, a.tc, 8, td, tc);
    const int d0 = td * kTile, c0 = tc * kTile;

    f32x4 acc[kI][kJ] = {};
    const Dy dy(a, d0);
    Q q(a, c0);
    // As in linear_i8.hip: a half step's products beside the reads of the next,
    // one barrier a step.  The int8 tile of step s + 2 is in registers by then.
    auto buffer = [&](int s) { return base + (s & 1) * 2 * kTileBytes; };
    struct Half {
        bf16x8 q[kI], y[kJ];
    };
    // the products of a half, beside the reads of half h of step s and (load)
    // the tiles of step s + 1, as whose int8 part q is written; past the sum's
    // end all of that is zeros and unused
    auto half = [&](const Half& f, int s, int h, Half& next, auto load) {
        ROI_LDS uint8_t* src = buffer(s);
        ROI_LDS uint8_t* dst = buffer(s + 1);
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) next.y[i] = dy.read(src + kTileBytes, bd + i, i, h);
            next.q[i] = q.read(src, bc + i, i, h);
            if constexpr (decltype(load)::value) {
                if (i < Dy::kLoads) dy.stage(i, (s + 1) * kSum, dst + kTileBytes);
                if (i % (kI / 4) == 0) q.write(i / (kI / 4), dst);
                if (i == kI - 1) q.load((s + 2) * kSum);
            }
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.q[i], f.y[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    if (a.steps > 0) {
        Half lo, hi;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < Dy::kLoads; ++i) dy.stage(i, s * kSum, buffer(s) + kTileBytes);
            q.load(s * kSum);
#pragma unroll
            for (int b = 0; b < 4; ++b) q.write(b, buffer(s));
        }
        q.load(2 * kSum);
        loads_barrier();
#pragma unroll
        for (int i = 0; i < kI; ++i) lo.q[i] = q.read(buffer(0), bc + i, i, 0);
#pragma unroll
        for (int j = 0; j < kJ; ++j) lo.y[j] = dy.read(buffer(0) + kTileBytes, bd + j, j, 0);
        for (int s = 0; s < a.steps; ++s) {
            half(lo, s, 1, hi, std::false_type{});
            loads_barrier();
            half(hi, s + 1, 0, lo, std::true_type{});
        }
        loads_barrier();
    }
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
        const int d = d0 + 16 * (bd + j) + (lane & 15);
        if (d >= a.D) continue;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            const int c = c0 + 16 * (bc + i) + 4 * g;
            if (c < a.cols) store4(a, d, c, acc[i][j]);
        }
    }
}

template <int kTile, bool kSumRows>
void launch_tiles(const GradArgs& a, hipStream_t stream)
{
    const dim3 grid(a.td * a.tc), block(Tile<kTile>::kThreads);
    // 16-byte chunks of dy's rows and 4-byte words of q's that end with the row
    const bool whole = (kSumRows ? a.D : a.K) % 8 == 0 && a.cols % 4 == 0;
    if (whole)
        hipLaunchKernelGGL((grad_tile_kernel<kTile, kSumRows, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((grad_tile_kernel<kTile, kSumRows, false>), grid, block, 0, stream, a);
}

template <bool kSumRows>
int launch(GradArgs a, const char* what, hipStream_t stream)
{
    const Cut c = cut_product(a.D, a.cols, a.K, kSum);
    if (c.tm * c.tn > (int64_t)(0xFFFFFFFFu / Tile<256>::kThreads))
        return fail(ROI_E_UNSUPPORTED, "the gradient has too many elements for one call");
    a.td = (uint32_t)c.tm;
    a.tc = (uint32_t)c.tn;
    a.splits = 1;
    a.steps = (int)c.steps;
    if (c.tile == 256)
        launch_tiles<256, kSumRows>(a, stream);
    else
        launch_tiles<128, kSumRows>(a, stream);
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
    const GradArgs a{grad_y, xq, xs, grad_w, static_cast<float*>(workspace), (int)tokens, (int)rows,
                     (int)cols, 0, 0, 1, 0};
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
    const GradArgs a{grad_y, wq, ws, grad_x, static_cast<float*>(workspace), (int)rows, (int)tokens,
                     (int)cols, 0, 0, 1, 0};
    return launch<false>(a, "roi_linear_i8_grad_input", stream);
}
