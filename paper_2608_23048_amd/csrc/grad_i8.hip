// grad_i8.hip -- gfx950 kernels of the two gradients of the int8 product:
//   grad_w[r, c] = sum_t grad_y[t, r] xs[t] xq[t, c]
//   grad_x[t, c] = sum_r grad_y[t, r] ws[r] wq[r, c]
// Both are out[d, c] = sum_k dy(d, k) s[k] q[k, c] with q int8 [K, cols], one
// scale a row, and dy bf16 with its sum index k in rows (the weight gradient:
// dy is [K, D]) or contiguous (the input gradient: dy is [D, K]).
//
// s q is formed in fp32 and rounded once to bf16 on its way to LDS (the value that
// dequantize_rows gives in bf16; the other operand and the result are bf16, and so
// are the matrix instructions); the products and sums are fp32.  With that rounding
// the gradients are off from 64 bits by 0.0023 in norm, without it, by the result's
// own, 0.0017.  q by itself is exact in bf16, but s goes with the summed index and
// stays in the sum; s q in two bf16 terms would be twice the matrix instructions,
// which bound the large gradients.  The int8 operand is the matrix instruction's
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
    float* partial; // fp32 parts of tiles (Held::part_at)
    uint16_t* ready; // s q, transposed: bf16 [cols, ready_k], or NULL
    int ready_k;     // K rounded up to whole steps
    int K, D, cols;
    int dy_row, q_row; // elements of a row of dy and of q
    Grid grid; // tiles along d and c
};

// dy's tile of a step in LDS.  kSumRows: [64 k][kTile d], the 16-byte chunk j of
// row k at place j ^ 2 (k & 3) ^ (k & 8), so that the rows that 32 lanes read
// together (four of each of two groups of 16) lie in different banks.  Otherwise
// [kTile d] k-rows (mm.hpp).  What lies past K is zero; past D, zero or the last row again.
template <int kTile, bool kSumRows, bool kUnseen = kSumRows, int kWaves = waves_of(kTile)>
struct DyTile {
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kLoads = kTile * kRowBytes / (16 * kThreads);
    static constexpr int kAcrossRow = kSumRows ? kTile / 8 : 8; // chunks of a row
    const uint8_t* base; // of row 0, column d0 (kSumRows), or of row d0
    int K, D, d0;
    uint32_t at;  // byte offset of load 0 from base
    int from[kSumRows ? 4 : 1]; // where read() starts, by block of 16 columns

    // block: the wave's first of 16 columns
    __device__ __forceinline__ DyTile(const uint16_t* p, int K_, int D_, int d0_, int block)
        : base(reinterpret_cast<const uint8_t*>(p) + 2 * (kSumRows ? d0_ : (int64_t)d0_ * K_)),
          K(K_), D(D_), d0(d0_)
    {
        at = 2 * ((uint32_t)row(0) * width() + 8 * chunk());
        if (kSumRows && 8 * chunk() >= D - d0) at = kNowhere;
        const int lane = threadIdx.x & 63, g = lane >> 4;
        if constexpr (kSumRows) {
            const int r = 8 * g + ((lane & 15) >> 2);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                from[j] = r * (2 * kTile) + (lane & 1) * 8 +
                          ((2 * (block + j) + ((lane & 3) >> 1)) ^ spread(r)) * 16;
        } else {
            from[0] = (16 * block + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
        }
    }
    __device__ __forceinline__ static int spread(int row)
    {
        return kSumRows ? (2 * (row & 3)) ^ (row & 8) : row & 7;
    }
    // Row and chunk of this thread's load i (the chunk is the same for all: the
    // rows differ by a multiple of sixteen).
    __device__ __forceinline__ static int row(int i)
    {
        return (i * kThreads + (int)threadIdx.x) / kAcrossRow;
    }
    __device__ __forceinline__ static int chunk()
    {
        return (threadIdx.x % kAcrossRow) ^ spread(row(0));
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
        load_to_lds<kUnseen>(buffer_at(p), live ? at : kNowhere,
                             2 * (i * kThreads / kAcrossRow) * width(),
                             dst + (i * kThreads + wave * 64) * 16);
    }
    // The 16 columns d of the wave's block j, sum indices 32 h + 8 g .. + 7.
    __device__ __forceinline__ bf16x8 read(const ROI_LDS uint8_t* src, int j, int h) const
    {
        if constexpr (kSumRows) {
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            const ROI_LDS uint8_t* p = src + from[j] + h * 32 * (2 * kTile);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ROI_LDS i16x4*)p);
            const i16x4 hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((ROI_LDS i16x4*)(p + 4 * (2 * kTile)));
            const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, both);
        } else { // chunk 4 + g is 64 bytes away: the places' third bit flips
            return lds_read<bf16x8>(src + 16 * j * kRowBytes + (from[0] ^ (64 * h)));
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
          left(a.cols - c0 - 4 * group()), cols(a.q_row)
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
            // a row past the sum's last is the last again, times a scale of zero; from
            // a step past the sum's end nothing is read (row below 0)
            const int row = least(8 * oct() + j, K - k0 - 1);
            if constexpr (kWhole && kOneOct) {
                const LoadAt at = row_load(8 * oct() + j, K - k0, 4 * group(), left > 0, cols);
                v[j] = __builtin_amdgcn_raw_buffer_load_b32(buffer_at(p), at.lane, at.wave, 0);
            } else if constexpr (kWhole)
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

// A tile's results from a wave's sums: a part of a cut tile as it is, else in
// bf16 and through LDS (all of which is free) to out.
template <typename T>
__device__ __forceinline__ void write_tile(const GradArgs& a, const Piece& piece,
                                           const f32x4 (&acc)[T::kI][T::kJ], ROI_LDS uint8_t* base)
{
    constexpr int kTile = T::kTile, kI = T::kI, kJ = T::kJ;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = scalar(threadIdx.x >> 6);
    const int bc = wave / T::kAcross * kI, bd = wave % T::kAcross * kJ;
    const int d0 = piece.m * kTile, c0 = piece.n * kTile;
    if (piece.part >= 0) {
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                *reinterpret_cast<f32x4*>(
                    a.partial + Held<T, 16>::part_at(piece.part, wave, i, j, 0)) = acc[i][j];
        return;
    }
    using Out = RowsOut<kI, 8>;
    ROI_LDS uint8_t* mine = base + wave * (16 * kJ * Out::kRow);
#pragma unroll
    for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int i = 0; i < kI; ++i)
            *reinterpret_cast<ROI_LDS u32x2*>(Out::at(mine, 16 * j + (lane & 15), 4 * i + g)) =
                u32x2{bf16x2_rne(acc[i][j][0], acc[i][j][1]), bf16x2_rne(acc[i][j][2], acc[i][j][3])};
#pragma unroll 2 // code that runs once is fetched once: it is kept short
    for (int n = 0; n < 16 * kJ / Out::kAtOnce; ++n) {
        int row, chunk;
        const Quad v = Out::get(mine, n, row, chunk);
        const int d = d0 + 16 * bd + row, c = c0 + 16 * bc + 8 * chunk;
        if (d < a.D) store_chunk(a.out + (int64_t)d * a.cols, c, a.cols, v);
    }
}

// As in linear_i8.hip, a half step's products stand beside the reads of the
// next, with one barrier a step.  LDS holds the int8 operand's bf16 tiles of two
// steps and dy's of three.  The int8 tile of step s + 3 goes to registers in step s
// and to LDS, scaled, in step s + 1.  dy's tile of step s + 3 is loaded to LDS in step
// s behind it.  In the input gradient it is awaited two steps later.  In the weight
// gradient it has until step s + 1 writes the int8 tile: its loads are in assembly,
// where the compiler does not count them, so that the waits it puts ahead of the int8
// registers' use are for dy's later loads too.  (2048 x 3584 x 3584 input gradient 56
// us without the sums of its parts, 2100 x 1032 x 4096 weight gradient 32.)
template <int kTile, bool kSumRows>
__global__ __launch_bounds__(Tile<kTile>::kThreads, 2) void grad_tile_kernel(GradArgs a)
{
    constexpr int kTileBytes = kTile * kRowBytes;
    static_assert(kTileBytes == kSum * kTile * 2, "both layouts of dy take the same LDS");
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    static_assert(kJ == 4 && kI % 2 == 0, "DyTile::read and QTile::read");
    using Dy = DyTile<kTile, kSumRows>;
    using Q = QTile<kTile, true>;
    static_assert(Dy::kLoads <= kI && kI >= 4, "a part a row");
    __shared__ __attribute__((aligned(16))) uint8_t lds[5][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // first block of 16 of this wave along c and d
    const int bc = wave / Tile<kTile>::kAcross * kI, bd = wave % Tile<kTile>::kAcross * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int d0 = piece.m * kTile, c0 = piece.n * kTile;
    const int k0 = piece.first * kSum;

    f32x4 acc[kI][kJ] = {};
    const Dy dy(a.dy, kSumRows ? a.K : a.dy_row, kSumRows ? a.dy_row : a.D, d0, bd);
    Q q(a, c0);
    struct Half {
        bf16x8 q[kI], y[kJ];
    };
    // the products of a half, beside the reads of half h of the step whose tiles
    // are at qs and ys; kLoad: also q, loaded, is written to qd and loaded for
    // sum index k, for which dy goes to yd.  Past the end of the sum or of this
    // part all of that is in bounds or zeros, and unused.
    auto half = [&](const Half& f, ROI_LDS uint8_t* qs, ROI_LDS uint8_t* ys, int h, Half& next,
                    auto load, ROI_LDS uint8_t* qd, ROI_LDS uint8_t* yd, int k) {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) next.y[i] = dy.read(ys, i, h);
            next.q[i] = q.read(qs, bc + i, i, h);
            if constexpr (decltype(load)::value) {
                if (i < 4) q.write(i, qd);
                if (i == (kI > 4 ? 4 : 3)) q.load(k);
                if (i == kI - 1) {
#pragma unroll
                    for (int l = 0; l < Dy::kLoads; ++l) dy.stage(l, k, yd);
                }
            }
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.q[i], f.y[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    if (piece.count > 0) {
        Half lo, hi;
        ROI_LDS uint8_t *q0 = base, *q1 = base + kTileBytes; // of this step and the next
        ROI_LDS uint8_t *y0 = base + 2 * kTileBytes, *y1 = y0 + kTileBytes, *y2 = y1 + kTileBytes;
        {
            Q second = q;
            q.load(k0);
            second.load(k0 + kSum);
#pragma unroll
            for (int i = 0; i < Dy::kLoads; ++i) dy.stage(i, k0, y0);
#pragma unroll
            for (int i = 0; i < Dy::kLoads; ++i) dy.stage(i, k0 + kSum, y1);
#pragma unroll
            for (int b = 0; b < 4; ++b) q.write(b, q0);
            q.load(k0 + 2 * kSum);
#pragma unroll
            for (int b = 0; b < 4; ++b) second.write(b, q1);
        }
        keep_order();
#pragma unroll
        for (int i = 0; i < Dy::kLoads; ++i) dy.stage(i, k0 + 2 * kSum, y2);
        loads_barrier<Dy::kLoads>();
#pragma unroll
        for (int i = 0; i < kI; ++i) lo.q[i] = q.read(q0, bc + i, i, 0);
#pragma unroll
        for (int j = 0; j < kJ; ++j) lo.y[j] = dy.read(y0, j, 0);
        for (int s = 0; s < piece.count; ++s) {
            half(lo, q0, y0, 1, hi, std::false_type{}, q0, y0, 0);
            loads_barrier<Dy::kLoads>();
            half(hi, q1, y1, 0, lo, std::true_type{}, q0, y0, k0 + (s + 3) * kSum);
            ROI_LDS uint8_t* const t = q0;
            q0 = q1;
            q1 = t;
            ROI_LDS uint8_t* const u = y0;
            y0 = y1;
            y1 = y2;
            y2 = u;
        }
        loads_barrier();
    }
    write_tile<Tile<kTile>>(a, piece, acc, base);
}

// The same for both operands in bf16 (a.ready): nothing passes registers on its
// way to LDS, which holds both tiles of two steps.  A step takes 1.4 us where the
// conversion beside it takes 1.7; the conversion by itself is one pass over q (17
// to 35 us of the 870 that either gradient takes at 8192 x 3584 x 18944).  Bound by
// the matrix cores and their clock: busy for 73 % of the time, at 1.8 GHz under
// that load, 1.33 PFLOP/s where the library's 8192^3 product reaches 1.30 (1.28 to
// 1.32 in the median of passes back to back, as the clock falls).
template <bool kSumRows>
__global__ __launch_bounds__(Tile<256>::kThreads) void grad_ready_kernel(GradArgs a)
{
    constexpr int kTile = 256, kTileBytes = kTile * kRowBytes;
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    using Dy = DyTile<kTile, kSumRows>;
    using Q = DyTile<kTile, false, kSumRows>;
    constexpr int kLoads = Dy::kLoads + Q::kLoads;
    static_assert(kLoads == kI, "a load a row");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0][0];
    const int wave = scalar(threadIdx.x >> 6);
    const int bc = wave / Tile<kTile>::kAcross * kI, bd = wave % Tile<kTile>::kAcross * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int d0 = piece.m * kTile, c0 = piece.n * kTile;
    const int k0 = piece.first * kSum;

    f32x4 acc[kI][kJ] = {};
    const Dy dy(a.dy, kSumRows ? a.K : a.dy_row, kSumRows ? a.dy_row : a.D, d0, bd);
    const Q q(a.ready, a.ready_k, a.cols, c0, bc);
    auto buffer = [&](int s) { return base + (s & 1) * 2 * kTileBytes; };
    auto stage = [&](int s, int i) {
        if (i < Q::kLoads)
            q.stage(i, k0 + s * kSum, buffer(s));
        else
            dy.stage(i - Q::kLoads, k0 + s * kSum, buffer(s) + kTileBytes);
    };
    struct Half {
        bf16x8 q[kI], y[kJ];
    };
    // the products of a half, beside the reads of half h of step s and (load) the
    // loads of step s + 1: past the end in bounds or zeros, and unused
    auto half = [&](const Half& f, int s, int h, Half& next, auto load) {
        ROI_LDS uint8_t* src = buffer(s);
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) next.y[i] = dy.read(src + kTileBytes, i, h);
            next.q[i] = q.read(src, i, h);
            if constexpr (decltype(load)::value) stage(s + 1, i);
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.q[i], f.y[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    if (piece.count > 0) {
        Half lo, hi;
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage(s, i);
        loads_barrier();
#pragma unroll
        for (int i = 0; i < kI; ++i) lo.q[i] = q.read(buffer(0), i, 0);
#pragma unroll
        for (int j = 0; j < kJ; ++j) lo.y[j] = dy.read(buffer(0) + kTileBytes, j, 0);
        for (int s = 0; s < piece.count; ++s) {
            half(lo, s, 1, hi, std::false_type{});
            loads_barrier();
            half(hi, s + 1, 0, lo, std::true_type{});
        }
        loads_barrier();
    }
    write_tile<Tile<kTile>>(a, piece, acc, base);
}

// For up to one 128-tile a compute unit: nothing else runs there while a block
// waits, so it has eight waves, which convert and multiply beside each other, and
// keeps more on its way.  Everything is loaded to LDS, q as it is; a step's tiles
// have between two and three steps to arrive (of kRing slots), and q's go from
// there through registers, scaled and rounded, to k-rows.  A step takes 0.57 us
// where the kernel above takes 0.80 (4096 x 896 x 896: the weight gradient 24.2 us
// against 28.3, the input's 16.1 against 18.2).  Short sums are bound by what comes
// before and after their steps, half of the time of 13 steps: the first loads, and
// the parts of cut tiles.
using DeepTile = Tile<128, 8>;
template <bool kSumRows>
__global__ __launch_bounds__(DeepTile::kThreads) void grad_deep_kernel(GradArgs a)
{
    using T = DeepTile;
    constexpr int kTile = 128, kTileBytes = kTile * kRowBytes, kRing = 5;
    constexpr int kThreads = T::kThreads, kI = T::kI, kJ = T::kJ;
    static_assert(kI == 4 && kJ == 2 && kThreads == 512, "laid out for these");
    using Dy = DyTile<kTile, kSumRows, kSumRows, T::kWaves>;
    using Q = QTile<kTile, true>;
    constexpr int kRaw = kSum * kTile, kSlot = kTileBytes + kRaw + 4 * kSum;
    constexpr int kRawLoads = kRaw / (16 * kThreads), kLoads = Dy::kLoads + kRawLoads + 1;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kTileBytes + kRing * kSlot];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    const int lane = threadIdx.x & 63;
    const int wave = scalar(threadIdx.x >> 6);
    const int bc = wave / T::kAcross * kI, bd = wave % T::kAcross * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int d0 = piece.m * kTile, c0 = piece.n * kTile;
    const int k0 = piece.first * kSum;

    f32x4 acc[kI][kJ] = {};
    const Dy dy(a.dy, kSumRows ? a.K : a.dy_row, kSumRows ? a.dy_row : a.D, d0, bd);
    const Q q(a, c0);
    ROI_LDS uint8_t* ring = base + 2 * kTileBytes;
    const uint8_t* raw = reinterpret_cast<const uint8_t*>(a.q) + c0;
    // step s of this part (past its end or the sum's: in bounds or zeros) to a slot
    auto stage = [&](int s, ROI_LDS uint8_t* slot) {
        const int k = k0 + s * kSum;
#pragma unroll
        for (int i = 0; i < Dy::kLoads; ++i) dy.stage(i, k, slot);
#pragma unroll
        for (int i = 0; i < kRawLoads; ++i) {
            const int row = (i * kThreads + (int)threadIdx.x) / 8;
            const int chunk = (threadIdx.x % 8) ^ (row & 4);
            const bool live = row < a.K - k && 16 * chunk < a.q_row - c0;
            load_to_lds<kSumRows>(buffer_at(raw + (int64_t)k * a.q_row),
                                  live ? (uint32_t)row * a.q_row + 16 * chunk : kNowhere, 0,
                                  slot + kTileBytes + (i * kThreads + wave * 64) * 16);
        }
        // the scales, by every wave to the same place
        load_words_to_lds<kSumRows>(buffer_at(a.scale + k), lane < a.K - k ? 4 * lane : kNowhere,
                                    slot + kTileBytes + kRaw);
    };
    struct Half {
        bf16x8 q[kI], y[kJ];
    };
    // a thread takes four sum indices of four columns: half a chunk of each, its
    // neighbour the other half, so that 16 lanes write 128 bytes of all banks; the
    // two read rows four apart, whose halves lie in LDS the other way round
    const int four = threadIdx.x / 64 * 2 + threadIdx.x % 2, group = threadIdx.x % 64 / 2;
    const int to = Q::place(4 * group, four / 2) + 8 * (four % 2);
    struct Raw {
        uint32_t v[4];
        f32x4 s;
    };
    auto read_raw = [&](ROI_LDS uint8_t* slot, Raw& r) {
        ROI_LDS uint8_t* p = slot + kTileBytes;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r.v[j] = lds_read<uint32_t>(p + (4 * four + j) * kTile + ((4 * group) ^ (64 * (four % 2))));
        r.s = lds_read<f32x4>(p + kRaw + 16 * four);
    };
    // column b: its place is that of column 0 with its low bits flipped by b
    auto write_column = [&](const Raw& r, int b, ROI_LDS uint8_t* dst) {
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = (float)(int8_t)(r.v[j] >> (8 * b)) * r.s[j];
        *reinterpret_cast<ROI_LDS u32x2*>(dst + (to ^ (16 * b)) + b * kRowBytes) =
            u32x2{bf16x2_rne(f[0], f[1]), bf16x2_rne(f[2], f[3])};
    };
    // the products of a half, beside the reads of half h of the step whose tiles
    // are at qs and ys; kLoad: also q's tile at `from` to qd and step s to `slot`
    auto half = [&](const Half& f, ROI_LDS uint8_t* qs, ROI_LDS uint8_t* ys, int h, Half& next,
                    auto load, ROI_LDS uint8_t* from, ROI_LDS uint8_t* qd, int s,
                    ROI_LDS uint8_t* slot) {
        Raw r;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (decltype(load)::value && i == 0) read_raw(from, r);
            if (i < kJ) next.y[i] = dy.read(ys, i, h);
            next.q[i] = q.read(qs, bc + i, i, h);
            if constexpr (decltype(load)::value) {
                if (i == 1) write_column(r, 0, qd);
                if (i == 2) write_column(r, 1, qd);
                if (i == 2) write_column(r, 2, qd);
                if (i == 3) write_column(r, 3, qd);
                if (i == 3) stage(s, slot);
            }
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.q[i], f.y[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    if (piece.count > 0) {
        Half lo, hi;
        ROI_LDS uint8_t *q0 = base, *q1 = base + kTileBytes;
        for (int s = 0; s < kRing; ++s) stage(s, ring + s * kSlot);
        loads_barrier<(kRing - 2) * kLoads>();
        {
            Raw r0, r1;
            read_raw(ring, r0);
            read_raw(ring + kSlot, r1);
#pragma unroll
            for (int b = 0; b < 4; ++b) write_column(r0, b, q0);
#pragma unroll
            for (int b = 0; b < 4; ++b) write_column(r1, b, q1);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kI; ++i) lo.q[i] = q.read(q0, bc + i, i, 0);
#pragma unroll
        for (int j = 0; j < kJ; ++j) lo.y[j] = dy.read(ring, j, 0);
        int at = 0; // this step's slot
        auto after = [&](int n) {
            const int p = at + n * kSlot;
            return ring + (p < kRing * kSlot ? p : p - kRing * kSlot);
        };
        for (int s = 0; s < piece.count; ++s) {
            half(lo, q0, ring + at, 1, hi, std::false_type{}, q0, q0, 0, q0);
            // the tiles of step s + 2 are there; two steps more are on their way
            loads_barrier<(kRing - 3) * kLoads>();
            half(hi, q1, after(1), 0, lo, std::true_type{}, after(2), q0, s + kRing, ring + at);
            ROI_LDS uint8_t* const t = q0;
            q0 = q1;
            q1 = t;
            at = at + kSlot < kRing * kSlot ? at + kSlot : 0;
        }
        loads_barrier();
    }
    write_tile<T>(a, piece, acc, base);
}

// s q in bf16, transposed to k-rows of 64 (zeros past K), for grad_ready_kernel:
// 64 rows of 128 columns a block, by way of LDS, so that both the reads and the
// writes are whole rows of at least 128 bytes.  Bound by 3 bytes an element.
template <bool kWhole>
__global__ __launch_bounds__(256) void ready_kernel(GradArgs a)
{
    using Q = QTile<128, kWhole>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[128 * kRowBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    const uint32_t across = (a.cols + 127) / 128;
    const int c0 = scalar(blockIdx.x % across) * 128, k0 = scalar(blockIdx.x / across) * kSum;
    Q q(a, c0);
    q.load(k0);
#pragma unroll
    for (int b = 0; b < 4; ++b) q.write(b, base);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int row = n * 32 + (int)threadIdx.x / 8, chunk = threadIdx.x % 8;
        const u32x4 v = lds_read<u32x4>(base + Q::place(row, chunk));
        if (c0 + row < a.cols)
            *reinterpret_cast<u32x4*>(a.ready + (int64_t)(c0 + row) * a.ready_k + k0 + 8 * chunk) = v;
    }
}

// The sums of the tiles that were cut: one wave for 16 x 16 results.
template <typename T>
__global__ __launch_bounds__(256) void grad_sum_kernel(GradArgs a)
{
    constexpr int kTile = T::kTile;
    const int lane = threadIdx.x & 63;
    const uint32_t id = scalar(blockIdx.x * 4 + threadIdx.x / 64);
    const int i = id % T::kI, j = id / T::kI % T::kJ;
    const int wave = id / (T::kJ * T::kI) % T::kWaves;
    const uint32_t tile = id / (T::kJ * T::kI * T::kWaves);
    const Piece piece = tile_piece(a.grid, a.grid.full + tile);
    const float* from = a.partial + Held<T, 16>::part_at((int64_t)tile * a.grid.splits, wave, i, j, 0);
    const f32x4 sum = sum_of_parts<T, f32x4>(from, (int)a.grid.splits);
    const int c = piece.n * kTile + 16 * (wave / T::kAcross * T::kI + i) + 4 * (lane >> 4);
    const int d = piece.m * kTile + 16 * (wave % T::kAcross * T::kJ + j) + (lane & 15);
    if (d >= a.D) return;
    uint16_t* p = a.out + (int64_t)d * a.cols + c;
    const Pair v{bf16x2_rne(sum[0], sum[1]), bf16x2_rne(sum[2], sum[3])};
    if (c + 4 <= a.cols) {
        store_any(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.cols) p[e] = (uint16_t)(v.w[e / 2] >> (16 * (e % 2)));
    }
}

template <typename T>
void launch_sums(const GradArgs& a, hipStream_t stream)
{
    if (a.grid.rest() > 0)
        hipLaunchKernelGGL((grad_sum_kernel<T>),
                           dim3(a.grid.rest() * T::kI * T::kJ * T::kWaves / 4), dim3(256), 0, stream, a);
}

template <int kTile, bool kSumRows>
void launch_tiles(const GradArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((grad_tile_kernel<kTile, kSumRows>), dim3(a.grid.blocks()),
                       dim3(Tile<kTile>::kThreads), 0, stream, a);
    launch_sums<Tile<kTile>>(a, stream);
}

template <bool kSumRows>
void launch_deep(const GradArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((grad_deep_kernel<kSumRows>), dim3(a.grid.blocks()),
                       dim3(DeepTile::kThreads), 0, stream, a);
    launch_sums<DeepTile>(a, stream);
}

template <bool kSumRows>
void launch_ready(const GradArgs& a, hipStream_t stream)
{
    const dim3 blocks((unsigned)((a.ready_k / kSum) * ((a.cols + 127) / 128)));
    if (a.cols % 4 == 0)
        hipLaunchKernelGGL((ready_kernel<true>), blocks, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((ready_kernel<false>), blocks, dim3(256), 0, stream, a);
    hipLaunchKernelGGL((grad_ready_kernel<kSumRows>), dim3(a.grid.blocks()),
                       dim3(Tile<256>::kThreads), 0, stream, a);
    launch_sums<Tile<256>>(a, stream);
}

int check_fits(const GradPlan& plan)
{
    return plan.cut.fits ? ROI_OK
                         : fail(ROI_E_UNSUPPORTED, "the gradient has too many elements for one call");
}

// Bytes of a gradient's workspace, or why it is refused.
int64_t workspace_of(int64_t tokens, int64_t rows, int64_t cols, bool by_tokens)
{
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const GradPlan plan = by_tokens ? plan_grad(rows, cols, tokens, true)
                                    : plan_grad(tokens, cols, rows, false);
    if (int st = check_fits(plan)) return st;
    ok();
    return plan.bytes;
}

template <bool kSumRows>
int launch(GradArgs a, const GradPlan& plan, void* workspace, const char* what, hipStream_t stream)
{
    if (int st = check_fits(plan)) return st;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    uint8_t* const dy = at;
    uint8_t* const q = dy + plan.dy_bytes;
    launch_copy_rows(RowsCopy{a.dy, dy, plan.dy_bytes ? (kSumRows ? a.K : a.D) : 0,
                              2 * (int64_t)(kSumRows ? a.D : a.K), 2 * plan.dy_row},
                     RowsCopy{a.q, q, plan.q_bytes ? a.K : 0, a.cols, plan.q_row}, stream);
    if (plan.dy_bytes) a.dy = reinterpret_cast<uint16_t*>(dy);
    if (plan.q_bytes) a.q = reinterpret_cast<int8_t*>(q);
    at = q + plan.q_bytes;
    a.dy_row = (int)plan.dy_row;
    a.q_row = (int)plan.q_row;
    a.ready = reinterpret_cast<uint16_t*>(at);
    a.ready_k = (int)plan.ready_k;
    a.partial = reinterpret_cast<float*>(at + plan.ready_bytes);
    a.grid = grid_of(plan.cut);
    if (plan.ready)
        launch_ready<kSumRows>(a, stream);
    else if (plan.deep)
        launch_deep<kSumRows>(a, stream);
    else if (plan.cut.tile == 256)
        launch_tiles<256, kSumRows>(a, stream);
    else
        launch_tiles<128, kSumRows>(a, stream);
    return launch_status(what);
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_i8_grad_weight_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    return workspace_of(tokens, rows, cols, true);
}

extern "C" int64_t roi_linear_i8_grad_input_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    return workspace_of(tokens, rows, cols, false);
}

extern "C" int roi_linear_i8_grad_weight(const uint16_t* grad_y, const int8_t* xq, const float* xs,
                                         int64_t tokens, int64_t rows, int64_t cols,
                                         uint16_t* grad_w, void* workspace, int64_t workspace_bytes,
                                         hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const GradPlan plan = plan_grad(rows, cols, tokens, true);
    if (int st = validate_grad_i8(grad_y, xq, xs, tokens, tokens, rows, cols, grad_w, rows,
                                  workspace, workspace_bytes, plan.bytes, &todo))
        return st;
    if (!todo) return ok();
    const GradArgs a{grad_y, xq, xs, grad_w, nullptr, nullptr, 0, (int)tokens, (int)rows, (int)cols, 0, 0, {}};
    return launch<true>(a, plan, workspace, "roi_linear_i8_grad_weight", stream);
}

extern "C" int roi_linear_i8_grad_input(const uint16_t* grad_y, const int8_t* wq, const float* ws,
                                        int64_t tokens, int64_t rows, int64_t cols,
                                        uint16_t* grad_x, void* workspace, int64_t workspace_bytes,
                                        hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const GradPlan plan = plan_grad(tokens, cols, rows, false);
    if (int st = validate_grad_i8(grad_y, wq, ws, rows, tokens, rows, cols, grad_x, tokens,
                                  workspace, workspace_bytes, plan.bytes, &todo))
        return st;
    if (!todo) return ok();
    const GradArgs a{grad_y, wq, ws, grad_x, nullptr, nullptr, 0, (int)rows, (int)tokens, (int)cols, 0, 0, {}};
    return launch<false>(a, plan, workspace, "roi_linear_i8_grad_input", stream);
}
