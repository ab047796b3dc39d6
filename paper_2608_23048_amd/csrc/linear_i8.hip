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

#include <type_traits>

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
    int* partial; // int32 parts of tiles (part_at)
    int tokens, rows, cols;
    Grid grid; // tiles along the rows and the tokens (few tokens: grid.tm alone)
};

// The scales of rows r .. r + 3, and what is added to their results: without a
// bias -0, which changes nothing.
__device__ __forceinline__ void row_scales(const LinearArgs& a, int r, float (&ws)[4],
                                           float (&add)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int rc = least(r + e, a.rows - 1);
        ws[e] = a.ws[rc];
        add[e] = a.bias ? bf16_bits_to_float(a.bias[rc]) : -0.0f;
    }
}

// Four results from their exact sums.  The scale of the weight comes first: sum
// ws stays far from overflow for any weight.
__device__ __forceinline__ f32x4 finish4(i32x4 sum, const float (&ws)[4], const float (&add)[4],
                                         float xs)
{
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)sum[i] * ws[i] * xs + add[i];
    return v;
}

// Rows r .. r + 3 of token t (those that y has).
template <typename Out>
__device__ __forceinline__ void store4(const LinearArgs& a, int64_t t, int r, f32x4 v)
{
    Out* y = static_cast<Out*>(a.y) + t * a.rows + r;
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
__device__ __forceinline__ i32x4 chunk16(const int8_t* row, int k, int len)
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
                                         const int8_t* const (&xrow)[kTok], int k, int cols,
                                         int g, i32x4 (&acc)[kTok])
{
    if constexpr (!kPacked) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = k + 32 * g + 16 * h;
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
            const int c = k + 64 * g + 32 * h;
            const i32x4 w = chunk16<kGuard>(wrow, c / 2, cols / 2);
            const int idx = !kGuard || c < cols ? (int)mrow[c / 32] : 0x44444444;
            const int b = k + 64 * (g / 2) + 32 * h + 16 * (g % 2);
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
    const int r0 = blockIdx.x % a.grid.tm * 16, t0 = blockIdx.x / a.grid.tm * (16 * kTok);
    // rows and tokens past the end repeat the last one; their results are dropped
    const int64_t r = least(r0 + (lane & 15), a.rows - 1);
    const int8_t* wrow = a.w + r * (kPacked ? a.cols / 2 : a.cols);
    const uint32_t* mrow = kPacked ? a.meta + r * (a.cols / 32) : nullptr;
    const int8_t* xrow[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        xrow[j] = a.x + (int64_t)least(t0 + 16 * j + (lane & 15), a.tokens - 1) * a.cols;
    }
    i32x4 acc[kTok] = {};
    const int whole = a.cols / kStep;
    int s = wave;
    for (; s + 3 * kFewWaves < whole; s += 4 * kFewWaves)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            few_step<kTok, kPacked, false>(wrow, mrow, xrow, (s + u * kFewWaves) * kStep, a.cols, g,
                                           acc);
    for (; s < whole; s += kFewWaves)
        few_step<kTok, kPacked, false>(wrow, mrow, xrow, s * kStep, a.cols, g, acc);
    if (whole * kStep < a.cols && wave == whole % kFewWaves)
        few_step<kTok, kPacked, true>(wrow, mrow, xrow, whole * kStep, a.cols, g, acc);
#pragma unroll
    for (int j = 0; j < kTok; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    for (int j = wave; j < kTok; j += kFewWaves) {
        i32x4 sum = {};
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) sum += part[v][j][lane];
        const int t = t0 + 16 * j + (lane & 15), ro = r0 + 4 * g;
        if (t >= a.tokens || ro >= a.rows) continue;
        float ws[4], add[4];
        row_scales(a, ro, ws, add);
        store4<Out>(a, t, ro, finish4(sum, ws, add, a.xs[t]));
    }
}

// --------------------------------------------------------------- many tokens
// A block makes one tile (mm.hpp) over steps of 128 columns, in two LDS buffers.
// A wave multiplies half a step's operands while it reads the next half's, row
// by row: past a row's products its registers take the next half's row.  One
// barrier a step, between the halves: past it every wave holds all it needs of
// this step's buffer, which takes the step after the next, and the next step's
// buffer, loading for a whole step, is complete.

// Rows row0 .. of an operand of `n` rows of `len` bytes, kBytes of each, that
// this thread brings to LDS.  Rows of 128 bytes lie as k-rows (mm.hpp); in rows
// of 64, place j ^ spread(row) holds chunk j, so that 16 lanes reading the same
// chunk of 16 rows cover all the LDS banks, and so do any aligned eight.
// kWhole: rows are whole 16-byte chunks.
template <int kTile, int kBytes, bool kWhole>
struct Rows {
    static constexpr int kThreads = Tile<kTile>::kThreads;
    static constexpr int kLoads = kTile * kBytes / (16 * kThreads);
    static constexpr int kChunks = kBytes / 16;
    const uint8_t* base;
    int left, len; // rows from row0 on, and their bytes
    uint32_t at;   // byte offset of load 0 from base

    __device__ __forceinline__ Rows(const int8_t* p, int row0, int n, int len_)
        : base(reinterpret_cast<const uint8_t*>(p) + (int64_t)row0 * len_), left(n - row0),
          len(len_), at((uint32_t)row(0) * len_ + 16 * chunk())
    {
    }
    __device__ __forceinline__ static int spread(int row)
    {
        return kChunks == 8 ? row & 7 : ((row >> 1) & 3) ^ ((row >> 3) & 1);
    }
    // Row and chunk of this thread's load i (the chunk is the same for all: the
    // rows differ by a multiple of sixteen).
    __device__ __forceinline__ static int row(int i)
    {
        return (i * kThreads + (int)threadIdx.x) / kChunks;
    }
    __device__ __forceinline__ static int chunk() { return (threadIdx.x % kChunks) ^ spread(row(0)); }
    // Load i of bytes k .. k + kBytes - 1 of the rows; zeros past the end.
    __device__ __forceinline__ void stage(int i, int k, ROI_LDS uint8_t* dst) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const bool live = row(i) < left && k + 16 * chunk() < len;
        if constexpr (kWhole)
            load_to_lds<false>(buffer_at(base + k), live ? at : kNowhere,
                               i * (kThreads / kChunks) * len, dst + (i * kThreads + wave * 64) * 16);
        else
            lds_write(dst + (i * kThreads + threadIdx.x) * 16,
                      live ? load_row<Quad>(base + (int64_t)row(i) * len, k + 16 * chunk(), len)
                           : Quad{});
    }
};

// A tile's results from a wave's sums: a part of a cut tile as it is, else scaled
// and through LDS (all of which is free) to y.
template <int kTile, typename Out>
__device__ __forceinline__ void write_tile(const LinearArgs& a, const Piece& piece,
                                           const i32x4 (&acc)[Tile<kTile>::kI][Tile<kTile>::kJ],
                                           ROI_LDS uint8_t* base)
{
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r0 = piece.m * kTile + wave / Tile<kTile>::kAcross * 16 * kI;
    const int t0 = piece.n * kTile + wave % Tile<kTile>::kAcross * 16 * kJ;
    if (piece.part >= 0) {
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                *reinterpret_cast<i32x4*>(a.partial + part_at<kTile>(piece.part, wave, i, j, lane)) =
                    acc[i][j];
        return;
    }
    // every scale before the first store, which might overwrite one for all the
    // compiler knows
    float ws[kI][4], add[kI][4], xs[kJ];
#pragma unroll
    for (int i = 0; i < kI; ++i) row_scales(a, r0 + 16 * i + 4 * g, ws[i], add[i]);
#pragma unroll
    for (int j = 0; j < kJ; ++j) xs[j] = a.xs[least(t0 + 16 * j + (lane & 15), a.tokens - 1)];
    // as many blocks of 16 tokens at a time as fit this wave's LDS
    using Lines = RowsOut<kI, 4 * sizeof(Out)>;
    constexpr int kAtATime = kTile * kRowBytes * 4 / Tile<kTile>::kWaves / (16 * Lines::kRow) < kJ
                                 ? kTile * kRowBytes * 4 / Tile<kTile>::kWaves / (16 * Lines::kRow)
                                 : kJ;
    static_assert(kAtATime >= 1 && kJ % kAtATime == 0, "results pass LDS");
    ROI_LDS uint8_t* mine = base + wave * (kAtATime * 16 * Lines::kRow);
#pragma unroll
    for (int first = 0; first < kJ; first += kAtATime) {
#pragma unroll
        for (int j = 0; j < kAtATime; ++j)
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const f32x4 v = finish4(acc[i][first + j], ws[i], add[i], xs[first + j]);
                ROI_LDS uint8_t* at = Lines::at(mine, 16 * j + (lane & 15), i, g);
                if constexpr (sizeof(Out) == 2)
                    *reinterpret_cast<ROI_LDS u32x2*>(at) =
                        u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
                else
                    *reinterpret_cast<ROI_LDS f32x4*>(at) = v;
            }
#pragma unroll
        for (int n = 0; n < 16 * kAtATime / Lines::kAtOnce; ++n) {
            int row, chunk;
            const Quad v = Lines::get(mine, n, row, chunk);
            const int t = t0 + 16 * first + row;
            const int r = r0 + chunk * (int)(16 / sizeof(Out));
            using Bits = std::conditional_t<sizeof(Out) == 2, uint16_t, uint32_t>;
            if (t < a.tokens)
                store_chunk(static_cast<Bits*>(a.y) + (int64_t)t * a.rows, r, a.rows, v);
        }
    }
}

template <int kTile, bool kWhole, typename Out>
__global__ __launch_bounds__(Tile<kTile>::kThreads) void linear_tile_kernel(LinearArgs a)
{
    constexpr int kTileBytes = kTile * kRowBytes;
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0][0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Tile<kTile>::kAcross * 16 * kI, wn = wave % Tile<kTile>::kAcross * 16 * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int r0 = piece.m * kTile, t0 = piece.n * kTile;

    i32x4 acc[kI][kJ] = {};
    using R = Rows<kTile, kRowBytes, kWhole>;
    const R wrows(a.w, r0, a.rows, a.cols), xrows(a.x, t0, a.tokens, a.cols);
    constexpr int kLoads = R::kLoads;
    auto buffer = [&](int s) { return base + (s & 1) * 2 * kTileBytes; };
    // loads `first` .. of step s, of the 2 kLoads that bring both tiles
    auto stage = [&](int s, int first, int count) {
        for (int i = first; i < first + count; ++i)
            if (i < kLoads)
                wrows.stage(i, (piece.first + s) * kRowBytes, buffer(s));
            else
                xrows.stage(i - kLoads, (piece.first + s) * kRowBytes, buffer(s) + kTileBytes);
    };
    struct Half {
        i32x4 w[kI], x[kJ];
    };
    auto read_w = [&](int s, int h, Half& f, int i) {
        f.w[i] = lds_read<i32x4>(buffer(s) + (wm + 16 * i + (lane & 15)) * kRowBytes +
                                 ((4 * h + g) ^ (lane & 7)) * 16);
    };
    auto read_x = [&](int s, int h, Half& f, int j) {
        f.x[j] = lds_read<i32x4>(buffer(s) + kTileBytes + (wn + 16 * j + (lane & 15)) * kRowBytes +
                                 ((4 * h + g) ^ (lane & 7)) * 16);
    };
    // the products of a half, beside the reads of half h of step s and (kLoad)
    // the loads of step s + 1: past the sum's end these bring zeros and those
    // read them, and neither is used
    auto half = [&](const Half& f, int s, int h, Half& next, auto load) {
        constexpr int kPart = 2 * kLoads / kI;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) read_x(s, h, next, i);
            read_w(s, h, next, i);
            if (decltype(load)::value) stage(s + 1, i * kPart, kPart);
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.w[i], f.x[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    static_assert(2 * kLoads % kI == 0, "loads are spread over the rows");
    if (piece.count > 0) {
        Half lo, hi;
        stage(0, 0, 2 * kLoads);
        stage(1, 0, 2 * kLoads);
        loads_barrier();
#pragma unroll
        for (int i = 0; i < kI; ++i) read_w(0, 0, lo, i);
#pragma unroll
        for (int j = 0; j < kJ; ++j) read_x(0, 0, lo, j);
        for (int s = 0; s < piece.count; ++s) {
            half(lo, s, 1, hi, std::false_type{});
            loads_barrier();
            half(hi, s + 1, 0, lo, std::true_type{});
        }
        loads_barrier();
    }
    write_tile<kTile, Out>(a, piece, acc, base);
}

// The same with 2:4 weights: a step of 128 columns is one instruction's sum, so
// that a step's operands are read while the step before is multiplied, and a
// step's tiles (64 bytes a weight row, its four metadata words, 128 bytes a
// token) have two steps to arrive, in three LDS buffers.
template <int kTile, typename Out>
__global__ __launch_bounds__(Tile<kTile>::kThreads) void linear_packed_kernel(LinearArgs a)
{
    constexpr int kI = Tile<kTile>::kI, kJ = Tile<kTile>::kJ;
    constexpr int kThreads = Tile<kTile>::kThreads;
    constexpr int kW = kTile * 64, kX = kTile * 128, kM = kTile * 16, kStage = kW + kX + kM;
    __shared__ __attribute__((aligned(16))) uint8_t lds[3][kStage];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0][0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Tile<kTile>::kAcross * 16 * kI, wn = wave % Tile<kTile>::kAcross * 16 * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int r0 = piece.m * kTile, t0 = piece.n * kTile;

    i32x4 acc[kI][kJ] = {};
    using W = Rows<kTile, 64, true>;
    using X = Rows<kTile, 128, true>;
    const W wrows(a.w, r0, a.rows, a.cols / 2);
    const X xrows(a.x, t0, a.tokens, a.cols);
    // metadata: a word a lane, four words a row
    constexpr int kMetaLoads = kTile * 4 / kThreads;
    const int words = a.cols / 32, word = threadIdx.x % 4;
    const uint32_t* meta = a.meta + (int64_t)r0 * words;
    constexpr int kLoads = W::kLoads + X::kLoads + kMetaLoads;
    static_assert(kLoads % kI == 0, "loads are spread over the rows");
    auto stage = [&](int s, int first, int count, ROI_LDS uint8_t* dst) {
        const int k = (piece.first + s) * 128;
        for (int i = first; i < first + count; ++i) {
            if (i < W::kLoads) {
                wrows.stage(i, k / 2, dst);
            } else if (i < W::kLoads + X::kLoads) {
                xrows.stage(i - W::kLoads, k, dst + kW);
            } else {
                const int l = i - W::kLoads - X::kLoads;
                const int row = (l * kThreads + (int)threadIdx.x) / 4;
                const bool live = row < a.rows - r0 && k + 32 * word < a.cols;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    buffer_at(meta + k / 32),
                    (ROI_LDS void*)(dst + kW + kX + (l * kThreads + wave * 64) * 4), 4,
                    live ? 4 * (row * words + word) : (int)kNowhere, 0, 0, 0);
            }
        }
    };
    struct Step {
        i32x4 w[kI];
        int m[kI];
        i32x8 x[kJ];
    };
    const int from_w = (wm + (lane & 15)) * 64 + (g ^ W::spread(lane & 15)) * 16;
    const int from_m = kW + kX + (wm + (lane & 15)) * 16 + g * 4;
    const int from_x = kW + (wn + (lane & 15)) * 128 + (g ^ X::spread(lane & 15)) * 16;
    auto read_w = [&](ROI_LDS uint8_t* src, Step& f, int i) {
        f.w[i] = lds_read<i32x4>(src + from_w + i * 16 * 64);
        f.m[i] = lds_read<int>(src + from_m + i * 16 * 16);
    };
    auto read_x = [&](ROI_LDS uint8_t* src, Step& f, int j) {
        const i32x4 lo = lds_read<i32x4>(src + from_x + j * 16 * 128);
        const i32x4 hi = lds_read<i32x4>(src + (from_x ^ 64) + j * 16 * 128);
        f.x[j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // the products of a step, beside the reads of the next (at src) and the loads
    // of step s, to dst; a block of tokens is read past the last product of the
    // one before it (there are no registers for both)
    auto step = [&](const Step& f, Step& next, ROI_LDS uint8_t* src, int s, ROI_LDS uint8_t* dst) {
        constexpr int kPart = kLoads / kI;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            read_w(src, next, i);
            stage(s, i * kPart, kPart, dst);
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                acc[i][j] = __builtin_amdgcn_smfmac_i32_16x16x128_i8(f.w[i], f.x[j], acc[i][j],
                                                                     f.m[i], 0, 0);
                if (i == kI - 1) read_x(src, next, j);
            }
            keep_order();
        }
    };
    if (piece.count > 0) {
        ROI_LDS uint8_t *b0 = base, *b1 = base + kStage, *b2 = base + 2 * kStage;
        Step even, odd;
        stage(0, 0, kLoads, b0);
        stage(1, 0, kLoads, b1);
        stage(2, 0, kLoads, b2);
        loads_barrier<2 * kLoads>();
#pragma unroll
        for (int i = 0; i < kI; ++i) read_w(b0, even, i);
#pragma unroll
        for (int j = 0; j < kJ; ++j) read_x(b0, even, j);
        // past the end of the sum or of this part, loads are in bounds or zeros,
        // and unused
        int s = 0;
        for (; s + 2 <= piece.count; s += 2) {
            loads_barrier<kLoads>();
            step(even, odd, b1, s + 3, b0);
            loads_barrier<kLoads>();
            step(odd, even, b2, s + 4, b1);
            ROI_LDS uint8_t* const t = b0;
            b0 = b2;
            b2 = b1;
            b1 = t;
        }
        if (s < piece.count) {
            loads_barrier<kLoads>();
            step(even, odd, b1, s + 3, b0);
        }
        loads_barrier();
    }
    static_assert(3 * kStage >= 4 * kTile * kRowBytes, "results pass LDS");
    write_tile<kTile, Out>(a, piece, acc, base);
}

// The sums of the tiles that were cut: one wave for the 16 x 64 results that a
// wave of the tile's kernel held at one i.
template <int kTile, typename Out>
__global__ __launch_bounds__(64) void linear_sum_kernel(LinearArgs a)
{
    using T = Tile<kTile>;
    const int lane = threadIdx.x, g = lane >> 4;
    const int i = blockIdx.x % T::kI, wave = blockIdx.x / T::kI % T::kWaves;
    const uint32_t tile = blockIdx.x / (T::kI * T::kWaves);
    const Piece piece = tile_piece(a.grid, a.grid.full + tile);
    i32x4 sum[T::kJ] = {};
    for (uint32_t p = 0; p < a.grid.splits; ++p)
#pragma unroll
        for (int j = 0; j < T::kJ; ++j)
            sum[j] += *reinterpret_cast<const i32x4*>(
                a.partial + part_at<kTile>((int64_t)tile * a.grid.splits + p, wave, i, j, lane));
    const int r = piece.m * kTile + 16 * (wave / T::kAcross * T::kI + i) + 4 * g;
    if (r >= a.rows) return;
    float ws[4], add[4];
    row_scales(a, r, ws, add);
#pragma unroll
    for (int j = 0; j < T::kJ; ++j) {
        const int t = piece.n * kTile + 16 * (wave % T::kAcross * T::kJ + j) + (lane & 15);
        if (t < a.tokens) store4<Out>(a, t, r, finish4(sum[j], ws, add, a.xs[t]));
    }
}

// Blocks of one launch: fewer than 2^32 threads.
bool fits(int64_t blocks, int threads) { return blocks <= (int64_t)(0xFFFFFFFFu / (uint32_t)threads); }

template <int kTile, typename Out>
void launch_tiles(const LinearArgs& a, hipStream_t stream)
{
    using T = Tile<kTile>;
    const dim3 grid(a.grid.blocks()), block(T::kThreads);
    if (a.meta)
        hipLaunchKernelGGL((linear_packed_kernel<kTile, Out>), grid, block, 0, stream, a);
    else if (a.cols % 16 == 0)
        hipLaunchKernelGGL((linear_tile_kernel<kTile, true, Out>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((linear_tile_kernel<kTile, false, Out>), grid, block, 0, stream, a);
    if (a.grid.rest() > 0)
        hipLaunchKernelGGL((linear_sum_kernel<kTile, Out>), dim3(a.grid.rest() * T::kI * T::kWaves),
                           dim3(64), 0, stream, a);
}

// Whether the call takes the kernel for few tokens, which needs no workspace.
bool few(int64_t tokens) { return tokens <= 64; }

Cut cut_linear(int64_t tokens, int64_t rows, int64_t cols, bool packed)
{
    return cut_product(rows, tokens, cols, kRowBytes, packed ? kPackedCost : kLinearCost);
}

template <typename Out>
int launch(LinearArgs a, hipStream_t stream)
{
    if (few(a.tokens)) {
        const int tok = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
        const int64_t tm = (a.rows + 15) / 16, tn = ((int64_t)a.tokens + 16 * tok - 1) / (16 * tok);
        if (!fits(tm * tn, 64 * kFewWaves))
            return fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
        a.grid.tm = (uint32_t)tm;
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
    const Cut c = cut_linear(a.tokens, a.rows, a.cols, a.meta != nullptr);
    if (!c.fits) return fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
    a.grid = Grid{(uint32_t)c.tm, (uint32_t)c.tn, (uint32_t)c.full, (uint32_t)c.splits, (int)c.steps};
    if (c.tile == 256)
        launch_tiles<256, Out>(a, stream);
    else
        launch_tiles<128, Out>(a, stream);
    return launch_status("roi_linear_i8");
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_i8_workspace(int64_t tokens, int64_t rows, int64_t cols, int packed)
{
    if (check_linear_sizes(tokens, rows, cols)) return -1;
    ok();
    return few(tokens) ? 0 : cut_linear(tokens, rows, cols, packed != 0).bytes;
}

extern "C" int roi_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq,
                             const uint32_t* meta, const float* ws, const uint16_t* bias,
                             int64_t tokens, int64_t rows, int64_t cols, void* y, int dtype,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const int64_t need =
        few(tokens) ? 0 : cut_linear(tokens, rows, cols, meta != nullptr).bytes;
    if (int st = validate_linear_i8(xq, xs, wq, meta, ws, bias, tokens, rows, cols, y, dtype,
                                    workspace, workspace_bytes, need, &todo))
        return st;
    if (!todo) return ok();
    const LinearArgs a{xq, xs, wq, meta, ws, bias, y, static_cast<int*>(workspace), (int)tokens,
                       (int)rows, (int)cols, {}};
    return dtype == ROI_BF16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}
