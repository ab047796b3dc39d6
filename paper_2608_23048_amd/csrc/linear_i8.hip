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
//   v_smfmac_i32_32x32x64_i8: the same with 32 rows, g = l / 32 and 64 columns
//     (the second operand's at 16 g and 32 + 16 g); result rows 8 (i / 4) + 4 g +
//     i % 4 of column l % 32 in element i of 16.
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
    int* partial; // int32 parts of tiles (Held::part_at)
    int tokens, rows, cols;
    Grid grid; // tiles along the rows and the tokens (few tokens: grid.tm alone)
};

// The scales of rows r .. r + 3, and what is added to their results: without a
// bias -0, which changes nothing.
__device__ __forceinline__ void row_scales(const LinearArgs& a, int r, f32x4& ws, f32x4& add)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int rc = least(r + e, a.rows - 1);
        ws[e] = a.ws[rc];
        add[e] = a.bias ? bf16_bits_to_float(a.bias[rc]) : -0.0f;
    }
}

// Four results from their exact sums, which are rounded to fp32 first (exact there
// up to 2^24).  The scale of the weight comes first: sums are below 2^31, so with ws
// below 2^97 (weights below 2e31) sum ws is finite; past that it can be an infinity,
// and so can the result, also where xs would bring it back.
__device__ __forceinline__ f32x4 finish4(i32x4 sum, f32x4 ws, f32x4 add, float xs)
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
// A block owns 16 kRow weight rows and up to kTokens tokens (8, or a multiple of
// 16); its waves share out the sum and add up their parts in LDS.  The weight is
// read once: bound by its bytes (68 MB in 12 us by itself: 16 tokens through 3584 x
// 18944).  A wave brings its steps of the sum (128 columns, 256 of a 2:4 weight)
// to a ring of kDepth slots in LDS of its own and needs no barrier.  Through LDS,
// because eight lanes then read 128 consecutive bytes of a row; operands loaded
// straight to registers are 64 separate pieces of 16 bytes a load, and the
// vector cache takes one a cycle: 14 us against 11 for a token through the 2:4
// 18944 x 3584 layer, 21.5 against 16 for 16 tokens through the dense 3584 x 18944.
template <int kWaves, int kRow, int kTokens, int kDepth, bool kPacked, bool kWhole, typename Out>
__global__ __launch_bounds__(64 * kWaves) void linear_few_kernel(LinearArgs a)
{
    constexpr int kTok = (kTokens + 15) / 16;
    constexpr int kHalves = kPacked ? 2 : 1; // of 128 columns of x
    constexpr int kXHalf = kTokens * 128;
    constexpr int kW = kRow * 2048, kX = kHalves * kXHalf, kM = kPacked ? kRow * 512 : 0;
    constexpr int kSlot = kW + kX + kM;
    constexpr int kLoads = 2 * kRow + kTokens / 8 * kHalves + (kPacked ? 2 * kRow : 0);
    constexpr int kColumns = 128 * kHalves;
    static_assert(kRow * kTok * 1024 <= kDepth * kSlot, "the parts of the sum take the ring's place");
    __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves][kDepth * kSlot];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = scalar(threadIdx.x >> 6);
    ROI_LDS uint8_t* ring = (ROI_LDS uint8_t*)&lds[0][0] + wave * (kDepth * kSlot);
    const int r0 = scalar(blockIdx.x % a.grid.tm) * (16 * kRow);
    const int t0 = scalar(blockIdx.x / a.grid.tm) * kTokens;

    // a load brings 128 bytes of eight rows: this lane's of the eight, its chunk
    // of a row (kept at the place of k-rows, mm.hpp), and its metadata word
    const int row = lane / 8, chunk = (lane % 8) ^ row, word = lane % 8;
    const int wlen = kPacked ? a.cols / 2 : a.cols, words = a.cols / 32;
    const uint8_t* wbase = reinterpret_cast<const uint8_t*>(a.w) + (int64_t)r0 * wlen;
    const uint8_t* xbase = reinterpret_cast<const uint8_t*>(a.x) + (int64_t)t0 * a.cols;
    const uint32_t* mbase = kPacked ? a.meta + (int64_t)r0 * words : nullptr;
    // step s of the sum (past its end: zeros) into a slot
    auto stage = [&](int s, ROI_LDS uint8_t* slot) {
        const int k = s * kColumns;
        auto bring = [&](const uint8_t* base, int first, int rows, int from, int len,
                         ROI_LDS uint8_t* dst) {
            const bool live = first + row < rows && from + 16 * chunk < len;
            load_to_lds<false>(buffer_at(base + from),
                               live ? (uint32_t)row * len + 16 * chunk : kNowhere, first * len, dst);
        };
#pragma unroll
        for (int i = 0; i < 2 * kRow; ++i)
            bring(wbase, 8 * i, a.rows - r0, k / kHalves, wlen, slot + i * 1024);
#pragma unroll
        for (int i = 0; i < kTokens / 8 * kHalves; ++i)
            bring(xbase, 8 * (i / kHalves), a.tokens - t0, k + 128 * (i % kHalves), a.cols,
                  slot + kW + (i % kHalves) * kXHalf + i / kHalves * 1024);
        if constexpr (kPacked) {
#pragma unroll
            for (int i = 0; i < 2 * kRow; ++i) {
                const bool live = 8 * i + row < a.rows - r0 && k + 32 * word < a.cols;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    buffer_at(mbase + k / 32), (ROI_LDS void*)(slot + kW + kX + i * 256), 4,
                    live ? 4 * (row * words + word) : (int)kNowhere, 4 * 8 * i * words, 0, 0);
            }
        }
    };
    // Rows that end within 16 bytes (dense weights) go by registers: fetched kAhead
    // steps ahead, at any address, rows past the end the last again.
    constexpr int kAhead = kWhole ? 1 : 4, kPieces = kWhole ? 1 : 2 * kRow + kTokens / 8;
    Quad held[kAhead][kPieces];
    auto fetch = [&](int s, Quad (&to)[kPieces]) {
        const int k = s * 128;
        auto start = [&](int i) {
            const bool w = i < 2 * kRow;
            const int rows = w ? a.rows - r0 : a.tokens - t0;
            return (w ? wbase : xbase) +
                   (int64_t)least(8 * (w ? i : i - 2 * kRow) + row, rows - 1) * a.cols;
        };
        if (k + 128 <= a.cols) { // the same for the wave
#pragma unroll
            for (int i = 0; i < kPieces; ++i) to[i] = load_any<Quad>(start(i) + k + 16 * chunk);
        } else if (k < a.cols) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                to[i] = load_row<Quad>(start(i), k + 16 * chunk, a.cols);
        }
    };
    auto put = [&](ROI_LDS uint8_t* slot, const Quad (&from)[kPieces]) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            lds_write(slot + (i < 2 * kRow ? i * 1024 : kW + (i - 2 * kRow) * 1024) + lane * 16,
                      from[i]);
    };
    i32x4 acc[kRow][kTok] = {};
    const int from = (lane & 15) * 128 + (g ^ (lane & 7)) * 16;
    // of eight tokens, the second eight lanes read the first's again
    const int from_x = (lane & (kTokens < 16 ? 7 : 15)) * 128 + (g ^ (lane & 7)) * 16;
    auto multiply = [&](ROI_LDS uint8_t* slot) {
#pragma unroll
        for (int h = 0; h < 2; ++h) { // chunk 4 h + g: the place's third bit flips
            i32x4 w[kRow];
#pragma unroll
            for (int i = 0; i < kRow; ++i) w[i] = lds_read<i32x4>(slot + i * 2048 + (from ^ (64 * h)));
            if constexpr (kPacked) {
                int m[kRow];
                i32x8 x[kTok];
#pragma unroll
                for (int i = 0; i < kRow; ++i)
                    m[i] = lds_read<int>(slot + kW + kX + i * 512 + (lane & 15) * 32 + h * 16 + g * 4);
#pragma unroll
                for (int j = 0; j < kTok; ++j) {
                    ROI_LDS uint8_t* p = slot + kW + h * kXHalf + j * 2048;
                    x[j] = __builtin_shufflevector(lds_read<i32x4>(p + from_x),
                                                   lds_read<i32x4>(p + (from_x ^ 64)), 0, 1, 2, 3, 4, 5,
                                                   6, 7);
                }
#pragma unroll
                for (int i = 0; i < kRow; ++i)
#pragma unroll
                    for (int j = 0; j < kTok; ++j)
                        acc[i][j] = __builtin_amdgcn_smfmac_i32_16x16x128_i8(w[i], x[j], acc[i][j],
                                                                             m[i], 0, 0);
            } else {
                i32x4 x[kTok];
#pragma unroll
                for (int j = 0; j < kTok; ++j)
                    x[j] = lds_read<i32x4>(slot + kW + j * 2048 + (from_x ^ (64 * h)));
#pragma unroll
                for (int i = 0; i < kRow; ++i)
#pragma unroll
                    for (int j = 0; j < kTok; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0,
                                                                          0);
            }
        }
    };
    // step n of this wave is step wave + n kWaves of the sum
    const int steps = (a.cols + kColumns - 1) / kColumns;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    if (mine > 0) {
        int slot = 0;
        auto next_slot = [&] { slot = slot + kSlot < kDepth * kSlot ? slot + kSlot : 0; };
        if constexpr (kWhole) {
#pragma unroll
            for (int n = 0; n < kDepth; ++n) stage(wave + n * kWaves, ring + n * kSlot);
            for (int n = 0; n < mine; ++n) {
                loads_wait<(kDepth - 1) * kLoads>();
                multiply(ring + slot);
                // the slot is read: its values are in registers before its next loads
                keep_order();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                stage(wave + (n + kDepth) * kWaves, ring + slot);
                next_slot();
            }
            loads_wait<0>();
        } else {
#pragma unroll
            for (int n = 0; n < kAhead; ++n) fetch(wave + n * kWaves, held[n]);
            for (int n = 0; n < mine; n += kAhead) {
#pragma unroll
                for (int h = 0; h < kAhead; ++h) {
                    if (n + h >= mine) break;
                    put(ring + slot, held[h]); // a wave's LDS operations are done in order
                    fetch(wave + (n + h + kAhead) * kWaves, held[h]);
                    multiply(ring + slot);
                    next_slot();
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRow; ++i)
#pragma unroll
        for (int j = 0; j < kTok; ++j)
            *reinterpret_cast<ROI_LDS i32x4*>(ring + ((i * kTok + j) * 64 + lane) * 16) = acc[i][j];
    __syncthreads();
    for (int b = wave; b < kRow * kTok; b += kWaves) {
        const int in = 16 * (b % kTok) + (lane & 15);
        const int t = t0 + in, r = r0 + 16 * (b / kTok) + 4 * g;
        if (in >= kTokens || t >= a.tokens || r >= a.rows) continue;
        f32x4 ws, add;
        row_scales(a, r, ws, add);
        const float xs = a.xs[t];
        i32x4 sum = {};
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
            sum += lds_read<i32x4>((ROI_LDS uint8_t*)&lds[0][0] + v * (kDepth * kSlot) +
                                   (b * 64 + lane) * 16);
        store4<Out>(a, t, r, finish4(sum, ws, add, xs));
    }
}

// --------------------------------------------------------------- many tokens
// A block makes one tile (mm.hpp) over steps of 128 columns, in kRing LDS buffers.
// A wave multiplies half a step's operands while it reads the next half's, row
// by row: past a row's products its registers take the next half's row.  One
// barrier a step, between the halves: past it every wave holds all it needs of
// this step's buffer, which takes the step kRing later, and the next step's
// buffer, loading for kRing - 1 steps, is complete.  256-tiles, and two 128-tiles
// on a compute unit, have LDS for two; a 128-tile that has a compute unit to
// itself takes four, and eight waves: 512 tokens through 3584 x 3584 take 16.1 us
// so and 21.3 with two and four.  8192 tokens through 18944 x 3584: 440 us in
// single passes, 2.5 POP/s, with the matrix cores busy for 66 % of the time at 1.8
// GHz (476 in the median of passes back to back, as the clock falls); a tile's first
// loads and its results are a quarter of its 28 steps' time.

// Rows row0 .. of an operand of `n` rows of `len` bytes, kRowBytes of each, that
// this thread brings to LDS, where place j ^ spread(row) of a row holds its chunk
// j.  A 16-byte LDS read goes by 16 lanes at a time, which are, of the wave's
// first half, 0-3, 12-15, 20-23 and 24-27, then the others; the spreads give any
// such 16 lanes all the banks when 16 consecutive lanes (kBlock 16) or 32 read
// the same chunk of as many rows.  Their lengths are multiples of 16 bytes.
template <typename T, int kBlock>
struct Rows {
    static constexpr int kThreads = T::kThreads;
    static constexpr int kLoads = T::kTile * kRowBytes / (16 * kThreads);
    static constexpr int kChunks = kRowBytes / 16;
    static_assert(kChunks == 8, "the spreads below");
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
        return kBlock == 16 ? row & 7 : (row >> 1) & 7;
    }
    // Row and chunk of this thread's load i (the chunk is the same for all: the
    // rows differ by a multiple of sixteen).
    __device__ __forceinline__ static int row(int i)
    {
        return (i * kThreads + (int)threadIdx.x) / kChunks;
    }
    __device__ __forceinline__ static int chunk() { return (threadIdx.x % kChunks) ^ spread(row(0)); }
    // Load i of bytes k .. k + kRowBytes - 1 of the rows; zeros past the end.
    __device__ __forceinline__ void stage(int i, int k, ROI_LDS uint8_t* dst) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const bool live = row(i) < left && k + 16 * chunk() < len;
        load_to_lds<false>(buffer_at(base + k), live ? at : kNowhere, i * (kThreads / kChunks) * len,
                           dst + (i * kThreads + wave * 64) * 16);
    }
};

// Quad q of a block's sums.
__device__ __forceinline__ i32x4 quad_of(const i32x4& v, int) { return v; }
__device__ __forceinline__ i32x4 quad_of(const i32x16& v, int q)
{
    return i32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
}

// The scales of a whole tile's rows and tokens, and what is added to the rows'
// results: loaded ahead of the tile's first steps and kept in LDS to its end, where
// a wave would otherwise wait for them.
template <typename T>
struct Scales {
    static constexpr int kBytes = 3 * 4 * T::kTile;
    static_assert(T::kTile <= T::kThreads, "one of each a thread");
    float ws, add, xs;

    __device__ __forceinline__ Scales(const LinearArgs& a, const Piece& piece)
    {
        if (piece.part >= 0 || threadIdx.x >= T::kTile) return;
        const int r = least(piece.m * T::kTile + (int)threadIdx.x, a.rows - 1);
        ws = a.ws[r];
        xs = a.xs[least(piece.n * T::kTile + (int)threadIdx.x, a.tokens - 1)];
        add = a.bias ? bf16_bits_to_float(a.bias[r]) : -0.0f;
    }
    __device__ __forceinline__ void keep(const Piece& piece, ROI_LDS uint8_t* lds) const
    {
        if (piece.part >= 0 || threadIdx.x >= T::kTile) return;
        ROI_LDS float* p = reinterpret_cast<ROI_LDS float*>(lds) + threadIdx.x;
        p[0] = ws;
        p[T::kTile] = add;
        p[2 * T::kTile] = xs;
    }
};

// A tile's results from a wave's sums: a part of a cut tile as it is, else scaled
// and through LDS (all of which is free) to y.
template <typename T, int kBlock, typename Out, typename Sum>
__device__ __forceinline__ void write_tile(
    const LinearArgs& a, const Piece& piece,
    const Sum (&acc)[Held<T, kBlock>::kI][Held<T, kBlock>::kJ], ROI_LDS uint8_t* base,
    const ROI_LDS uint8_t* scales)
{
    using H = Held<T, kBlock>;
    const int wave = scalar(threadIdx.x >> 6);
    const int r0 = piece.m * T::kTile + wave / T::kAcross * 16 * T::kI;
    const int t0 = piece.n * T::kTile + wave % T::kAcross * 16 * T::kJ;
    if (piece.part >= 0) {
#pragma unroll
        for (int i = 0; i < H::kI; ++i)
#pragma unroll
            for (int j = 0; j < H::kJ; ++j)
#pragma unroll
                for (int q = 0; q < H::kQuads; ++q)
                    *reinterpret_cast<i32x4*>(a.partial + H::part_at(piece.part, wave, i, j, q)) =
                        quad_of(acc[i][j], q);
        return;
    }
    const ROI_LDS uint8_t* row_scale = scales + 4 * (wave / T::kAcross * 16 * T::kI);
    const ROI_LDS uint8_t* token_scale =
        scales + 4 * (2 * T::kTile + wave % T::kAcross * 16 * T::kJ);
    float xs[H::kJ];
#pragma unroll
    for (int j = 0; j < H::kJ; ++j) xs[j] = lds_read<float>(token_scale + 4 * H::column(j));
    // as many blocks of tokens at a time as fit this wave's LDS
    using Lines = RowsOut<T::kI, 4 * sizeof(Out)>;
    constexpr int kFit = T::kTile * kRowBytes * 4 / T::kWaves / (kBlock * Lines::kRow);
    constexpr int kAtATime = kFit < H::kJ ? kFit : H::kJ;
    static_assert(kAtATime >= 1 && H::kJ % kAtATime == 0, "results pass LDS");
    ROI_LDS uint8_t* mine = base + wave * (kAtATime * kBlock * Lines::kRow);
#pragma unroll
    for (int first = 0; first < H::kJ; first += kAtATime) {
        // a row of blocks' scales are read ahead of the results before it: the
        // compiler keeps reads of LDS behind writes
        f32x4 ws[2][H::kQuads], add[2][H::kQuads];
        auto read = [&](int i) {
#pragma unroll
            for (int q = 0; q < H::kQuads; ++q) {
                ws[i & 1][q] = lds_read<f32x4>(row_scale + 16 * H::quad(i, q));
                add[i & 1][q] = lds_read<f32x4>(row_scale + 16 * H::quad(i, q) + 4 * T::kTile);
            }
        };
        read(0);
#pragma unroll
        for (int i = 0; i < H::kI; ++i) {
            if (i + 1 < H::kI) read(i + 1);
#pragma unroll
            for (int j = 0; j < kAtATime; ++j)
#pragma unroll
                for (int q = 0; q < H::kQuads; ++q) {
                    const f32x4 v = finish4(quad_of(acc[i][first + j], q), ws[i & 1][q],
                                            add[i & 1][q], xs[first + j]);
                    ROI_LDS uint8_t* at = Lines::at(mine, H::column(j), H::quad(i, q));
                    if constexpr (sizeof(Out) == 2)
                        *reinterpret_cast<ROI_LDS u32x2*>(at) =
                            u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
                    else
                        *reinterpret_cast<ROI_LDS f32x4*>(at) = v;
                }
        }
#pragma unroll 2 // code that runs once is fetched once: it is kept short
        for (int n = 0; n < kBlock * kAtATime / Lines::kAtOnce; ++n) {
            int row, chunk;
            const Quad v = Lines::get(mine, n, row, chunk);
            const int t = t0 + kBlock * first + row;
            const int r = r0 + chunk * (int)(16 / sizeof(Out));
            using Bits = std::conditional_t<sizeof(Out) == 2, uint16_t, uint32_t>;
            if (t < a.tokens)
                store_chunk(static_cast<Bits*>(a.y) + (int64_t)t * a.rows, r, a.rows, v);
        }
    }
}

template <typename T, int kRing, typename Out>
__global__ __launch_bounds__(T::kThreads, 2) void linear_tile_kernel(LinearArgs a)
{
    constexpr int kTile = T::kTile, kTileBytes = kTile * kRowBytes;
    constexpr int kI = T::kI, kJ = T::kJ;
    static_assert(kRing == 2 || kRing == 4, "slots are counted in bits");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[]; // kRing steps of two tiles
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::kAcross * 16 * kI, wn = wave % T::kAcross * 16 * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int r0 = piece.m * kTile, t0 = piece.n * kTile;

    i32x4 acc[kI][kJ] = {};
    using R = Rows<T, 16>;
    const R wrows(a.w, r0, a.rows, a.cols), xrows(a.x, t0, a.tokens, a.cols);
    constexpr int kLoads = R::kLoads;
    auto buffer = [&](int s) { return base + (s & (kRing - 1)) * 2 * kTileBytes; };
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
    // the products of a half, beside the reads of half h of step s and (kLoad) the
    // loads of step s + kRing - 1: past the sum's end these bring zeros and those
    // read them, and neither is used
    auto half = [&](const Half& f, int s, int h, Half& next, auto load) {
        constexpr int kPart = 2 * kLoads / kI;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) read_x(s, h, next, i);
            read_w(s, h, next, i);
            if (decltype(load)::value) stage(s + kRing - 1, i * kPart, kPart);
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.w[i], f.x[j], acc[i][j], 0, 0, 0);
            keep_order();
        }
    };
    static_assert(2 * kLoads % kI == 0, "loads are spread over the rows");
    const Scales<T> scales(a, piece);
    if (piece.count > 0) {
        Half lo, hi;
        for (int s = 0; s < kRing; ++s) stage(s, 0, 2 * kLoads);
        scales.keep(piece, base + kRing * 2 * kTileBytes);
        loads_barrier<(kRing - 1) * 2 * kLoads>();
#pragma unroll
        for (int i = 0; i < kI; ++i) read_w(0, 0, lo, i);
#pragma unroll
        for (int j = 0; j < kJ; ++j) read_x(0, 0, lo, j);
        for (int s = 0; s < piece.count; ++s) {
            half(lo, s, 1, hi, std::false_type{});
            loads_barrier<(kRing - 2) * 2 * kLoads>();
            half(hi, s + 1, 0, lo, std::true_type{});
        }
        loads_barrier();
    } else { // a sum over nothing
        scales.keep(piece, base + kRing * 2 * kTileBytes);
        __syncthreads();
    }
    write_tile<T, 16, Out>(a, piece, acc, base, base + kRing * 2 * kTileBytes);
}

// The same with 2:4 weights, on the 32 x 32 sparse instructions: a half step is
// 64 columns, whose second operand is 8 registers a block of 32 tokens (the 16 x
// 16 form takes 128 columns at once and twice the registers, too many to read
// ahead).  Weights and metadata come for two steps at a time, 128 and 32 bytes a
// row: requests to the L2 were what bound the step (a step at a time 26 million in
// 175 us for 4096 tokens through 3584 x 18944; so, 18 million in 163, and with no
// registers in scratch 156).  The
// tokens' tiles have kRing - 1 steps to arrive: two where a tile has a compute unit
// to itself (512 tokens through 3584 x 3584: 15.7 us, 17.6 with one), else one, for
// which there is LDS.  Of a 256-tile's step of 1870 cycles (at 1.8 GHz, which is
// what this load leaves) the matrix cores take 1024, the LDS reads 660 and the loads
// to LDS about 420; waves wait for 29 % of it, at the barrier and for the tokens.
template <int kTile, int kRing>
constexpr int packed_lds() { return kRing * kTile * 128 + 2 * kTile * (128 + 32); }
template <typename T, int kRing, typename Out>
__global__ __launch_bounds__(T::kThreads, 2) void linear_packed_kernel(LinearArgs a)
{
    using H = Held<T, 32>;
    constexpr int kTile = T::kTile;
    constexpr int kI = H::kI, kJ = H::kJ;
    constexpr int kThreads = T::kThreads;
    constexpr int kX = kTile * 128;                                    // of a step
    constexpr int kW = kTile * 128, kM = kTile * 32, kPair = kW + kM; // of two
    static_assert(kRing == 2 || kRing == 3, "the waits below");
    static_assert(packed_lds<T::kTile, kRing>() == kRing * kX + 2 * kPair, "the launch's");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    const int lane = threadIdx.x & 63, half_of = lane >> 5, in = lane & 31;
    const int wave = scalar(threadIdx.x >> 6);
    const int wm = wave / T::kAcross * 32 * kI, wn = wave % T::kAcross * 32 * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int r0 = piece.m * kTile, t0 = piece.n * kTile;

    i32x16 acc[kI][kJ] = {};
    using R = Rows<T, 32>;
    const R wrows(a.w, r0, a.rows, a.cols / 2), xrows(a.x, t0, a.tokens, a.cols);
    // metadata: a word a lane, eight words a row, word j at place j ^ (row / 4 & 7),
    // so that the words that 32 lanes read lie in the 32 banks of a 4-byte read
    constexpr int kMetaLoads = kTile * 8 / kThreads;
    const int words = a.cols / 32, word = (threadIdx.x % 8) ^ (threadIdx.x / 32 & 7);
    static_assert(kThreads / 8 % 32 == 0, "the same word for all of a thread's loads");
    const uint32_t* meta = a.meta + (int64_t)r0 * words;
    constexpr int kPairLoads = R::kLoads + kMetaLoads;
    // loads first .. of the tokens of step s
    auto stage_x = [&](int s, int first, int count, ROI_LDS uint8_t* dst) {
        for (int i = first; i < first + count; ++i)
            xrows.stage(i, (piece.first + s) * 128, dst);
    };
    // and of the weights and metadata of steps s and s + 1
    auto stage_w = [&](int s, int first, int count, ROI_LDS uint8_t* dst) {
        const int k = (piece.first + s) * 128;
        for (int i = first; i < first + count; ++i) {
            if (i < R::kLoads) {
                wrows.stage(i, k / 2, dst);
            } else {
                const int l = i - R::kLoads;
                const int row = (l * kThreads + (int)threadIdx.x) / 8;
                const bool live = row < a.rows - r0 && k + 32 * word < a.cols;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    buffer_at(meta + k / 32),
                    (ROI_LDS void*)(dst + kW + (l * kThreads + wave * 64) * 4), 4,
                    live ? 4 * (row * words + word) : (int)kNowhere, 0, 0, 0);
            }
        }
    };
    struct Half {
        i32x4 w[kI];
        int m[kI];
        i32x8 x[kJ];
    };
    // Half h of a step: the weight's chunk and the word 2 h + half_of, in the
    // second of two steps 4 more, the tokens' chunks 4 h + half_of and 4 h + 2 +
    // half_of; the places' bits flip with these.
    const int from_w = (wm + in) * 128 + (half_of ^ R::spread(in)) * 16;
    const int from_m = kW + (wm + in) * 32 + (half_of ^ (in >> 2 & 7)) * 4;
    const int from_x = (wn + in) * 128 + (half_of ^ R::spread(in)) * 16;
    auto read_w = [&](ROI_LDS uint8_t* src, int quarter, Half& f, int i) {
        f.w[i] = lds_read<i32x4>(src + i * 32 * 128 + (from_w ^ (32 * quarter)));
        f.m[i] = lds_read<int>(src + i * 32 * 32 + (from_m ^ (8 * quarter)));
    };
    auto read_x = [&](ROI_LDS uint8_t* src, int h, Half& f, int j) {
        const i32x4 lo = lds_read<i32x4>(src + j * 32 * 128 + (from_x ^ (64 * h)));
        const i32x4 hi = lds_read<i32x4>(src + j * 32 * 128 + (from_x ^ (64 * h) ^ 32));
        f.x[j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // the products of a half, beside the reads of quarter q of the two steps whose
    // weights are at ws, tokens at xs, and `load(i)`
    auto half = [&](const Half& f, ROI_LDS uint8_t* ws, ROI_LDS uint8_t* xs, int q, Half& next,
                    auto load) {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (i < kJ) read_x(xs, q & 1, next, i);
            read_w(ws, q, next, i);
            load(i);
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                acc[i][j] = __builtin_amdgcn_smfmac_i32_32x32x64_i8(f.w[i], f.x[j], acc[i][j],
                                                                    f.m[i], 0, 0);
            keep_order();
        }
    };
    const Scales<T> scales(a, piece);
    if (piece.count > 0) {
        ROI_LDS uint8_t *x0 = base, *x1 = base + kX, *x2 = base + (kRing - 1) * kX;
        ROI_LDS uint8_t *w0 = base + kRing * kX, *w1 = w0 + kPair; // of this pair of steps and the next
        constexpr int kXPart = R::kLoads / kI, kWPart = kPairLoads / kI;
        static_assert(R::kLoads % kI == 0 && kPairLoads % kI == 0, "loads are spread over the rows");
        auto none = [](int) {};
        Half lo, hi;
        stage_x(0, 0, R::kLoads, x0);
        stage_w(0, 0, kPairLoads, w0);
        stage_x(1, 0, R::kLoads, x1);
        if (kRing > 2) stage_x(2, 0, R::kLoads, x2);
        stage_w(2, 0, kPairLoads, w1);
        scales.keep(piece, base + packed_lds<T::kTile, kRing>());
        loads_barrier<(kRing - 1) * R::kLoads + kPairLoads>();
#pragma unroll
        for (int i = 0; i < kI; ++i) read_w(w0, 0, lo, i);
#pragma unroll
        for (int j = 0; j < kJ; ++j) read_x(x0, 0, lo, j);
        // past the end of the sum or of this part, loads are in bounds or zeros,
        // and unused
        for (int s = 0; s < piece.count; s += 2) {
            half(lo, w0, x0, 1, hi, none);
            // the next pair's weights are the last loads
            loads_barrier<(kRing - 2) * R::kLoads + kPairLoads>();
            half(hi, w0, x1, 2, lo, [&](int i) { stage_x(s + kRing, i * kXPart, kXPart, x0); });
            if (s + 1 == piece.count) break;
            half(lo, w0, x1, 3, hi, none);
            loads_barrier<(kRing - 2) * R::kLoads>();
            half(hi, w1, kRing == 2 ? x0 : x2, 0, lo, [&](int i) {
                if (i < kI / 2)
                    stage_x(s + 1 + kRing, i * 2 * kXPart, 2 * kXPart, x1);
                else
                    stage_w(s + 4, (i - kI / 2) * 2 * kWPart, 2 * kWPart, w0);
            });
            ROI_LDS uint8_t* const t = w0;
            w0 = w1;
            w1 = t;
            if (kRing > 2) {
                ROI_LDS uint8_t* const x = x2;
                x2 = x1;
                x1 = x0;
                x0 = x;
            }
        }
        loads_barrier();
    } else { // a sum over nothing
        scales.keep(piece, base + packed_lds<T::kTile, kRing>());
        __syncthreads();
    }
    write_tile<T, 32, Out>(a, piece, acc, base, base + packed_lds<T::kTile, kRing>());
}

// The sums of the tiles that were cut: one wave for a quad of results a lane.
template <typename T, int kBlock, typename Out>
__global__ __launch_bounds__(256) void linear_sum_kernel(LinearArgs a)
{
    using H = Held<T, kBlock>;
    constexpr int kTile = T::kTile;
    constexpr int kAll = H::kI * H::kJ * H::kQuads;
    const uint32_t id = scalar(blockIdx.x * 4 + threadIdx.x / 64);
    const int q = id % H::kQuads, i = id / H::kQuads % H::kI;
    const int j = id / (H::kQuads * H::kI) % H::kJ;
    const int wave = id / kAll % T::kWaves;
    const uint32_t tile = id / (kAll * T::kWaves);
    const Piece piece = tile_piece(a.grid, a.grid.full + tile);
    const int* from = a.partial + H::part_at((int64_t)tile * a.grid.splits, wave, i, j, q);
    const i32x4 sum = sum_of_parts<T, i32x4>(from, (int)a.grid.splits);
    const int r = piece.m * kTile + wave / T::kAcross * 16 * T::kI + 4 * H::quad(i, q);
    const int t = piece.n * kTile + wave % T::kAcross * 16 * T::kJ + H::column(j);
    if (r >= a.rows || t >= a.tokens) return;
    f32x4 ws, add;
    row_scales(a, r, ws, add);
    store4<Out>(a, t, r, finish4(sum, ws, add, a.xs[t]));
}

template <typename T, int kRing, int kPackedRing, typename Out>
void launch_tiles(const LinearArgs& a, hipStream_t stream)
{
    const dim3 grid(a.grid.blocks()), block(T::kThreads), sums(a.grid.rest() * T::kI * T::kJ * T::kWaves / 4);
    constexpr int kPackedLds = packed_lds<T::kTile, kPackedRing>() + Scales<T>::kBytes;
    if (a.meta) {
        hipLaunchKernelGGL((linear_packed_kernel<T, kPackedRing, Out>), grid, block, kPackedLds,
                           stream, a);
        if (sums.x > 0)
            hipLaunchKernelGGL((linear_sum_kernel<T, 32, Out>), sums, dim3(256), 0, stream, a);
    } else {
        hipLaunchKernelGGL((linear_tile_kernel<T, kRing, Out>), grid, block,
                           kRing * 2 * T::kTile * kRowBytes + Scales<T>::kBytes, stream, a);
        if (sums.x > 0)
            hipLaunchKernelGGL((linear_sum_kernel<T, 16, Out>), sums, dim3(256), 0, stream, a);
    }
}

template <int kWaves, int kRow, int kTokens, int kDepth, bool kPacked, typename Out>
int launch_few_as(LinearArgs a, hipStream_t stream)
{
    const int64_t tm = ((int64_t)a.rows + 16 * kRow - 1) / (16 * kRow);
    const int64_t tn = ((int64_t)a.tokens + kTokens - 1) / kTokens;
    a.grid.tm = (uint32_t)tm; // few tokens and fewer than 2^22 rows: a launch has room
    const dim3 grid((unsigned)(tm * tn)), block(64 * kWaves);
    if (a.cols % 16 == 0)
        hipLaunchKernelGGL((linear_few_kernel<kWaves, kRow, kTokens, kDepth, kPacked, true, Out>), grid,
                           block, 0, stream, a);
    else
        hipLaunchKernelGGL((linear_few_kernel<kWaves, kRow, kTokens, kDepth, false, false, Out>), grid,
                           block, 0, stream, a); // never 2:4: that has whole words
    return launch_status("roi_linear_i8");
}

template <bool kPacked, typename Out>
int launch_few(const LinearArgs& a, hipStream_t stream)
{
    // Blocks of 32 rows read the tokens half as often, those of 16 are twice as many:
    // 32 tokens through 3584 x 18944 take 20.5 us in blocks of 16 rows and 26.3 of
    // 32, through 4864 x 4864 (more than a block a compute unit) 9.9 and 8.6.
    if (a.tokens > 16) {
        const int64_t blocks = (int64_t)((a.rows + 15) / 16) * ((a.tokens + 31) / 32);
        return blocks <= kUnits ? launch_few_as<4, 1, 32, 2, kPacked, Out>(a, stream)
                                : launch_few_as<4, 2, 32, 2, kPacked, Out>(a, stream);
    }
    // With at least two blocks a compute unit a shallow ring lets more of them
    // run at once: one token through 18944 x 3584 at 2:4 takes 11.2 us with two
    // slots and 13.8 with three, through 3584 x 18944 13.2 and 10.5.
    const bool many = a.rows >= 16 * 512;
    if (a.tokens > 8)
        return many ? launch_few_as<4, 1, 16, 2, kPacked, Out>(a, stream)
                    : launch_few_as<4, 1, 16, 3, kPacked, Out>(a, stream);
    return many ? launch_few_as<4, 1, 8, 2, kPacked, Out>(a, stream)
                : launch_few_as<4, 1, 8, 3, kPacked, Out>(a, stream);
}

int check_fits(const LinearPlan& plan)
{
    return plan.few || plan.cut.fits ? ROI_OK
                                     : fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
}

template <typename Out>
int launch(LinearArgs a, const LinearPlan& plan, void* workspace, hipStream_t stream)
{
    if (plan.few)
        return a.meta ? launch_few<true, Out>(a, stream) : launch_few<false, Out>(a, stream);
    if (int st = check_fits(plan)) return st;
    const Cut& c = plan.cut;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    if (plan.x_bytes) {
        uint8_t* const x = at;
        uint8_t* const w = x + plan.x_bytes;
        launch_copy_rows(RowsCopy{a.x, x, a.tokens, a.cols, plan.row},
                         RowsCopy{a.w, w, a.rows, a.cols, plan.row}, stream);
        a.x = reinterpret_cast<int8_t*>(x);
        a.w = reinterpret_cast<int8_t*>(w);
        at = w + plan.w_bytes;
        a.cols = (int)plan.row;
    }
    a.partial = reinterpret_cast<int*>(at);
    a.grid = grid_of(c);
    if (c.tile == 256)
        launch_tiles<Tile<256>, 2, 2, Out>(a, stream);
    else if (a.grid.blocks() <= kUnits)
        launch_tiles<Tile<128, 8>, 4, 3, Out>(a, stream);
    else
        launch_tiles<Tile<128>, 2, 2, Out>(a, stream);
    return launch_status("roi_linear_i8");
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_i8_workspace(int64_t tokens, int64_t rows, int64_t cols, int packed)
{
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    if (int st = check_linear_sum(cols, packed != 0)) return st;
    const LinearPlan plan = plan_linear(tokens, rows, cols, packed != 0);
    if (int st = check_fits(plan)) return st;
    ok();
    return plan.few ? 0 : plan.bytes;
}

extern "C" int roi_linear_i8(const int8_t* xq, const float* xs, const int8_t* wq,
                             const uint32_t* meta, const float* ws, const uint16_t* bias,
                             int64_t tokens, int64_t rows, int64_t cols, void* y, int dtype,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const LinearPlan plan = plan_linear(tokens, rows, cols, meta != nullptr);
    if (int st = validate_linear_i8(xq, xs, wq, meta, ws, bias, tokens, rows, cols, y, dtype,
                                    workspace, workspace_bytes, plan.few ? 0 : plan.bytes, &todo))
        return st;
    if (!todo) return ok();
    const LinearArgs a{xq, xs, wq, meta, ws, bias, y, nullptr, (int)tokens,
                       (int)rows, (int)cols, {}};
    return dtype == ROI_BF16 ? launch<uint16_t>(a, plan, workspace, stream)
                             : launch<float>(a, plan, workspace, stream);
}
