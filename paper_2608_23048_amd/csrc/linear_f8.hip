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
    int scales;     // bytes of a row of scales
    int w_shift;    // a row r of the weight has scales row r >> w_shift
    float* partial; // fp32 parts of tiles (Held::part_at)
    Grid grid;      // tiles along the rows and the tokens (few tokens: grid.tm alone)
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

// The bytes of a 16-byte piece of a row that lie before the row's end, `n` (1 .. 15)
// of them; the others become zeros.
__device__ __forceinline__ void cut_piece(ROI_LDS uint8_t* p, int n)
{
    u32x4 v = *reinterpret_cast<ROI_LDS u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int have = n - 4 * i;
        v[i] = have >= 4 ? v[i] : have <= 0 ? 0u : v[i] & (0xFFFFFFFFu >> (32 - 8 * have));
    }
    *reinterpret_cast<ROI_LDS u32x4*>(p) = v;
}

__device__ __forceinline__ i32x8 joined(i32x4 lo, i32x4 hi)
{
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Waits for all LDS reads, known to the compiler: reads that are on their way at only
// one of a loop's entries would have it wait for all in every turn.
__device__ __forceinline__ void lds_reads_wait() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// ---------------------------------------------------------------- few tokens
// A block owns 16 kRow weight rows and up to kTokens tokens (8, or a multiple of
// 16); its waves share out the sum by steps of 128 values and add up their parts in
// LDS.  The weight is read once for each kTokens: bound by its bytes (16 tokens through
// 3584 x 18944 take 12.2 us, 5.6 TB/s, the matrix cores busy for 5 % of it).  A wave
// brings its steps to a ring of kDepth slots in LDS of its own and needs no barrier.
// Step s of the sum goes to wave s % 4, so that a wave's scales are one byte of
// consecutive words.
template <int kRow, int kTokens, int kDepth, int kFormat>
__global__ __launch_bounds__(256) void linear_f8_few_kernel(LinearF8Args a)
{
    constexpr int kWaves = 4;
    constexpr int kTok = (kTokens + 15) / 16;
    constexpr int kW = kRow * 2048, kX = kTokens * 128;
    constexpr int kSlot = kW + kX + 256; // the operands and a word of scales for each row
    constexpr int kLoads = 2 * kRow + kTokens / 8 + 1;
    static_assert(16 * kRow + kTokens <= 64, "a lane for each row");
    static_assert(kRow * kTok * 1024 <= kDepth * kSlot, "the parts of the sum take the ring's place");
    __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves][kDepth * kSlot];
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = scalar(threadIdx.x >> 6);
    ROI_LDS uint8_t* ring = (ROI_LDS uint8_t*)&lds[0][0] + wave * (kDepth * kSlot);
    const int r0 = scalar(blockIdx.x % a.grid.tm) * (16 * kRow);
    const int t0 = scalar(blockIdx.x / a.grid.tm) * kTokens;

    // a load brings 128 bytes of eight rows: this lane's of the eight, and its chunk
    // of a row (kept at the place of k-rows, mm.hpp)
    const int row = lane / 8, chunk = (lane % 8) ^ row;
    const int w_stride = (int)a.w_stride, x_stride = (int)a.x_stride;
    const uint8_t* wbase = a.w + (int64_t)r0 * w_stride;
    const uint8_t* xbase = a.x + (int64_t)t0 * x_stride;
    // this lane's row of scales
    const bool of_w = lane < 16 * kRow;
    const uint8_t* scales =
        of_w ? a.ws + (int64_t)(least(r0 + lane, a.rows - 1) >> a.w_shift) * a.scales
             : a.xs + (int64_t)least(t0 + (lane - 16 * kRow) % kTokens, a.tokens - 1) * a.scales;
    const int words = a.scales / 4;
    // the wave's step n into a slot (past the sum's end: zeros)
    auto stage = [&](int n, ROI_LDS uint8_t* slot) {
        const int k = (wave + n * kWaves) * 128;
        auto bring = [&](const uint8_t* base, int first, int rows, int stride, ROI_LDS uint8_t* dst) {
            const bool live = first + row < rows && k + 16 * chunk < a.cols;
            load_to_lds<false>(buffer_at(base + k),
                               live ? (uint32_t)row * stride + 16 * chunk : kNowhere, first * stride,
                               dst);
        };
#pragma unroll
        for (int i = 0; i < 2 * kRow; ++i) bring(wbase, 8 * i, a.rows - r0, w_stride, slot + i * 1024);
#pragma unroll
        for (int i = 0; i < kTokens / 8; ++i)
            bring(xbase, 8 * i, a.tokens - t0, x_stride, slot + kW + i * 1024);
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(scales + 4 * least(n, words - 1)),
            (ROI_LDS void*)(slot + kW + kX), 4, 0, 0);
    };
    f32x4 acc[kRow][kTok] = {};
    const int from = (lane & 15) * 128 + (g ^ (lane & 7)) * 16;
    // of eight tokens, the second eight lanes read the first's again
    const int from_x = (lane & (kTokens < 16 ? 7 : 15)) * 128 + (g ^ (lane & 7)) * 16;
    auto multiply = [&](ROI_LDS uint8_t* slot) {
        i32x8 w[kRow], x[kTok];
        int ws[kRow], xs[kTok];
#pragma unroll
        for (int i = 0; i < kRow; ++i) {
            w[i] = joined(lds_read<i32x4>(slot + i * 2048 + from), lds_read<i32x4>(slot + i * 2048 + (from ^ 64)));
            ws[i] = lds_read<int>(slot + kW + kX + (16 * i + (lane & 15)) * 4) >> (8 * wave);
        }
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            ROI_LDS uint8_t* p = slot + kW + j * 2048;
            x[j] = joined(lds_read<i32x4>(p + from_x), lds_read<i32x4>(p + (from_x ^ 64)));
            xs[j] = lds_read<int>(slot + kW + kX + (16 * (kRow + j) + (lane & (kTokens < 16 ? 7 : 15))) * 4) >>
                    (8 * wave);
        }
#pragma unroll
        for (int i = 0; i < kRow; ++i)
#pragma unroll
            for (int j = 0; j < kTok; ++j)
                acc[i][j] = multiply_block<kFormat>(w[i], x[j], acc[i][j], ws[i], xs[j]);
    };
    const int steps = (a.cols + 127) / 128;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    const int tail = a.cols % 16;
    if (mine > 0) {
        int slot = 0;
#pragma unroll
        for (int n = 0; n < kDepth; ++n) stage(n, ring + n * kSlot);
        for (int n = 0; n < mine; ++n) {
            loads_wait<(kDepth - 1) * kLoads>();
            if (tail && wave + n * kWaves == steps - 1 && lane < 16 * kRow + kTokens) {
                const int last = a.cols % 128 / 16; // the chunk that the rows end in
                cut_piece(ring + slot + lane * 128 + (last ^ (lane & 7)) * 16, tail);
            }
            multiply(ring + slot);
            // the slot is read: its values are in registers before its next loads
            keep_order();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            stage(n + kDepth, ring + slot);
            slot = slot + kSlot < kDepth * kSlot ? slot + kSlot : 0;
        }
        loads_wait<0>();
    }
#pragma unroll
    for (int i = 0; i < kRow; ++i)
#pragma unroll
        for (int j = 0; j < kTok; ++j)
            *reinterpret_cast<ROI_LDS f32x4*>(ring + ((i * kTok + j) * 64 + lane) * 16) = acc[i][j];
    __syncthreads();
    for (int b = wave; b < kRow * kTok; b += kWaves) {
        const int in = 16 * (b % kTok) + (lane & 15);
        const int t = t0 + in, r = r0 + 16 * (b / kTok) + 4 * g;
        if (in >= kTokens || t >= a.tokens || r >= a.rows) continue;
        f32x4 sum = {};
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
            sum += lds_read<f32x4>((ROI_LDS uint8_t*)&lds[0][0] + v * (kDepth * kSlot) +
                                   (b * 64 + lane) * 16);
        finish_f8(a, t, r, sum);
    }
}

// --------------------------------------------------------------- many tokens
// A block makes one tile (mm.hpp) over steps of 128 values, in kRing LDS buffers of
// both operands.  A wave holds its tokens' operands of a step (kJ blocks of 16) and
// passes the weight's rows (kI) by in pairs, the next pair read ahead.  In the last
// pair a block of tokens is read again, for the next step, as soon as both its
// products are under way.  One barrier a step, ahead of that pair: past it every wave
// holds all it needs of this step's buffer, which takes the step kRing later, and the
// next step's, loading for kRing - 1 steps, is complete.  The scales of four steps
// are a word a row, which comes beside the operands.
//
// A block goes through its tiles without a pause: the loads run kRing steps ahead
// of the products, past a tile's end into the next one.
//
// A 256-tile of four waves reads each operand's byte of LDS twice a step, and a wave's
// 256 sums a lane leave room for the operands a step ahead; with eight waves of 128 x 64
// LDS is read half as much again (the product below: 529 us, with four waves 491, and
// without a pause between tiles 437).  128-tiles share a compute unit two by two, or have
// eight waves and four buffers where each has one to itself.  8192 tokens through
// 18944 x 3584 take 424 to 462 us, as the clock has it (2.4 to 2.6 PFLOP/s; the matrix
// cores are busy for 65 % of the time at 2.05 GHz): bound by their issue and their power.

// Rows of an operand that a thread brings to LDS, where place j ^ (row & 7) of a row
// holds its chunk j.  What lies behind the last of the operand's bytes is left out
// by the buffer's size (the offsets of the lane and of the wave count) and becomes
// zeros; what lies behind a row's values, but before that, comes along.
template <typename T>
struct F8Rows {
    static constexpr int kThreads = T::kThreads;
    static constexpr int kLoads = T::kTile * kRowBytes / (16 * kThreads);
    // a tile's rows: the first one and the bytes of all (0: none)
    struct At {
        const uint8_t* base;
        int size;
    };
    int stride;
    uint32_t at; // byte offset of load 0 from the first row; those of load i are i kThreads / 8 rows on

    __device__ __forceinline__ explicit F8Rows(int64_t stride_) : stride((int)stride_)
    {
        const int row = threadIdx.x / 8;
        at = (uint32_t)row * (uint32_t)stride_ + 16 * ((threadIdx.x % 8) ^ (row & 7));
    }
    __device__ __forceinline__ At rows(const uint8_t* p, int row0, int n, int len) const
    {
        return At{p + (int64_t)row0 * stride, (least(n - row0, T::kTile) - 1) * stride + (len + 15) / 16 * 16};
    }
    // The buffer of values k .. of the rows.
    __device__ __forceinline__ static __amdgpu_buffer_rsrc_t buffer(const At& t, int k)
    {
        const int left = t.size - k;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(t.base + k), 0, left > 0 ? left : 0,
                                                 0x00020000);
    }
    __device__ __forceinline__ void stage(__amdgpu_buffer_rsrc_t from, int i, ROI_LDS uint8_t* dst) const
    {
        load_to_lds<false>(from, at, i * (kThreads / 8) * stride,
                           dst + (i * kThreads + scalar(threadIdx.x >> 6) * 64) * 16);
    }
};

// A tile's results from a wave's sums, which become zeros: a part of a cut tile as it
// is, else 16 tokens at a time through the wave's `mine` of LDS to y.
template <typename T>
__device__ __forceinline__ void write_f8_tile(const LinearF8Args& a, const Piece& piece,
                                              f32x4 (&acc)[T::kI][T::kJ], ROI_LDS uint8_t* mine)
{
    using H = Held<T, 16>;
    const int wave = scalar(threadIdx.x >> 6);
    const int r0 = piece.m * T::kTile + wave / T::kAcross * 16 * T::kI;
    const int t0 = piece.n * T::kTile + wave % T::kAcross * 16 * T::kJ;
    if (piece.part >= 0) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i)
#pragma unroll
            for (int j = 0; j < T::kJ; ++j) {
                *reinterpret_cast<f32x4*>(a.partial + H::part_at(piece.part, wave, i, j, 0)) = acc[i][j];
                acc[i][j] = f32x4{};
                keep_order();
            }
        return;
    }
    f32x4 add[T::kI]; // without a bias -0, which changes nothing
#pragma unroll
    for (int i = 0; i < T::kI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            add[i][e] = a.bias ? bf16_bits_to_float(a.bias[least(r0 + 4 * H::quad(i, 0) + e, a.rows - 1)]) : -0.0f;
    using Lines = RowsOut<T::kI, 8>; // of a token: 16 kI values of 2 bytes
#pragma unroll
    for (int j = 0; j < T::kJ; ++j) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i) {
            const f32x4 v = acc[i][j] + add[i];
            *reinterpret_cast<ROI_LDS u32x2*>(Lines::at(mine, threadIdx.x % 16, H::quad(i, 0))) =
                u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
            acc[i][j] = f32x4{};
        }
        keep_order();
#pragma unroll
        for (int n = 0; n < 16 / Lines::kAtOnce; ++n) {
            int row, chunk;
            const Quad v = Lines::get(mine, n, row, chunk);
            const int t = t0 + 16 * j + row;
            if (t < a.tokens) store_chunk(a.y + (int64_t)t * a.rows, r0 + chunk * 8, a.rows, v);
        }
        keep_order();
    }
}

// Two operands a step, a word of scales for each of their rows, and 16 tokens of a
// wave's results.
template <typename T, int kRing>
constexpr int f8_lds()
{
    return kRing * 2 * T::kTile * (kRowBytes + 4) + T::kWaves * 16 * T::kI * 32;
}
// Blocks of a compute unit.
template <typename T>
constexpr int f8_blocks() { return T::kWaves == 4 && T::kTile == 128 ? 2 : 1; }

template <typename T, int kRing, int kFormat>
__global__ __launch_bounds__(T::kThreads, f8_blocks<T>() * T::kWaves / 4) void linear_f8_tile_kernel(
    LinearF8Args a)
{
    constexpr int kTile = T::kTile, kTileBytes = kTile * kRowBytes;
    constexpr int kI = T::kI, kJ = T::kJ;
    static_assert(kRing == 2 || kRing == 4, "slots are counted in bits");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    ROI_LDS uint8_t* scale_lds = base + kRing * 2 * kTileBytes;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = scalar(threadIdx.x >> 6);
    ROI_LDS uint8_t* mine = scale_lds + kRing * 2 * kTile * 4 + wave * (16 * kI * 32);
    const int wm = wave / T::kAcross * 16 * kI, wn = wave % T::kAcross * 16 * kJ;
    const uint32_t pieces = a.grid.blocks();

    using R = F8Rows<T>;
    const R wrows(a.w_stride), xrows(a.x_stride);
    constexpr int kLoads = R::kLoads;
    // Words of scales: kTile of the weight's rows, then kTile of the tokens'.  With a
    // thread for each row a load for each operand, else one for both, waves being of
    // one operand, and those without any bringing the first's again.
    constexpr bool kApart = T::kThreads == kTile;
    constexpr int kScaleLoads = kApart ? 2 : 1;
    const int scale_first = kApart ? wave * 64 : wave * 64 % (2 * kTile);
    const bool scale_of_w = kApart || scale_first < kTile;
    // What is loaded next: step S of the sum, `left` steps from the end of its piece.
    struct Aim {
        typename R::At w, x;
        const uint8_t* scales;   // of this wave's operand (kApart: the weight's)
        const uint8_t* x_scales; // kApart
        uint32_t scale_at, x_scale_at;
        int scale_size; // 0 behind the last piece
        int S, left;
        uint32_t index;
    };
    auto aim_at = [&](Aim& m, uint32_t index) {
        m.index = index;
        if (index >= pieces) {
            m.w.size = m.x.size = m.scale_size = 0;
            m.left = 0x7FFFFFFF;
            return;
        }
        const Piece p = piece_of(a.grid, index);
        const int r0 = p.m * kTile, t0 = p.n * kTile;
        m.w = wrows.rows(a.w, r0, a.rows, a.cols);
        m.x = xrows.rows(a.x, t0, a.tokens, a.cols);
        // place p of an operand's words is that of row 16 (p % k) + p / k of a wave's 16 k
        // rows, so that a lane's k words are consecutive
        auto row_of = [](int p, int k) { return p / (16 * k) * (16 * k) + p % k * 16 + p % (16 * k) / k; };
        const int place = (scale_first + lane) % kTile;
        const int at_w = row_of(place, kI), at_x = row_of(place, kJ);
        const uint8_t* of_w = a.ws + (int64_t)(r0 >> a.w_shift) * a.scales;
        const uint8_t* of_x = a.xs + (int64_t)t0 * a.scales;
        const uint32_t w_row = (uint32_t)((least(r0 + at_w, a.rows - 1) >> a.w_shift) - (r0 >> a.w_shift));
        const uint32_t x_row = (uint32_t)least(at_x, a.tokens - 1 - t0);
        m.scales = scale_of_w ? of_w : of_x;
        m.scale_at = (uint32_t)a.scales * (scale_of_w ? w_row : x_row);
        m.x_scales = of_x;
        m.x_scale_at = (uint32_t)a.scales * x_row;
        m.scale_size = 0x7FFFFFFF;
        m.S = p.first;
        m.left = p.count;
    };
    auto move_on = [&](Aim& m) {
        if (--m.left == 0)
            aim_at(m, m.index + gridDim.x);
        else
            ++m.S;
    };
    // n counts the block's steps over all its pieces
    auto buffer = [&](int n) { return base + (n & (kRing - 1)) * 2 * kTileBytes; };
    auto words = [&](int n) { return scale_lds + (n & (kRing - 1)) * 2 * kTile * 4; };
    auto stage_scales = [&](const Aim& m, int n) {
        auto bring = [&](const uint8_t* p, uint32_t at, int first) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, m.scale_size, 0x00020000),
                (ROI_LDS void*)(words(n) + first * 4), 4, (int)at, m.S & ~3, 0, 0);
        };
        bring(m.scales, m.scale_at, scale_first);
        if (kApart) bring(m.x_scales, m.x_scale_at, kTile + scale_first);
    };
    const int from_w = (wm + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
    const int from_x = kTileBytes + (wn + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
    auto read_w = [&](int n, int i) {
        ROI_LDS uint8_t* p = buffer(n) + i * 16 * kRowBytes;
        return joined(lds_read<i32x4>(p + from_w), lds_read<i32x4>(p + (from_w ^ 64)));
    };
    auto read_x = [&](int n, int j) {
        ROI_LDS uint8_t* p = buffer(n) + j * 16 * kRowBytes;
        return joined(lds_read<i32x4>(p + from_x), lds_read<i32x4>(p + (from_x ^ 64)));
    };
    // the words of step n, kI of the weight's and kJ of the tokens' a lane
    static_assert(kI % 4 == 0 && (kJ == 2 || kJ % 4 == 0), "vectors of words");
    auto read_words = [&](int n, int (&w_words)[kI], int (&x_words)[kJ]) {
        ROI_LDS uint8_t* p = words(n) + (wm + (lane & 15) * kI) * 4;
#pragma unroll
        for (int i = 0; i < kI; i += 4) {
            const i32x4 v = lds_read<i32x4>(p + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) w_words[i + e] = v[e];
        }
        p = words(n) + (kTile + wn + (lane & 15) * kJ) * 4;
        if constexpr (kJ == 2) {
            const i32x2 v = lds_read<i32x2>(p);
            x_words[0] = v[0];
            x_words[1] = v[1];
        } else {
#pragma unroll
            for (int j = 0; j < kJ; j += 4) {
                const i32x4 v = lds_read<i32x4>(p + 4 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) x_words[j + e] = v[e];
            }
        }
    };

    f32x4 acc[kI][kJ] = {};
    int ws[kI], xs[kJ];
    i32x8 w[4], x[kJ];
    constexpr int kPairs = kI / 2, kInPair = 2 * kJ;
    static_assert(kPairs == 2 || kPairs == 4, "where the loads go");
    // The products of rows 2 p and 2 p + 1, `beside(m)` after the m-th of them.
    auto pair = [&](int p, auto beside) {
#pragma unroll
        for (int m = 0; m < kInPair; ++m) {
            const int i = 2 * p + m % 2, j = m / 2;
            acc[i][j] = multiply_block<kFormat>(w[i % 4], x[j], acc[i][j], ws[i], xs[j]);
            keep_order();
            beside(m);
            keep_order();
        }
    };
    // Number of the load that goes beside product m when `count` go beside a pair's, or -1.
    constexpr auto load_beside = [](int m, int count) {
        return m % (kInPair / count) == 0 ? m / (kInPair / count) : -1;
    };
    // Step n, the loads of step n + kRing as `next` says, and those of the weight that
    // step n - 1 has left from `last`, step last_S.  `after`: step n + 1 of the sum.
    // The loads are spread over the step: more at a time than the vector memory takes
    // in holds up the wave and its products.  With four pairs the tokens are read, and
    // their buffer free, past the first.  No branches: the compiler moves products past
    // those further on.
    auto step = [&](int n, const typename R::At& last, int last_S, const Aim& next, int after) {
        constexpr bool kLong = kPairs == 4;
        constexpr int kBeside = kLong ? kLoads / 2 : kLoads;
        __amdgpu_buffer_rsrc_t last_w, next_w, next_x;
#pragma unroll
        for (int p = 0; p < kPairs - 1; ++p) {
            pair(p, [&](int m) {
                if (m < 2) w[(2 * p + 2 + m) % 4] = read_w(n, 2 * p + 2 + m);
                if (m == 0 && p == 0) last_w = R::buffer(last, last_S * kRowBytes);
                if (m == 0 && p == 1) next_x = R::buffer(next.x, next.S * kRowBytes);
                const int l = load_beside(m, kBeside);
                if (l < 0) return;
                if (p == 0)
                    wrows.stage(last_w, kLoads - kBeside + l, buffer(n - 1));
                else
                    xrows.stage(next_x, (p - 1) * kBeside + l, buffer(n) + kTileBytes);
            });
            if (kLong && p == 0) {
                asm volatile("s_barrier" ::: "memory");
                keep_order();
            }
        }
        loads_barrier<(kRing - 2) * (2 * kLoads + kScaleLoads) + (kLong ? kLoads : 0)>();
        keep_order();
        int next_ws[kI], next_xs[kJ], shift = 0;
        pair(kPairs - 1, [&](int m) {
            constexpr int kHalf = kInPair / 2;
            if (m < 2) w[m] = read_w(n + 1, m);
            if (m == 0) read_words(n + 1, next_ws, next_xs);
            if (m == 0 && kLong) next_w = R::buffer(next.w, next.S * kRowBytes);
            if (m == 0 && !kLong) next_x = R::buffer(next.x, next.S * kRowBytes);
            if (m == kHalf - 1) shift = (after & 3) * 8;
            if (m >= kHalf) {
                xs[m - kHalf] = next_xs[m - kHalf] >> shift;
#pragma unroll
                for (int i = (m - kHalf) * kI / kHalf; i < (m + 1 - kHalf) * kI / kHalf; ++i)
                    if (i < kI - 2) ws[i] = next_ws[i] >> shift;
            }
            if (m % 2) x[m / 2] = read_x(n + 1, m / 2);
            const int l = load_beside(m, kBeside);
            if (l < 0) return;
            if (kLong)
                wrows.stage(next_w, l, buffer(n));
            else
                xrows.stage(next_x, l, buffer(n) + kTileBytes);
        });
        ws[kI - 2] = next_ws[kI - 2] >> shift;
        ws[kI - 1] = next_ws[kI - 1] >> shift;
        stage_scales(next, n);
    };

    Aim next;
    aim_at(next, blockIdx.x);
    Piece piece = piece_of(a.grid, blockIdx.x);
#pragma unroll
    for (int n = 0; n < kRing; ++n) {
        if (n > 0) move_on(next);
        const __amdgpu_buffer_rsrc_t wb = R::buffer(next.w, next.S * kRowBytes);
        const __amdgpu_buffer_rsrc_t xb = R::buffer(next.x, next.S * kRowBytes);
        stage_scales(next, n);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) xrows.stage(xb, i, buffer(n) + kTileBytes);
        // the last one's weight is loaded beside the first products
        const int count = n < kRing - 1 ? kLoads : kPairs == 4 ? kLoads / 2 : 0;
#pragma unroll
        for (int i = 0; i < count; ++i) wrows.stage(wb, i, buffer(n));
    }
    // the steps behind the first go on loading
    loads_barrier<(kRing - 1) * (kScaleLoads + 2 * kLoads) - (kPairs == 4 ? kLoads / 2 : kLoads)>();
    auto first_operands = [&](int n) {
        w[0] = read_w(n, 0);
        w[1] = read_w(n, 1);
#pragma unroll
        for (int j = 0; j < kJ; ++j) x[j] = read_x(n, j);
    };
    first_operands(0);
    read_words(0, ws, xs);
#pragma unroll
    for (int i = 0; i < kI; ++i) ws[i] >>= (piece.first & 3) * 8;
#pragma unroll
    for (int j = 0; j < kJ; ++j) xs[j] >>= (piece.first & 3) * 8;
    lds_reads_wait();
    const int ragged = a.cols % 128;
    int n = 0;
    for (uint32_t index = blockIdx.x;;) {
        index += gridDim.x;
        const Piece after = index < pieces ? piece_of(a.grid, index) : Piece{};
        // `run` steps go on alike: to the end of this piece or of the loads', or to a
        // ragged step, by themselves
        int s = 0, run = 0;
        for (; s < piece.count; ++s, ++n, --run) {
            const typename R::At last = next.w;
            const int last_S = next.S;
            ++next.S;
            --next.left;
            if (run == 0) {
                if (next.left == 0) aim_at(next, next.index + gridDim.x);
                run = least(piece.count - s, next.left);
                const int to_ragged = a.grid.steps - 1 - piece.first - s;
                if (ragged && to_ragged > 0) run = least(run, to_ragged);
                if (ragged && to_ragged == 0) {
                    // zeros behind the rows' ends, and once more what has been read
                    for (int at = threadIdx.x; at < 2 * kTile; at += T::kThreads) {
                        ROI_LDS uint8_t* row = buffer(n) + at * kRowBytes;
                        int c = ragged / 16;
                        if (ragged % 16) {
                            cut_piece(row + (c ^ (at & 7)) * 16, ragged % 16);
                            ++c;
                        }
                        for (; c < 8; ++c) *reinterpret_cast<ROI_LDS u32x4*>(row + (c ^ (at & 7)) * 16) = u32x4{};
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    first_operands(n);
                    lds_reads_wait();
                }
            }
            step(n, last, last_S, next, s + 1 < piece.count ? piece.first + s + 1 : after.first);
        }
        write_f8_tile<T>(a, piece, acc, mine);
        if (index >= pieces) break;
        piece = after;
    }
    loads_wait<0>(); // the loads behind the last piece, into this block's LDS
}

// The sums of the tiles that were cut: one wave for a quad of results a lane.
template <typename T>
__global__ __launch_bounds__(256) void linear_f8_sum_kernel(LinearF8Args a)
{
    using H = Held<T, 16>;
    constexpr int kAll = T::kI * T::kJ;
    const uint32_t id = scalar(blockIdx.x * 4 + threadIdx.x / 64);
    const int i = id % T::kI, j = id / T::kI % T::kJ;
    const int wave = id / kAll % T::kWaves;
    const uint32_t tile = id / (kAll * T::kWaves);
    const Piece piece = tile_piece(a.grid, a.grid.full + tile);
    const float* from = a.partial + H::part_at((int64_t)tile * a.grid.splits, wave, i, j, 0);
    const f32x4 sum = sum_of_parts<T, f32x4>(from, (int)a.grid.splits);
    const int r = piece.m * T::kTile + wave / T::kAcross * 16 * T::kI + 4 * H::quad(i, 0);
    const int t = piece.n * T::kTile + wave % T::kAcross * 16 * T::kJ + H::column(j);
    if (r < a.rows && t < a.tokens) finish_f8(a, t, r, sum);
}

template <typename T, int kRing, int kFormat>
void launch_f8_tiles(const LinearF8Args& a, hipStream_t stream)
{
    const uint32_t most = (uint32_t)(f8_blocks<T>() * kUnits), blocks = a.grid.blocks();
    const dim3 grid(blocks < most ? blocks : most), sums(a.grid.rest() * T::kI * T::kJ * T::kWaves / 4);
    hipLaunchKernelGGL((linear_f8_tile_kernel<T, kRing, kFormat>), grid, dim3(T::kThreads),
                       (f8_lds<T, kRing>()), stream, a);
    if (sums.x > 0) hipLaunchKernelGGL((linear_f8_sum_kernel<T>), sums, dim3(256), 0, stream, a);
}

template <int kRow, int kTokens, int kDepth, int kFormat>
void launch_f8_few_as(LinearF8Args a, hipStream_t stream)
{
    const int64_t tm = ((int64_t)a.rows + 16 * kRow - 1) / (16 * kRow);
    const int64_t tn = ((int64_t)a.tokens + kTokens - 1) / kTokens;
    a.grid.tm = (uint32_t)tm;
    hipLaunchKernelGGL((linear_f8_few_kernel<kRow, kTokens, kDepth, kFormat>), dim3((unsigned)(tm * tn)),
                       dim3(256), 0, stream, a);
}

template <int kFormat>
void launch_f8_few(const LinearF8Args& a, hipStream_t stream)
{
    if (a.tokens > 16) {
        const int64_t blocks = (int64_t)((a.rows + 15) / 16) * ((a.tokens + 31) / 32);
        return blocks <= kUnits ? launch_f8_few_as<1, 32, 2, kFormat>(a, stream)
                                : launch_f8_few_as<2, 32, 2, kFormat>(a, stream);
    }
    const bool many = a.rows >= 16 * 512;
    if (a.tokens > 8)
        return many ? launch_f8_few_as<1, 16, 2, kFormat>(a, stream)
                    : launch_f8_few_as<1, 16, 3, kFormat>(a, stream);
    return many ? launch_f8_few_as<1, 8, 2, kFormat>(a, stream)
                : launch_f8_few_as<1, 8, 3, kFormat>(a, stream);
}

template <int kFormat>
void launch_f8(LinearF8Args a, const LinearPlan& plan, void* workspace, hipStream_t stream)
{
    if (plan.few) return launch_f8_few<kFormat>(a, stream);
    a.partial = static_cast<float*>(workspace);
    a.grid = grid_of(plan.cut);
    if (plan.cut.tile == 256)
        launch_f8_tiles<Tile<256, 4>, 2, kFormat>(a, stream);
    else if (a.grid.blocks() <= kUnits)
        launch_f8_tiles<Tile<128, 8>, 4, kFormat>(a, stream);
    else
        launch_f8_tiles<Tile<128>, 2, kFormat>(a, stream);
}

int check_f8_fits(const LinearPlan& plan)
{
    return plan.cut.fits ? ROI_OK : fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int64_t roi_linear_f8_workspace(int64_t tokens, int64_t rows, int64_t cols)
{
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const LinearPlan plan = plan_linear_f8(tokens, rows, cols);
    if (int st = check_f8_fits(plan)) return st;
    ok();
    return plan.bytes;
}

extern "C" int roi_linear_f8(const uint8_t* xq, int64_t x_stride, const uint8_t* xs, int x_format,
                             const uint8_t* wq, int64_t w_stride, const uint8_t* ws, int w_square,
                             const uint16_t* bias, int64_t tokens, int64_t rows, int64_t cols,
                             uint16_t* y, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream)
{
    bool todo;
    if (int st = check_linear_sizes(tokens, rows, cols)) return st;
    const LinearPlan plan = plan_linear_f8(tokens, rows, cols);
    if (int st = validate_linear_f8(xq, x_stride, xs, x_format, wq, w_stride, ws, w_square != 0, bias,
                                    tokens, rows, cols, y, workspace, workspace_bytes, plan.bytes,
                                    &todo))
        return st;
    if (!todo) return ok();
    if (int st = check_f8_fits(plan)) return st;
    const LinearF8Args a{xq, xs, wq, ws, bias, y, x_stride, w_stride, (int)tokens, (int)rows, (int)cols,
                         (int)roi_block_scales(cols), w_square ? 7 : 0, nullptr, {}};
    if (x_format == ROI_E4M3)
        launch_f8<ROI_E4M3>(a, plan, workspace, stream);
    else
        launch_f8<ROI_E5M2>(a, plan, workspace, stream);
    return launch_status("roi_linear_f8");
}
