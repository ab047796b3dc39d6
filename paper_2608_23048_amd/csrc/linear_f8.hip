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

// ---------------------------------------------------------------- few tokens
// A block owns 16 kRow weight rows and up to kTokens tokens (8, or a multiple of
// 16); its waves share out the sum by steps of 128 values and add up their parts in
// LDS.  The weight is read once: bound by its bytes.  A wave brings its steps to a
// ring of kDepth slots in LDS of its own and needs no barrier.  Step s of the sum
// goes to wave s % 4, so that a wave's scales are one byte of consecutive words.
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
// A block makes one tile (mm.hpp) over steps of 128 values, with kRing LDS buffers of
// each operand.  A wave holds its tokens' operands of a step (kJ blocks of 16) and
// passes the weight's rows (kI) by, two rows read ahead; beside them it reads the
// next step's tokens.  One barrier a step, ahead of the last two rows: past it every
// wave holds all it needs of this step's weight and the next step's tokens, whose
// buffers take the loads kRing steps on, and the next step's weight and the tokens
// behind it, loading for kRing - 1 steps, are complete.  The scales of four steps
// are a word a row, which comes beside the operands four steps ahead.

// Rows row0 .. of an operand that this thread brings to LDS, where place j ^ (row & 7)
// of a row holds its chunk j.
template <typename T>
struct F8Rows {
    static constexpr int kThreads = T::kThreads;
    static constexpr int kLoads = T::kTile * kRowBytes / (16 * kThreads);
    const uint8_t* base;
    int left, len, stride; // rows from row0 on, their values and the bytes between them
    uint32_t at;           // byte offset of load 0 from base

    __device__ __forceinline__ F8Rows(const uint8_t* p, int row0, int n, int len_, int64_t stride_)
        : base(p + (int64_t)row0 * stride_), left(n - row0), len(len_), stride((int)stride_),
          at((uint32_t)row(0) * (uint32_t)stride_ + 16 * chunk())
    {
    }
    // Row and chunk of this thread's load i (the chunk is the same for all: the rows
    // differ by a multiple of sixteen).
    __device__ __forceinline__ static int row(int i) { return (i * kThreads + (int)threadIdx.x) / 8; }
    __device__ __forceinline__ static int chunk() { return (threadIdx.x % 8) ^ (row(0) & 7); }
    // Load i of values k .. k + 127 of the rows; zeros past the end.
    __device__ __forceinline__ void stage(int i, int k, ROI_LDS uint8_t* dst) const
    {
        const int wave = scalar(threadIdx.x >> 6);
        const bool live = row(i) < left && k + 16 * chunk() < len;
        load_to_lds<false>(buffer_at(base + k), live ? at : kNowhere, i * (kThreads / 8) * stride,
                           dst + (i * kThreads + wave * 64) * 16);
    }
};

// A tile's results from a wave's sums: a part of a cut tile as it is, else through LDS
// (all of which is free) to y.
template <typename T>
__device__ __forceinline__ void write_f8_tile(const LinearF8Args& a, const Piece& piece,
                                              const f32x4 (&acc)[T::kI][T::kJ], ROI_LDS uint8_t* base)
{
    using H = Held<T, 16>;
    const int wave = scalar(threadIdx.x >> 6);
    const int r0 = piece.m * T::kTile + wave / T::kAcross * 16 * T::kI;
    const int t0 = piece.n * T::kTile + wave % T::kAcross * 16 * T::kJ;
    if (piece.part >= 0) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i)
#pragma unroll
            for (int j = 0; j < T::kJ; ++j)
                *reinterpret_cast<f32x4*>(a.partial + H::part_at(piece.part, wave, i, j, 0)) = acc[i][j];
        return;
    }
    // a row of a token's results: 16 kI values of 2 bytes
    using Lines = RowsOut<T::kI, 8>;
    ROI_LDS uint8_t* mine = base + wave * (16 * T::kJ * Lines::kRow);
#pragma unroll
    for (int i = 0; i < T::kI; ++i) {
        f32x4 add = {};
        if (a.bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                add[e] = bf16_bits_to_float(a.bias[least(r0 + 4 * H::quad(i, 0) + e, a.rows - 1)]);
        }
#pragma unroll
        for (int j = 0; j < T::kJ; ++j) {
            f32x4 v = acc[i][j];
            if (a.bias) v += add;
            *reinterpret_cast<ROI_LDS u32x2*>(Lines::at(mine, H::column(j), H::quad(i, 0))) =
                u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
        }
    }
#pragma unroll 2 // code that runs once is fetched once: it is kept short
    for (int n = 0; n < 16 * T::kJ / Lines::kAtOnce; ++n) {
        int row, chunk;
        const Quad v = Lines::get(mine, n, row, chunk);
        const int t = t0 + row;
        if (t < a.tokens) store_chunk(a.y + (int64_t)t * a.rows, r0 + chunk * 8, a.rows, v);
    }
}

template <typename T, int kRing>
constexpr int f8_lds() { return kRing * 2 * T::kTile * kRowBytes + 2 * 2 * T::kTile * 4; }

template <typename T, int kRing, int kFormat>
__global__ __launch_bounds__(T::kThreads, T::kTile == 256 && T::kWaves == 4 ? 1 : 2) void linear_f8_tile_kernel(LinearF8Args a)
{
    constexpr int kTile = T::kTile, kTileBytes = kTile * kRowBytes;
    constexpr int kI = T::kI, kJ = T::kJ;
    static_assert(kRing == 2 || kRing == 4, "slots are counted in bits");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    ROI_LDS uint8_t* base = (ROI_LDS uint8_t*)&lds[0];
    ROI_LDS uint8_t* scale_lds = base + kRing * 2 * kTileBytes;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = scalar(threadIdx.x >> 6);
    const int wm = wave / T::kAcross * 16 * kI, wn = wave % T::kAcross * 16 * kJ;
    const Piece piece = piece_of(a.grid, blockIdx.x);
    const int r0 = piece.m * kTile, t0 = piece.n * kTile;

    f32x4 acc[kI][kJ] = {};
    using R = F8Rows<T>;
    const R wrows(a.w, r0, a.rows, a.cols, a.w_stride), xrows(a.x, t0, a.tokens, a.cols, a.x_stride);
    constexpr int kLoads = R::kLoads;
    auto w_buffer = [&](int s) { return base + (s & (kRing - 1)) * kTileBytes; };
    auto x_buffer = [&](int s) { return base + (kRing + (s & (kRing - 1))) * kTileBytes; };
    auto stage_w = [&](int s, int i) { wrows.stage(i, (piece.first + s) * kRowBytes, w_buffer(s)); };
    auto stage_x = [&](int s, int i) { xrows.stage(i, (piece.first + s) * kRowBytes, x_buffer(s)); };
    // quarter n of the loads that step s frees its buffers for: the weight of step
    // s + kRing and the tokens of the step behind that
    constexpr int kQuarter = kLoads / 2;
    auto stage = [&](int s, int n) {
#pragma unroll
        for (int i = 0; i < kQuarter; ++i) {
            if (n < 2)
                stage_w(s + kRing, n * kQuarter + i);
            else
                stage_x(s + 1 + kRing, (n - 2) * kQuarter + i);
        }
    };
    // the words of scales of group q (steps 4 q .. 4 q + 3 of the sum): kTile of the
    // weight's rows, then kTile of the tokens'; past the last group that one again
    constexpr int kScaleLoads = (2 * kTile + T::kThreads - 1) / T::kThreads;
    auto stage_scales = [&](int q) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const int at = i * T::kThreads + (int)threadIdx.x; // whole waves on either side
            if (at >= 2 * kTile) return;
            const uint8_t* row =
                at < kTile ? a.ws + (int64_t)(least(r0 + at, a.rows - 1) >> a.w_shift) * a.scales
                           : a.xs + (int64_t)least(t0 + at - kTile, a.tokens - 1) * a.scales;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)(row + 4 * least(q, a.scales / 4 - 1)),
                (ROI_LDS void*)(scale_lds + ((q & 1) * 2 * kTile + i * T::kThreads + wave * 64) * 4), 4, 0,
                0);
        }
    };
    const int from_w = (wm + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
    const int from_x = (wn + (lane & 15)) * kRowBytes + (g ^ (lane & 7)) * 16;
    auto read_w = [&](int s, int i) {
        ROI_LDS uint8_t* p = w_buffer(s) + i * 16 * kRowBytes;
        return joined(lds_read<i32x4>(p + from_w), lds_read<i32x4>(p + (from_w ^ 64)));
    };
    auto read_x = [&](int s, int j) {
        ROI_LDS uint8_t* p = x_buffer(s) + j * 16 * kRowBytes;
        return joined(lds_read<i32x4>(p + from_x), lds_read<i32x4>(p + (from_x ^ 64)));
    };
    int ws[kI], xs[kJ];
    auto read_scales = [&](int q) {
        ROI_LDS uint8_t* p = scale_lds + (q & 1) * 2 * kTile * 4 + (lane & 15) * 4;
#pragma unroll
        for (int i = 0; i < kI; ++i) ws[i] = lds_read<int>(p + (wm + 16 * i) * 4);
#pragma unroll
        for (int j = 0; j < kJ; ++j) xs[j] = lds_read<int>(p + (kTile + wn + 16 * j) * 4);
    };
    static_assert(kI % 4 == 0 && kLoads % 2 == 0, "registers and loads by quarters");
    i32x8 w[4], now[kJ], next[kJ];
    const int tail = a.cols % 16;
    // step s from the tokens in `now`, reading the next step's into `next`.  One step a
    // turn of the loop, and the tokens moved at its end: with two the compiler holds the
    // sums twice.
    auto step = [&](int s) {
        // Branches stand here only: the compiler moves products past those further on.
        const int S = piece.first + s;
        if (s > 0) {
            if ((S & 3) == 0) {
                read_scales(S >> 2);
                stage_scales((S >> 2) + 1);
            } else {
#pragma unroll
                for (int i = 0; i < kI; ++i) ws[i] >>= 8;
#pragma unroll
                for (int j = 0; j < kJ; ++j) xs[j] >>= 8;
            }
        }
        if (tail && S == a.grid.steps - 1) {
            // zeros for what the last piece of the rows holds behind their ends: the
            // tokens' in registers, the weight's in LDS, where its first rows are read
            // again
            const int last = a.cols % 128 / 16;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int have = tail - e % 4 * 4; // of this word's bytes
                const uint32_t keep = g + e / 4 * 4 < last    ? 0xFFFFFFFFu
                                      : g + e / 4 * 4 > last || have <= 0 ? 0u
                                      : have >= 4             ? 0xFFFFFFFFu
                                                              : 0xFFFFFFFFu >> (32 - 8 * have);
#pragma unroll
                for (int j = 0; j < kJ; ++j) now[j][e] &= (int)keep;
            }
            for (int at = threadIdx.x; at < kTile; at += T::kThreads)
                cut_piece(w_buffer(s) + at * kRowBytes + (last ^ (at & 7)) * 16, tail);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            w[0] = read_w(s, 0);
            w[1] = read_w(s, 1);
        }
        constexpr int kAhead = kI - 2; // rows ahead of the barrier
#pragma unroll
        for (int i = 0; i < kI; ++i) {
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                acc[i][j] = multiply_block<kFormat>(w[i % 4], now[j], acc[i][j], ws[i], xs[j]);
                if (j == 0) {
                    keep_order();
                    if (i < kAhead) {
                        w[(i + 2) % 4] = read_w(s, i + 2);
#pragma unroll
                        for (int n = i * kJ / kAhead; n < (i + 1) * kJ / kAhead; ++n)
                            next[n] = read_x(s + 1, n);
                        if (i < 2) stage(s - 1, 2 + i);
                    } else {
                        w[i - kAhead] = read_w(s + 1, i - kAhead);
                        stage(s, i - kAhead);
                    }
                }
            }
            keep_order();
            if (i == kAhead - 1) {
                loads_barrier<(kRing - 2) * 2 * kLoads>();
                keep_order();
            }
        }
#pragma unroll
        for (int j = 0; j < kJ; ++j) now[j] = next[j];
    };
    if (piece.count > 0) {
        stage_scales(piece.first >> 2);
        stage_scales((piece.first >> 2) + 1);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) stage_x(0, i);
#pragma unroll
        for (int s = 0; s < kRing; ++s) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage_w(s, i);
            if (s + 1 == kRing) break;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage_x(s + 1, i);
        }
        loads_barrier<(kRing - 2) * 2 * kLoads + kLoads>();
        read_scales(piece.first >> 2);
#pragma unroll
        for (int i = 0; i < kI; ++i) ws[i] >>= 8 * (piece.first & 3);
#pragma unroll
        for (int j = 0; j < kJ; ++j) xs[j] >>= 8 * (piece.first & 3);
        w[0] = read_w(0, 0);
        w[1] = read_w(0, 1);
#pragma unroll
        for (int j = 0; j < kJ; ++j) now[j] = read_x(0, j);
        // every wave has its tokens of step 0: their buffer takes those of step kRing
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        // past the end of the sum or of this part, loads are in bounds or zeros, and unused
        for (int s = 0; s < piece.count; ++s) step(s);
    }
    loads_barrier();
    write_f8_tile<T>(a, piece, acc, base);
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
    const dim3 grid(a.grid.blocks()), sums(a.grid.rest() * T::kI * T::kJ * T::kWaves / 4);
    hipLaunchKernelGGL((linear_f8_tile_kernel<T, kRing, kFormat>), grid, dim3(T::kThreads),
                       (f8_lds<T, kRing>()), stream, a);
    if (sums.x > 0) hipLaunchKernelGGL((linear_f8_sum_kernel<T>), sums, dim3(256), 0, stream, a);
}

template <int kRow, int kTokens, int kDepth, int kFormat>
void launch_f8_few_as(LinearF8Args a, hipStream_t stream)
{
    const int64_t tm = ((int64_t)a.rows + 16 * kRow - 1) / (16 * kRow);
    const int64_t tn = ((int64_t)a.tokens + kTokens - 1) / kTokens;
    a.grid.tm = (uint32_t)tm; // few tokens and fewer than 2^22 rows: a launch has room
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
    return plan.few || plan.cut.fits ? ROI_OK
                                     : fail(ROI_E_UNSUPPORTED, "y has too many elements for one call");
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
