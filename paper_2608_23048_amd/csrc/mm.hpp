// mm.hpp -- pieces shared by the tiled products (linear_i8.hip, grad_i8.hip):
// how blocks are given tiles, how tiles travel from HBM to LDS, and how they
// lie there.
//
// Tiles of operands whose sum index is contiguous ("k-rows") lie in LDS as rows
// of 128 bytes: 128 int8 or 64 bf16 values of the sum, eight 16-byte chunks.
// The matrix instructions' operands are 16 lanes reading the same chunk of 16
// consecutive rows; chunk j of row r is kept at place j ^ (r & 7), so that any
// eight of those lanes cover all the LDS banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "reach.hpp"
#include "rows.hpp"

namespace roi {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

#define ROI_LDS __attribute__((address_space(3)))

constexpr int kRowBytes = 128; // of a k-row in LDS

// Blocks of a product: a square tile over kWaves waves, two by kAcross, each
// with kI x kJ results of 16 x 16.  Their kernels are bound to two waves a SIMD,
// which they run at (a 256-tile, two 128-tiles, or one over eight waves, on a
// compute unit): with more registers than that the compiler keeps the sums in
// accumulation registers and moves them about, 100 moves a step.
constexpr int waves_of(int tile) { return tile == 256 ? 8 : 4; }
template <int kTile_, int kWaves_ = waves_of(kTile_)>
struct Tile {
    static constexpr int kTile = kTile_, kWaves = kWaves_;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kAcross = kWaves / 2;
    static constexpr int kI = kTile / 32, kJ = kTile / (16 * kAcross);
};

// Keeps the compiler from moving instructions across: the loops below are laid
// out by hand.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// The buffer that starts at p.  Its size is the largest that offsets below
// kNowhere use; every other offset is checked by the kernels themselves.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7FFFFFFF, 0x00020000);
}

// 16 bytes a lane from the buffer into LDS, lane l's at dst + 16 l (dst and
// `more`, a further offset, are the same for the wave); loads_barrier() is what
// waits for it.  kUnseen: in assembly, because the compiler has every transposing
// LDS read wait for all loads to LDS that it knows of.  (It has no result
// register.  The s_nop covers the wait states between a write of m0 or of a
// scalar operand and this read.  The compiler, which reserves m0, may take its value
// from before: a kernel uses one form or the other for all of its loads to LDS.)
template <bool kUnseen>
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t offset,
                                            uint32_t more, ROI_LDS uint8_t* dst)
{
    if constexpr (kUnseen)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :
                     : "s"((uint32_t)(uintptr_t)dst), "v"(offset), "s"(src), "s"(more)
                     : "memory");
    else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (ROI_LDS void*)dst, 16, (int)offset, (int)more,
                                                 0, 0);
}

// The same with 4 bytes a lane, lane l's at dst + 4 l.
template <bool kUnseen>
__device__ __forceinline__ void load_words_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t offset,
                                                  ROI_LDS uint8_t* dst)
{
    if constexpr (kUnseen)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
                     :
                     : "s"((uint32_t)(uintptr_t)dst), "v"(offset), "s"(src)
                     : "memory");
    else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (ROI_LDS void*)dst, 4, (int)offset, 0, 0, 0);
}

__device__ __forceinline__ int least(int a, int b) { return a < b ? a : b; }

// A barrier past which what every wave has loaded to LDS is there, its last
// kLater loads from memory apart (loads to LDS are counted with the loads from
// memory, in their order), and its other LDS operations are done.  Written out
// because the compiler's barrier waits for all loads to LDS at some places.
template <int kLater = 0>
__device__ __forceinline__ void loads_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// The wait alone, for what a wave has loaded to its own part of LDS.
template <int kLater>
__device__ __forceinline__ void loads_wait()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLater) : "memory");
}

template <typename V>
__device__ __forceinline__ V lds_read(const ROI_LDS uint8_t* p)
{
    return *reinterpret_cast<const ROI_LDS V*>(p);
}
__device__ __forceinline__ void lds_write(ROI_LDS uint8_t* p, const Quad& v)
{
    *reinterpret_cast<ROI_LDS u32x4*>(p) = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
}

// Block b of n, so that the blocks of one XCD (dispatched round-robin over the
// eight) get consecutive numbers: they share operand tiles in its L2.
__device__ __forceinline__ uint32_t xcd_order(uint32_t b, uint32_t n)
{
    const uint32_t q = n / 8, r = n % 8, x = b % 8;
    return x * q + (x < r ? x : r) + b / 8;
}

// What a block does: steps first .. first + count - 1 of the sum of tile (m, n).
// The first `full` tiles are whole; the others' sums are cut into `splits`
// parts, of which this is number `part` (-1: a whole tile).  Blocks take the
// tiles in bands of eight tile rows, so that the tiles in flight on an XCD form
// a block of few rows and columns, and the parts of equal place in the sum
// together.
struct Grid {
    uint32_t tm, tn, full, splits;
    int steps;        // of the sum
    int part, longer; // steps of a part; the first `longer` parts have one more
    __host__ __device__ uint32_t rest() const { return tm * tn - full; }
    __host__ __device__ uint32_t blocks() const { return full + rest() * splits; }
};
inline Grid grid_of(const Cut& c)
{
    return Grid{(uint32_t)c.tm,  (uint32_t)c.tn,           (uint32_t)c.full,
                (uint32_t)c.splits, (int)c.steps, (int)(c.steps / c.splits),
                (int)(c.steps % c.splits)};
}
struct Piece {
    int m, n, first, count, part;
};
// A value that is the same for the wave, in a scalar register (the divisions
// below are done in vector ones).
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ Piece tile_piece(const Grid& g, uint32_t t)
{
    constexpr uint32_t kBand = 8;
    const uint32_t first = t / (kBand * g.tn) * kBand;
    const uint32_t height = g.tm - first < kBand ? g.tm - first : kBand;
    const uint32_t in = t - first * g.tn;
    return Piece{scalar((int)(first + in % height)), scalar((int)(in / height)), 0, g.steps, -1};
}
__device__ __forceinline__ Piece piece_of(const Grid& g, uint32_t block)
{
    if (block < g.full) return tile_piece(g, xcd_order(block, g.full));
    const uint32_t b = xcd_order(block - g.full, g.rest() * g.splits);
    const uint32_t i = b % g.rest(), j = b / g.rest();
    Piece p = tile_piece(g, g.full + i);
    p.first = scalar((int)j * g.part + least((int)j, g.longer));
    p.count = g.part + ((int)j < g.longer ? 1 : 0);
    p.part = scalar((int)(i * g.splits + j));
    return p;
}

// Which results a lane holds of a wave's, by the matrix instructions' blocks of
// 16 x 16 (v_mfma 16x16: a quad of four consecutive rows of one column) or
// 32 x 32 (four such quads).  Quads are counted along the rows, four each.
template <typename T, int kBlock>
struct Held {
    static constexpr int kI = T::kI * 16 / kBlock, kJ = T::kJ * 16 / kBlock;
    static constexpr int kQuads = kBlock == 16 ? 1 : 4; // of a block
    __device__ __forceinline__ static int quad(int i, int q)
    {
        const int lane = threadIdx.x & 63;
        return kBlock == 16 ? 4 * i + lane / 16 : 8 * i + 2 * q + lane / 32;
    }
    __device__ __forceinline__ static int column(int j)
    {
        return kBlock * j + (int)(threadIdx.x & 63) % kBlock;
    }
    // Where quad q of block (i, j) of a part of a tile lies in the workspace: four
    // values a lane, in the order of the tile's threads.
    __device__ __forceinline__ static int64_t part_at(int64_t part, int wave, int i, int j, int q)
    {
        constexpr int kAll = kI * kJ * kQuads;
        return part * (T::kTile * T::kTile) +
               ((wave * kAll + (i * kJ + j) * kQuads + q) * 64 + (int)(threadIdx.x & 63)) * 4;
    }
};

// The sum of a lane's quad over the parts of a tile, in their order; `from` is its
// place in the first.  Four (eight where there are more) are on their way at a
// time, past the last that one again.
template <typename T, int kAtATime, typename Quad4, typename Value>
__device__ __forceinline__ Quad4 sum_batches(const Value* from, int splits)
{
    Quad4 sum = {};
    for (int p = 0; p < splits; p += kAtATime) {
        Quad4 v[kAtATime];
#pragma unroll
        for (int e = 0; e < kAtATime; ++e)
            v[e] = *reinterpret_cast<const Quad4*>(
                from + (int64_t)least(p + e, splits - 1) * (T::kTile * T::kTile));
#pragma unroll
        for (int e = 0; e < kAtATime; ++e)
            if (p + e < splits) sum += v[e];
    }
    return sum;
}
template <typename T, typename Quad4, typename Value>
__device__ __forceinline__ Quad4 sum_of_parts(const Value* from, int splits)
{
    return splits <= 4 ? sum_batches<T, 4, Quad4>(from, splits)
                       : sum_batches<T, 8, Quad4>(from, splits);
}

// Results of a wave to memory, by way of its own part of LDS: a lane holds four
// consecutive columns, and 16 lanes 16 different rows, so stored as they are
// they would be 32-byte pieces; past LDS a wave stores whole rows.  kBytes: of
// four results.  Chunk j of 16 bytes of row r is kept at place j ^ (r mod the
// chunks of a row).
template <int kI, int kBytes>
struct RowsOut {
    static constexpr int kChunks = kI * 4 * kBytes / 16; // of a row
    static constexpr int kRow = kChunks * 16;
    static constexpr int kAtOnce = 64 / kChunks;         // rows a wave stores at once
    static_assert(kChunks >= 8 && kChunks <= 64, "rows of 128 to 1024 bytes");

    // The four results of a quad in row `row`.
    __device__ __forceinline__ static ROI_LDS uint8_t* at(ROI_LDS uint8_t* lds, int row, int quad)
    {
        const int byte = quad * kBytes;
        return lds + row * kRow + ((byte / 16) ^ (row % kChunks)) * 16 + byte % 16;
    }
    // Store number n: this lane's row, its chunk, and the chunk's bytes.
    __device__ __forceinline__ static Quad get(ROI_LDS uint8_t* lds, int n, int& row, int& chunk)
    {
        const int lane = threadIdx.x & 63;
        row = n * kAtOnce + lane / kChunks;
        chunk = lane % kChunks;
        const u32x4 v = *reinterpret_cast<const ROI_LDS u32x4*>(
            lds + row * kRow + (chunk ^ (row % kChunks)) * 16);
        return Quad{v.x, v.y, v.z, v.w};
    }
};

// Element first .. of a row that ends at `end`, from 16 bytes of T.
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int first, int end, const Quad& v)
{
    constexpr int kN = 16 / sizeof(T);
    if (first + kN <= end) {
        store_any(row + first, v);
    } else {
        uint64_t lo = v.w[0] | ((uint64_t)v.w[1] << 32), hi = v.w[2] | ((uint64_t)v.w[3] << 32);
        for (int e = first; e < end; ++e) {
            row[e] = (T)lo;
            lo = lo >> (8 * sizeof(T)) | hi << (64 - 8 * sizeof(T));
            hi >>= 8 * sizeof(T);
        }
    }
}

} // namespace roi
