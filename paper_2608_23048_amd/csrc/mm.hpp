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
#include "rows.hpp"

namespace roi {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

#define ROI_LDS __attribute__((address_space(3)))

constexpr int kRowBytes = 128; // of a k-row in LDS

// Blocks of a product: a square tile over kWaves waves, two by kAcross, each
// with kI x kJ results of 16 x 16.
template <int kTile>
struct Tile {
    static constexpr int kWaves = kTile == 256 ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kAcross = kWaves / 2;
    static constexpr int kI = kTile / 32, kJ = kTile / (16 * kAcross);
};

// Keeps the compiler from moving instructions across: the loops below are laid
// out by hand.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// A byte offset that no buffer below reaches: a load from there gives zeros.
constexpr uint32_t kNowhere = 0x80000000u;

// The buffer that starts at p.  Its size is the largest that offsets below
// kNowhere use; every other offset is checked by the kernels themselves.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7FFFFFFF, 0x00020000);
}

// 16 bytes a lane from the buffer into LDS, lane l's at dst + 16 l (dst and
// `more`, a further offset, are the same for the wave).
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t offset,
                                            uint32_t more, ROI_LDS uint8_t* dst)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (ROI_LDS void*)dst, 16, (int)offset, (int)more, 0,
                                             0);
}

__device__ __forceinline__ int least(int a, int b) { return a < b ? a : b; }

// A barrier past which what every wave has loaded to LDS is there: the barrier
// itself waits for a wave's LDS operations only, and loads to LDS are counted
// with the loads from memory.
__device__ __forceinline__ void loads_barrier()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
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

// Tile t of tm x tn, in bands of `band` tile rows, so that the tiles in flight
// on an XCD form a block of few rows and columns.
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t tm, uint32_t tn, uint32_t band,
                                        int& m, int& n)
{
    const uint32_t first = t / (band * tn) * band;
    const uint32_t height = tm - first < band ? tm - first : band;
    const uint32_t in = t - first * tn;
    m = (int)(first + in % height);
    n = (int)(in / height);
}

} // namespace roi
