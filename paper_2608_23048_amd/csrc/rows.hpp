// rows.hpp -- loads and stores shared by the int8 row kernels and products:
// vectors at any byte address (a row of odd length starts anywhere), and reads
// that stop at a row's end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace roi {

struct Pair {
    uint32_t w[2];
};
struct Quad {
    uint32_t w[4];
};

// gfx950 loads and stores global vectors at any byte address; the packed
// wrapper tells the compiler that no alignment is known.
template <typename V>
struct __attribute__((packed)) AnyAddress {
    V v;
};
template <typename V>
__device__ __forceinline__ V load_any(const void* p)
{
    return static_cast<const AnyAddress<V>*>(p)->v;
}
template <typename V>
__device__ __forceinline__ void store_any(void* p, const V& v)
{
    static_cast<AnyAddress<V>*>(p)->v = v;
}

// The same past the caches' usual order, for what is touched once.
template <typename V>
__device__ __forceinline__ V stream_load_any(const void* p)
{
    constexpr int kWords = sizeof(V) / 4;
    typedef uint32_t Vec __attribute__((ext_vector_type(kWords < 4 ? kWords : 4), aligned(1)));
    V v;
#pragma unroll
    for (int i = 0; i < kWords / (kWords < 4 ? kWords : 4); ++i) {
        const Vec x = __builtin_nontemporal_load(static_cast<const Vec*>(p) + i);
        __builtin_memcpy(reinterpret_cast<char*>(&v) + sizeof(Vec) * i, &x, sizeof(Vec));
    }
    return v;
}
template <typename V>
__device__ __forceinline__ void stream_store_any(void* p, const V& v)
{
    typedef uint32_t Vec __attribute__((ext_vector_type(sizeof(V) / 4), aligned(1)));
    Vec x;
    __builtin_memcpy(&x, &v, sizeof(V));
    __builtin_nontemporal_store(x, static_cast<Vec*>(p));
}

// Bytes k .. k + N - 1 of a row of `len` bytes, zeros past its end (nothing
// past it is read): the row's last N bytes, moved down, where it ends within them.
template <typename V>
__device__ __forceinline__ V load_row(const uint8_t* row, int64_t k, int64_t len)
{
    constexpr int N = sizeof(V);
    if (k + N <= len) return load_any<V>(row + k);
    V v{};
    if (k >= len) return v;
    if (len >= N) {
        v = load_any<V>(row + len - N);
        const int bits = 8 * (int)(k + N - len); // 8 .. 8 N - 8
        if constexpr (N == 4) {
            v.w[0] >>= bits;
        } else if constexpr (N == 8) {
            const uint64_t x = (v.w[0] | (uint64_t)v.w[1] << 32) >> bits;
            v = V{(uint32_t)x, (uint32_t)(x >> 32)};
        } else {
            uint64_t lo = v.w[0] | (uint64_t)v.w[1] << 32, hi = v.w[2] | (uint64_t)v.w[3] << 32;
            if (bits >= 64) {
                lo = hi >> (bits - 64);
                hi = 0;
            } else {
                lo = lo >> bits | hi << (64 - bits);
                hi >>= bits;
            }
            v = V{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
        }
        return v;
    }
    for (int i = 0; i < N; ++i)
        if (k + i < len) v.w[i / 4] |= (uint32_t)row[k + i] << (8 * (i % 4));
    return v;
}

// Rows of `len` bytes to rows of `row` bytes (a multiple of 16, at least len; `to`
// is aligned to 16), zeros behind each; with `rows` 0 nothing.
struct RowsCopy {
    const void* from;
    void* to;
    int64_t rows, len, row;
};
// Both copies in one launch (rows_i8.hip).
void launch_copy_rows(const RowsCopy& a, const RowsCopy& b, hipStream_t stream);

} // namespace roi
