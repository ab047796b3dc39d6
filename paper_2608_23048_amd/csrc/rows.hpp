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

// Bytes k .. k + N - 1 of a row of `len` bytes, zeros past its end (nothing
// past it is read).
template <typename V>
__device__ __forceinline__ V load_row(const uint8_t* row, int64_t k, int64_t len)
{
    constexpr int N = sizeof(V);
    if (k + N <= len) return load_any<V>(row + k);
    V v{};
    for (int i = 0; i < N; ++i)
        if (k + i < len) v.w[i / 4] |= (uint32_t)row[k + i] << (8 * (i % 4));
    return v;
}

} // namespace roi
