// f8.hpp -- 8-bit floats with one power-of-two scale for each block of 128
// values: how a block's scale follows from its largest magnitude, conversions
// and reductions (blocks_f8.hip, linear_f8.hip, adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "rows.hpp"

namespace roi {

constexpr int kF8Block = 128;
constexpr uint32_t kInfinity = 0x7F800000u; // fp32 bits; magnitudes from here on are not finite
constexpr int kNoScale = 127;               // the byte behind a row's last block

// What E is less than the biased exponent: e4m3 magnitudes end at 1.75 2^8, e5m2's
// at 1.75 2^15.
template <int kFormat>
constexpr int kF8Top = kFormat == ROI_E4M3 ? 8 : 15;

// The byte E of a block whose largest finite magnitude has these bits.  Adding
// 2^21 - 1 carries into the exponent exactly where the fraction is over 3/4.
template <int kFormat>
__device__ __forceinline__ int scale_byte(uint32_t largest)
{
    const int e = (int)((largest + 0x1FFFFFu) >> 23) - kF8Top<kFormat>;
    return e > 1 ? e : 1;
}
// 2^(127 - E) for E from 0 to 253, and 2^(E - 127) for E from 1.
__device__ __forceinline__ float inverse_scale(int e) { return __uint_as_float((uint32_t)(254 - e) << 23); }
__device__ __forceinline__ float scale_value(int e)
{
    return e == 0 ? 0x1p-127f : __uint_as_float(e == 255 ? 0x7FC00000u : (uint32_t)e << 23);
}

// Magnitude bits of a value, 0 if it is not finite.
__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < kInfinity ? b : 0;
}

template <int kFormat>
__device__ __forceinline__ uint32_t to_f8x4(float a, float b, float c, float d)
{
    int v = 0;
    if constexpr (kFormat == ROI_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
    }
    return (uint32_t)v;
}
template <int kFormat>
__device__ __forceinline__ void from_f8x4(uint32_t w, float (&f)[4])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 lo, hi;
    if constexpr (kFormat == ROI_E4M3) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    }
    f[0] = lo.x;
    f[1] = lo.y;
    f[2] = hi.x;
    f[3] = hi.y;
}

__device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The largest over the 16 lanes of a row, in all of them.
template <int kRotate>
__device__ __forceinline__ uint32_t most_with_rotated(uint32_t v)
{
    return most(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + kRotate, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t most_of_16(uint32_t v)
{
    v = most_with_rotated<8>(v);
    v = most_with_rotated<4>(v);
    v = most_with_rotated<2>(v);
    return most_with_rotated<1>(v);
}
// The larger of this lane's and that of lane ^ 16, and of lane ^ 32: both swap
// instructions of a value with itself leave it in one result and the other lane's in the
// other.
__device__ __forceinline__ uint32_t most_with_16(uint32_t v)
{
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return most(s[0], s[1]);
}
__device__ __forceinline__ uint32_t most_with_32(uint32_t v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return most(s[0], s[1]);
}
// The largest over the 32 lanes of a half wave, in all of them.
__device__ __forceinline__ uint32_t most_of_32(uint32_t v) { return most_with_16(most_of_16(v)); }

} // namespace roi
