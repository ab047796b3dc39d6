// adamw.hip -- one AdamW step over many tensors, moments in fp32 or in 8 bits.
//
// With 8 bits a value moves 16 bytes (param 4 + 4, grad 4, moments 2 x (1 + 1)) and
// 4 / 128 of scales instead of 28; both forms are bound by HBM (358 million values in
// 8 bits take 962 us, 6.0 TB/s; 802816 in 32 bits 4.5, 5.0 TB/s).  A half wave holds
// a block of 128 consecutive values, four a lane, so that the block's largest
// moments take five cross-lane steps and a lane's four noise words one Philox
// call.  The moments are rounded by the stochastic conversion instruction: as
// measured on gfx950, v_cvt_sr_fp8_f32 of t in [0, 448] and a word gives
// floor(t / u + (word >> 12) 2^-20) u, with u the spacing at t (2^-9 below 2^-6).
#include <hip/hip_runtime.h>

#include <new>

#include "f8.hpp"
#include "host.hpp"
#include "roi.h"

namespace roi {
namespace {

// A launch takes as many pieces (tensors) as 4 KiB of arguments hold; a piece is given
// blocks by its units of 512 values, a wave each.
constexpr int kStepPieces = 62;
constexpr int kUnit = 512, kWavesOfBlock = 4;
constexpr int64_t kMostStepBlocks = 0xFFFFFE; // of a launch
struct StepPiece {
    float* param;
    const void* grad;
    void* avg;
    void* sq;
    uint8_t* avg_scale;
    uint8_t* sq_scale;
    uint64_t first_numel; // the first block in the high 24 bits (all ones: no piece), the values in 40
    uint64_t offset;

    __host__ __device__ int64_t numel() const { return (int64_t)(first_numel & kMaxStepValues - 1); }
    __host__ __device__ int64_t blocks() const
    {
        const int64_t n = (numel() + kUnit * kWavesOfBlock - 1) / (kUnit * kWavesOfBlock);
        return n < kMostStepBlocks ? n : kMostStepBlocks;
    }
};
struct StepBatch {
    StepPiece p[kStepPieces];
    AdamStep adam;
    double beta1, beta2;
    float beta1_rest, one_m_beta1_rest; // what adam.beta1 and one_m_beta1 lack
    uint32_t k0, k1, step_lo, step_hi;
};
static_assert(sizeof(StepBatch) <= 4096, "kernel arguments");

// The piece that owns this block: the last that starts at or before it.  A lane looks
// at a piece each: a search would wait for the arguments' memory at each of its six
// steps (61 tensors of 5001 values took 5.5 us a launch so).
__device__ __forceinline__ int find_step_piece(const StepBatch& a, uint32_t block)
{
    const int lane = threadIdx.x & 63;
    const uint32_t first = lane < kStepPieces ? (uint32_t)(a.p[lane].first_numel >> 40) : 0xFFFFFFu;
    return __builtin_popcountll(__builtin_amdgcn_ballot_w64(first <= block)) - 1;
}

// Values k .. k + 3 of n; zeros past the end.
__device__ __forceinline__ f32x4 load_four(const float* p, int64_t k, int64_t n)
{
    if (k + 4 <= n) return stream_load(reinterpret_cast<const f32x4*>(p + k));
    f32x4 v = {};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k + i < n) v[i] = p[k + i];
    return v;
}
__device__ __forceinline__ f32x4 load_four(const uint16_t* p, int64_t k, int64_t n)
{
    u32x2 w = {};
    if (k + 4 <= n) {
        w = stream_load(reinterpret_cast<const u32x2*>(p + k));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < n) w[i / 2] |= (uint32_t)p[k + i] << (16 * (i % 2));
    }
    return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u),
                 __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u)};
}
__device__ __forceinline__ uint32_t load_four(const uint8_t* p, int64_t k, int64_t n)
{
    if (k + 4 <= n) return stream_load(reinterpret_cast<const uint32_t*>(p + k));
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k + i < n) w |= (uint32_t)p[k + i] << (8 * i);
    return w;
}
__device__ __forceinline__ void store_four(float* p, int64_t k, int64_t n, f32x4 v)
{
    if (k + 4 <= n) {
        stream_store(v, reinterpret_cast<f32x4*>(p + k));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < n) p[k + i] = v[i];
    }
}
__device__ __forceinline__ void store_four(uint8_t* p, int64_t k, int64_t n, uint32_t w)
{
    if (k + 4 <= n) {
        stream_store(w, reinterpret_cast<uint32_t*>(p + k));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < n) p[k + i] = (uint8_t)(w >> (8 * i));
    }
}

// t (|t| <= 448) to e4m3 by the random word, as byte kByte of the result; NaN where
// `finite` is false.
template <int kByte>
__device__ __forceinline__ int round_by(float t, uint32_t word, int old)
{
    return __builtin_amdgcn_cvt_sr_fp8_f32(t, (int)word, old, kByte);
}

// m' = beta1 m + (1 - beta1) g to a rounding of its own, also where the two cancel: what
// the products and their sum leave out, and what the factors lost to fp32, is added last.
__device__ __forceinline__ float mixed(const StepBatch& a, float m, float g)
{
    const float p = a.adam.one_m_beta1 * g, q = a.adam.beta1 * m, sum = q + p, of_p = sum - q;
    const float rest = __builtin_fmaf(a.adam.beta1, m, -q) + __builtin_fmaf(a.adam.one_m_beta1, g, -p) +
                       ((q - (sum - of_p)) + (p - of_p));
    return sum + __builtin_fmaf(a.beta1_rest, m, __builtin_fmaf(a.one_m_beta1_rest, g, rest));
}

// Whether fp32 bits of t, with an error of up to 4 of them, and the 20 bits that are
// added leave the rounding open: the sum's low bits are near 0 (an e4m3 step is 2^20 of
// t's bits from 2^-6 on, below it 2^-9).
__device__ __forceinline__ bool undecided(float t, uint32_t chance)
{
    const uint32_t low = t < 0x1p-6f ? (uint32_t)(t * 0x1p29f) : __float_as_uint(t);
    return ((low + chance + 4) & 0xFFFFF) < 8;
}
// Whether so near a largest magnitude's fraction is to 3/4 (scale_byte).
__device__ __forceinline__ bool undecided_scale(uint32_t largest)
{
    return ((largest + 0x1FFFFFu + 4) & 0x7FFFFFu) < 8;
}
// Four elements' new moments (m, r: old values in, new m and root out) and parameters in fp32.
__device__ __forceinline__ void step_four(const StepBatch& a, float m_scale, float r_scale, f32x4 g,
                                          f32x4& par, float (&m)[4], float (&r)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float root = r[e] * r_scale;
        m[e] = mixed(a, m[e] * m_scale, g[e]);
        const float v = __builtin_fmaf(a.adam.beta2, root * root, a.adam.one_m_beta2 * (g[e] * g[e]));
        r[e] = __builtin_amdgcn_sqrtf(v);
        const float den = __builtin_fmaf(r[e], a.adam.inv_sqrt_bc2, a.adam.eps);
        par[e] = __builtin_fmaf(-a.adam.step_size * m[e], __builtin_amdgcn_rcpf(den), par[e] * a.adam.decay);
    }
}
__device__ __forceinline__ uint4 words_of_four(const StepBatch& a, uint64_t element)
{
    const uint64_t block = element >> 2;
    return philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), a.step_lo, a.step_hi, a.k0, a.k1);
}
// E of a block (the largest over its 32 lanes) from four magnitudes a lane in 64 bits.
__device__ __forceinline__ int wide_scale(const double (&x)[4])
{
    uint32_t most_e = 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint64_t b = __builtin_bit_cast(uint64_t, x[e]);
        const int of = (int)((b + ((1ull << 50) - 1)) >> 52) - 1023 + 127 - kF8Top<ROI_E4M3>;
        most_e = most(most_e, (uint32_t)(of > 1 ? of : 1));
    }
    return (int)most_of_32(most_e);
}
// floor(t / u + chance) u of t = x 2^(127 - scale).
__device__ __forceinline__ float wide_round(double x, int scale, double chance)
{
    const double t = x * __builtin_bit_cast(double, (uint64_t)(1023 + 127 - scale) << 52);
    const int power = (int)(__builtin_bit_cast(uint64_t, t) >> 52);
    const int step = (power > 1023 - 6 ? power : 1023 - 6) - 3; // u = 2^(step - 1023)
    return (float)(__builtin_floor(t * __builtin_bit_cast(double, (uint64_t)(2046 - step) << 52) + chance) *
                   __builtin_bit_cast(double, (uint64_t)step << 52));
}

// The moments of four elements, m and r in 32 bits, again in 64, which decide: their bytes
// and their blocks' scales.  kFinite: in 32 bits all of the wave's are finite.  Squares of
// what fp32 holds are finite in 64 bits, and so is an old moment that is held as 2^128 (a
// largest one may be rounded up to it); what is not finite there is stored as NaN.
template <bool kFinite>
__device__ __forceinline__ void moments_again(const StepBatch& a, uint32_t mq, uint32_t rq, int old_ms,
                                              int old_rs, f32x4 g, const float (&m)[4],
                                              const float (&r)[4], const uint32_t (&bits)[4], int& mo,
                                              int& ro, int& ms, int& rs)
{
    auto value = [](float q, int scale) {
        return kFinite ? (double)(q * scale_value(scale)) : (double)q * (double)scale_value(scale);
    };
    // takes what is not finite out of x; NaN bytes in its places
    auto take_out = [](double(&x)[4]) {
        int nan = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!kFinite && !(x[e] < __builtin_inf())) {
                x[e] = 0.0;
                nan |= 127 << (8 * e);
            }
        return nan;
    };
    double x[4];
    float f[4], old[4], sign[4];
    from_f8x4<ROI_E4M3>(mq, old);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = a.beta1 * value(old[e], old_ms) + (1.0 - a.beta1) * (double)g[e];
        // of the sign that it has in 32 bits, if it has a value there
        if (kFinite || __builtin_fabsf(m[e]) < __builtin_inff())
            sign[e] = m[e];
        else
            sign[e] = __builtin_fabs(x[e]) < __builtin_inf() ? (float)x[e] : 0.0f;
        x[e] = __builtin_fabs(x[e]);
    }
    int nan = take_out(x);
    ms = wide_scale(x);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        f[e] = __builtin_copysignf(wide_round(x[e], ms, (double)(bits[e] & 4095) * 0x1p-12), sign[e]);
    mo = (int)to_f8x4<ROI_E4M3>(f[0], f[1], f[2], f[3]) | nan;
    from_f8x4<ROI_E4M3>(rq, old);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double root = value(old[e], old_rs), g_e = (double)g[e];
        x[e] = __builtin_sqrt(a.beta2 * (root * root) + (1.0 - a.beta2) * (g_e * g_e));
    }
    nan = take_out(x);
    rs = wide_scale(x);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = wide_round(x[e], rs, (double)(bits[e] >> 12) * 0x1p-20);
        const bool above = kFinite || r[e] < __builtin_inff() ? r[e] > 0.0f : x[e] > 0.0;
        if (above && f[e] < 0x1p-9f) f[e] = 0x1p-9f;
    }
    ro = (int)to_f8x4<ROI_E4M3>(f[0], f[1], f[2], f[3]) | nan;
}

// Values k .. k + 3 of a lane whose wave has some that are not finite in fp32, from memory:
// what is finite in 64 bits is stored as any other value, whatever its neighbours are.
// Where g or the old root passes 2^64 its square is an infinity, and where an old moment is
// held as 2^128 that is: the parameter's step is taken on 2^-75 of them.
template <typename G>
__device__ __forceinline__ void step_not_finite(const StepBatch& a, const StepPiece& p, int64_t k,
                                                int64_t n, int64_t block, bool live)
{
    uint8_t* avg = static_cast<uint8_t*>(p.avg);
    uint8_t* sq = static_cast<uint8_t*>(p.sq);
    const f32x4 g = load_four(static_cast<const G*>(p.grad), k, n), was = load_four(p.param, k, n);
    const uint32_t mq = load_four(avg, k, n), rq = load_four(sq, k, n);
    int ms = live ? p.avg_scale[block] : 1, rs = live ? p.sq_scale[block] : 1;
    const float m_scale = scale_value(ms), r_scale = scale_value(rs);
    float m[4], r[4], old_m[4], old_r[4];
    from_f8x4<ROI_E4M3>(mq, old_m);
    from_f8x4<ROI_E4M3>(rq, old_r);
    f32x4 par = was;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m[e] = old_m[e];
        r[e] = old_r[e];
    }
    step_four(a, m_scale, r_scale, g, par, m, r);
    constexpr float kBy = 0x1p-75f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (__builtin_fabsf(m[e]) < __builtin_inff() && r[e] < __builtin_inff()) continue;
        const float ge = g[e] * kBy, root = old_r[e] * (r_scale * kBy);
        const float v = __builtin_fmaf(a.adam.beta2, root * root, a.adam.one_m_beta2 * (ge * ge));
        const float re = r[e] < __builtin_inff() ? r[e] * kBy : __builtin_amdgcn_sqrtf(v);
        const float me = __builtin_fmaf(a.adam.beta1, old_m[e] * (m_scale * kBy), a.adam.one_m_beta1 * ge);
        const float den = __builtin_fmaf(re, a.adam.inv_sqrt_bc2, a.adam.eps * kBy);
        par[e] = __builtin_fmaf(-a.adam.step_size * me, __builtin_amdgcn_rcpf(den), was[e] * a.adam.decay);
    }
    store_four(p.param, k, n, par);
    const uint4 word = words_of_four(a, p.offset + (uint64_t)k);
    const uint32_t bits[4] = {word.x, word.y, word.z, word.w};
    int mo, ro;
    moments_again<false>(a, mq, rq, ms, rs, g, m, r, bits, mo, ro, ms, rs);
    store_four(avg, k, n, (uint32_t)mo);
    store_four(sq, k, n, (uint32_t)ro);
    if ((threadIdx.x & 31) == 0 && live) {
        p.avg_scale[block] = (uint8_t)ms;
        p.sq_scale[block] = (uint8_t)rs;
    }
}

// In 8 bits the stored moments are those of 64-bit arithmetic: a rounding that fp32 leaves
// open is done again in 64 bits, by one wave in some 200 (of moments that are 0, one in 16:
// every 4096th has chance 0).  Without that 358 million values took 911 us, and some 300
// moments came out on the other side.  What is not finite waits until the others of a
// turn are stored: beside them it took registers and scalar registers (985 to 1019 us, so
// 962).  Five waves fit on a SIMD; four take 1093 us, six 1112, eight with some
// registers in memory 2057.
template <typename G, int kBits>
__global__ __launch_bounds__(256, kBits == 8 ? 5 : 8) void adamw_kernel(StepBatch a)
{
    const int i = __builtin_amdgcn_readfirstlane(find_step_piece(a, blockIdx.x));
    const StepPiece p = a.p[i];
    const uint32_t first = (uint32_t)(p.first_numel >> 40);
    const int lane = threadIdx.x & 63;
    const int64_t n = p.numel(), units = (n + kUnit - 1) / kUnit, blocks = p.blocks();
    const G* grad = static_cast<const G*>(p.grad);
    for (int64_t u = (int64_t)(blockIdx.x - first) * kWavesOfBlock + (threadIdx.x >> 6); u < units;
         u += blocks * kWavesOfBlock) {
        const int64_t k0 = u * kUnit + 4 * lane;
        f32x4 par[2], g[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            par[j] = load_four(p.param, k0 + 256 * j, n);
            g[j] = load_four(grad, k0 + 256 * j, n);
        }
        if constexpr (kBits == 32) {
            float* avg = static_cast<float*>(p.avg);
            float* sq = static_cast<float*>(p.sq);
            f32x4 m[2], v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[j] = load_four(avg, k0 + 256 * j, n);
                v[j] = load_four(sq, k0 + 256 * j, n);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float pe = par[j][e], me = m[j][e], ve = v[j][e];
                    adamw_update(a.adam, g[j][e], pe, me, ve);
                    par[j][e] = pe;
                    m[j][e] = me;
                    v[j][e] = ve;
                }
                store_four(p.param, k0 + 256 * j, n, par[j]);
                store_four(avg, k0 + 256 * j, n, m[j]);
                store_four(sq, k0 + 256 * j, n, v[j]);
            }
        } else {
            uint8_t* avg = static_cast<uint8_t*>(p.avg);
            uint8_t* sq = static_cast<uint8_t*>(p.sq);
            uint32_t mq[2], rq[2];
            int ms[2], rs[2];
            const int64_t block0 = u * 4 + lane / 32; // of 128 values
            const int64_t held = (n + kF8Block - 1) / kF8Block;
            int later = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                mq[j] = load_four(avg, k0 + 256 * j, n);
                rq[j] = load_four(sq, k0 + 256 * j, n);
                const bool live = block0 + 2 * j < held;
                ms[j] = live ? p.avg_scale[block0 + 2 * j] : 1;
                rs[j] = live ? p.sq_scale[block0 + 2 * j] : 1;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float m[4], r[4];
                from_f8x4<ROI_E4M3>(mq[j], m);
                from_f8x4<ROI_E4M3>(rq[j], r);
                const int old_ms = ms[j], old_rs = rs[j];
                const float m_scale = scale_value(old_ms), r_scale = scale_value(old_rs);
                step_four(a, m_scale, r_scale, g[j], par[j], m, r);
                uint32_t m_most = 0, r_most = 0; // what is not finite above every number
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    m_most = most(m_most, __float_as_uint(m[e]) & 0x7FFFFFFFu);
                    r_most = most(r_most, __float_as_uint(r[e]));
                }
                const bool finite = __builtin_amdgcn_ballot_w64(most(m_most, r_most) >= kInfinity) == 0;
                if (__builtin_expect(!finite, 0)) {
                    later |= 1 << j;
                    continue;
                }
                store_four(p.param, k0 + 256 * j, n, par[j]);
                m_most = most_of_32(m_most);
                r_most = most_of_32(r_most);
                ms[j] = scale_byte<ROI_E4M3>(m_most);
                rs[j] = scale_byte<ROI_E4M3>(r_most);
                const float m_inv = inverse_scale(ms[j]), r_inv = inverse_scale(rs[j]);
                const uint4 word = words_of_four(a, p.offset + (uint64_t)(k0 + 256 * j));
                const uint32_t bits[4] = {word.x, word.y, word.z, word.w};
                float t[4], s[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    t[e] = m[e] * m_inv;
                    s[e] = r[e] * r_inv;
                    if (s[e] > 0.0f && s[e] < 0x1p-9f) s[e] = 0x1p-9f; // m is not divided by eps alone
                }
                int mo = round_by<0>(t[0], bits[0] << 20, 0);
                mo = round_by<1>(t[1], bits[1] << 20, mo);
                mo = round_by<2>(t[2], bits[2] << 20, mo);
                mo = round_by<3>(t[3], bits[3] << 20, mo);
                int ro = round_by<0>(s[0], bits[0], 0);
                ro = round_by<1>(s[1], bits[1], ro);
                ro = round_by<2>(s[2], bits[2], ro);
                ro = round_by<3>(s[3], bits[3], ro);
                bool near = undecided_scale(m_most) || undecided_scale(r_most);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    near |= undecided(__builtin_fabsf(t[e]), bits[e] << 20 >> 12) || undecided(s[e], bits[e] >> 12);
                if (__builtin_amdgcn_ballot_w64(near)) // one in some 200
                    moments_again<true>(a, mq[j], rq[j], old_ms, old_rs, g[j], m, r, bits, mo, ro, ms[j], rs[j]);
                store_four(avg, k0 + 256 * j, n, (uint32_t)mo);
                store_four(sq, k0 + 256 * j, n, (uint32_t)ro);
                if (lane % 32 == 0 && block0 + 2 * j < held) {
                    p.avg_scale[block0 + 2 * j] = (uint8_t)ms[j];
                    p.sq_scale[block0 + 2 * j] = (uint8_t)rs[j];
                }
            }
            if (__builtin_expect(later, 0)) {
#pragma unroll 1
                for (int j = 0; j < 2; ++j)
                    if (later >> j & 1)
                        step_not_finite<G>(a, p, k0 + 256 * j, n, block0 + 2 * j, block0 + 2 * j < held);
            }
        }
    }
}

using StepFn = void (*)(StepBatch);

int adamw_run(const roi_step_tensor* t, int count, int grad_dtype, int bits, uint64_t seed,
              uint64_t step, const roi_step_params* opt, hipStream_t stream)
{
    StepBatch b{};
    bool todo;
    if (int st = validate_step(t, count, grad_dtype, bits, opt, &b.adam, &todo)) return st;
    if (!todo) return ok();
    const StepFn fn = bits == 8 ? (grad_dtype == ROI_FP32 ? adamw_kernel<float, 8> : adamw_kernel<uint16_t, 8>)
                                : (grad_dtype == ROI_FP32 ? adamw_kernel<float, 32> : adamw_kernel<uint16_t, 32>);
    b.beta1_rest = (float)(opt->beta1 - (double)b.adam.beta1);
    b.beta1 = opt->beta1;
    b.beta2 = opt->beta2;
    b.one_m_beta1_rest = (float)(1.0 - opt->beta1 - (double)b.adam.one_m_beta1);
    b.k0 = (uint32_t)seed;
    b.k1 = (uint32_t)(seed >> 32);
    b.step_lo = (uint32_t)step;
    b.step_hi = (uint32_t)(step >> 32);
    int pieces = 0;
    int64_t blocks = 0;
    auto flush = [&]() -> int {
        if (pieces == 0) return ROI_OK;
        for (int i = pieces; i < kStepPieces; ++i) b.p[i].first_numel = ~(uint64_t)0;
        hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(64 * kWavesOfBlock), 0, stream, b);
        pieces = 0;
        blocks = 0;
        return launch_status("roi_adamw_grouped");
    };
    for (int i = 0; i < count; ++i) {
        if (t[i].numel == 0) continue;
        StepPiece p{t[i].param,     t[i].grad,     t[i].exp_avg,          t[i].exp_avg_sq,
                    t[i].avg_scale, t[i].sq_scale, (uint64_t)t[i].numel, t[i].elem_offset};
        if (pieces == kStepPieces || blocks + p.blocks() > kMostStepBlocks)
            if (int st = flush()) return st;
        p.first_numel |= (uint64_t)blocks << 40;
        blocks += p.blocks();
        b.p[pieces++] = p;
    }
    return flush();
}

} // namespace
} // namespace roi

using namespace roi;

extern "C" int roi_adamw_grouped(const roi_step_tensor* tensors, int count, int grad_dtype, int bits,
                                 uint64_t seed, uint64_t step, const roi_step_params* opt,
                                 hipStream_t stream)
{
    try {
        return adamw_run(tensors, count, grad_dtype, bits, seed, step, opt, stream);
    } catch (const std::bad_alloc&) {
        return ROI_E_HIP;
    }
}
