// Activations in 8 bits: the elements of the three types, one group's unit and codes, the activation functions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "ogq_common.cuh"

namespace ogq {

constexpr int kAct8Group = 32;     // columns that share a unit
constexpr uint32_t kAct8MinByte = 7, kAct8MaxByte = 248, kAct8NanByte = 255;  // units 2^-120 ... 2^121; NaN

__host__ __device__ inline int64_t act8_groups(int64_t cols) { return (cols + kAct8Group - 1) / kAct8Group; }

// ---------------------------------------------------------------------------
// Elements
// ---------------------------------------------------------------------------
// Plain loads throughout: an output may be the input it belongs to (y over x, dx over dy), which the read-only path
// does not allow.
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Eight elements from a 16-byte boundary, as they lie in memory.
template <class E> struct Raw8 { uint4 a; };
template <> struct Raw8<float> { uint4 a, b; };

template <class E>
__device__ __forceinline__ Raw8<E> load_raw8(const E* p)
{
    Raw8<E> r;
    r.a = *reinterpret_cast<const uint4*>(p);
    if constexpr (sizeof(E) == 4) r.b = *reinterpret_cast<const uint4*>(p + 4);
    return r;
}
template <class E>
__device__ __forceinline__ Raw8<E> zero_raw8()
{
    Raw8<E> r;
    r.a = make_uint4(0, 0, 0, 0);
    if constexpr (sizeof(E) == 4) r.b = r.a;
    return r;
}

__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8])
{
    v[0] = __uint_as_float(r.a.x); v[1] = __uint_as_float(r.a.y); v[2] = __uint_as_float(r.a.z); v[3] = __uint_as_float(r.a.w);
    v[4] = __uint_as_float(r.b.x); v[5] = __uint_as_float(r.b.y); v[6] = __uint_as_float(r.b.z); v[7] = __uint_as_float(r.b.w);
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&v)[8])
{
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<__half>& r, float (&v)[8])
{
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

template <class E>
__device__ __forceinline__ void store8(E* p, const float (&v)[8])
{
    if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (__is_same(E, __half)) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---------------------------------------------------------------------------
// One group
// ---------------------------------------------------------------------------
// Byte of the group whose largest magnitude has the bits m (of an fp32 number; NaN above infinity above all finite ones):
// e = exponent(m) - 6, one more when the mantissa is above 127/64; the carry of the addition is that comparison.
__device__ __forceinline__ uint32_t act8_byte(uint32_t m)
{
    if (m >= 0x7f800000u) return kAct8NanByte;
    const int b = (int)((m + 0x1ffffu) >> 23) - 6;
    return (uint32_t)min(max(b, (int)kAct8MinByte), (int)kAct8MaxByte);
}
__device__ __forceinline__ float act8_unit(uint32_t byte) { return __uint_as_float(byte << 23); }  // 255: infinity, and 0 * infinity = NaN
// 1 / unit; a group that reads as NaN has codes 0: its values are not multiplied but replaced
__device__ __forceinline__ float act8_inverse_unit(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Code of one value, in the low byte of the result; t = value / unit is exact (a power of two), and so is the addition of
// 1.5 * 2^23, whose rounding to an integer is the one to nearest even.
__device__ __forceinline__ uint32_t act8_code(float v, uint32_t byte)
{
    if (byte == kAct8NanByte) return 0u;
    float t = __fmul_rn(v, act8_inverse_unit(byte));
    if (byte == kAct8MaxByte) t = fminf(fmaxf(t, -127.f), 127.f);  // the only unit that can be too small
    return __float_as_uint(__fadd_rn(t, 12582912.f));
}
__device__ __forceinline__ uint32_t act8_code_random(float v, uint32_t byte, uint32_t word)
{
    if (byte == kAct8NanByte) return 0u;
    float t = __fmul_rn(v, act8_inverse_unit(byte));
    if (byte == kAct8MaxByte) t = fminf(fmaxf(t, -127.f), 127.f);
    const float f = floorf(t);
    const float up = (float)(word >> 8) < __fmul_rn(__fsub_rn(t, f), 16777216.f) ? 1.f : 0.f;
    return __float_as_uint(__fadd_rn(__fadd_rn(f, up), 12582912.f));
}

// Eight codes in a row.
__device__ __forceinline__ uint2 pack_codes(const uint32_t (&c)[8])
{
    return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}

template <bool RANDOM>
__device__ __forceinline__ uint2 act8_codes(const float (&v)[8], uint32_t byte, uint64_t index, uint32_t which, uint32_t stream_id,
                                            const PhiloxKeys& keys)
{
    uint32_t c[8];
    if constexpr (RANDOM) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t block = index / 4 + h;
            const uint4 r = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), which, stream_id, keys);
            c[4 * h] = act8_code_random(v[4 * h], byte, r.x);
            c[4 * h + 1] = act8_code_random(v[4 * h + 1], byte, r.y);
            c[4 * h + 2] = act8_code_random(v[4 * h + 2], byte, r.z);
            c[4 * h + 3] = act8_code_random(v[4 * h + 3], byte, r.w);
        }
    } else if (byte >= kAct8MaxByte) {  // seldom
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = act8_code(v[i], byte);
    } else {
        const float inv = act8_inverse_unit(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__fmaf_rn(v[i], inv, 12582912.f));
    }
    return pack_codes(c);
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t max_abs_bits(const float (&v)[8])
{
    uint32_t m = abs_bits(v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

// The same of eight values as they lie in memory: magnitudes of 16-bit types compare as whole numbers, two at a time.
__device__ __forceinline__ uint32_t max_abs_bits(const Raw8<float>& r)
{
    const uint32_t k = 0x7fffffffu;
    return max(max(max(r.a.x & k, r.a.y & k), max(r.a.z & k, r.a.w & k)), max(max(r.b.x & k, r.b.y & k), max(r.b.z & k, r.b.w & k)));
}
__device__ __forceinline__ uint32_t max_abs_16(const uint4& a)
{
    const uint32_t k = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(a.x & k, a.y & k), __vmaxu2(a.z & k, a.w & k));
    return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ uint32_t max_abs_bits(const Raw8<__nv_bfloat16>& r) { return max_abs_16(r.a) << 16; }
__device__ __forceinline__ uint32_t max_abs_bits(const Raw8<__half>& r)
{
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)max_abs_16(r.a))));
}

// Values of eight codes: byte u = code + 128 as the low mantissa bits of 2^23, less 2^23 + 128, is exact.
__device__ __forceinline__ void act8_values(uint2 c, float unit, float (&v)[8])
{
    const uint32_t w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = __fmul_rn(__fsub_rn(__uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7650 | (i & 3))), 8388736.f), unit);
}

// ---------------------------------------------------------------------------
// Activation functions.  ACCURATE (fp32 activations) or for results that are rounded to 8 or 11 bits, with the hardware's approximate exponential and
// reciprocal (2^-22 and 2^-23; the argument's rounding adds |z| 2^-24).
// Phi, the normal distribution function, from 1 - Phi(|z|) = erfc(|z| / sqrt 2) / 2:
//   ACCURATE: the Chebyshev fit in Press et al., Numerical Recipes, section 6.2, erfc(x) = t exp(-x^2 + p(t)), t = 1 / (1 + x / 2), p of
//   degree 9, off by at most 1.2e-7 of the value, far tails included, and z^2 2^-23 from the rounding of the exponential's argument.  (CUDA's erfcf and expf: 54 us
//   for the forward pass of group norm with GELU on 16.8 M fp32 values that is bound by memory at 30.)
//   Otherwise: exp(-z^2/2) (a1 t + ... + a7 t^7), t = 1 / (1 + p |z|), the a's and p of least largest error of exp(z^2/2) (1 - Phi) over |z| <= 13.5 (a linear
//   program at 3,000 places), relative and allowed to grow with exp(z^2/4) up to ten times: 1.7e-7 of the value off at 0, 1.7e-6 at most.  It shares its exponential with
//   the density in the slope.  (A fit of five terms bounded in its absolute error only, Abramowitz and Stegun 7.1.26, was 1.6e-3 of the value off at -5, near bf16's half
//   step of 2e-3, and 5e-4, fp16's, at -4; it takes one instruction less in the slope alone and two elsewhere.)
// ---------------------------------------------------------------------------
__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504f;

// 1 / (1 + exp(-z)), and one less that in `rest`.  ACCURATE: what rounding z log2(e) takes from ex2's argument is made up for (without that f(z) was 3.8e-6 of itself
// off at z = -80), and the rest comes from the exponential, so that it is not a difference.  From z = 128 on exp(-z) is 0, where it or its correction overflow it is
// 2^127, whose reciprocal is 0.  (expf and a reciprocal to nearest: 4 x 16384 x 256 with SiLU, forward and backward, 131 us; so 113 us; neither 112.)
template <bool ACCURATE>
__device__ __forceinline__ float sigmoid(float z, float& rest)
{
    if constexpr (ACCURATE) {
        const float c = fminf(z, 128.f), h = __fmul_rn(c, -kLog2e);
        const float l = __fmaf_rn(c, -1.92596299e-8f, __fmaf_rn(c, -kLog2e, -h));  // log2(e) less kLog2e
        const float p = fast_exp2(h);
        const float e = fminf(__fmaf_rn(p, __fmul_rn(l, 0.693147181f), p), 0x1p127f);
        const float s = fast_reciprocal(__fadd_rn(1.f, e));
        rest = __fmul_rn(e, s);
        return s;
    } else {
        const float s = fast_reciprocal(__fadd_rn(1.f, fast_exp2(__fmul_rn(z, -kLog2e))));
        rest = __fsub_rn(1.f, s);
        return s;
    }
}

// 1 - Phi(|z|) over e = exp(-z^2/2), the fit of 16-bit types
__device__ __forceinline__ float normal_tail_over_e(float z)
{
    const float t = fast_reciprocal(__fmaf_rn(fabsf(z), 0.259f, 1.f));
    float p = __fmaf_rn(t, -0.0753390088f, 0.241071129f);
    p = __fmaf_rn(p, t, -0.122635168f);
    p = __fmaf_rn(p, t, 0.177393909f);
    p = __fmaf_rn(p, t, 0.0688966541f);
    p = __fmaf_rn(p, t, 0.107552936f);
    p = __fmaf_rn(p, t, 0.103059548f);
    return __fmul_rn(p, t);
}
__device__ __forceinline__ float normal_e(float z) { return fast_exp2(__fmul_rn(__fmul_rn(z, -0.5f * kLog2e), z)); }
constexpr float kDensity = 0.39894228040143268f;  // 1 / sqrt(2 pi)

// Phi(z), and exp(-z^2/2) in e
template <bool ACCURATE>
__device__ __forceinline__ float normal_cdf(float z, float& e)
{
    e = normal_e(z);
    float tail;
    if constexpr (ACCURATE) {
        const float x = fabsf(z) * 0.70710678118654752f;
        const float t = fast_reciprocal(__fmaf_rn(x, 0.5f, 1.f));
        float p = __fmaf_rn(t, 0.17087277f, -0.82215223f);
        p = __fmaf_rn(p, t, 1.48851587f);
        p = __fmaf_rn(p, t, -1.13520398f);
        p = __fmaf_rn(p, t, 0.27886807f);
        p = __fmaf_rn(p, t, -0.18628806f);
        p = __fmaf_rn(p, t, 0.09678418f);
        p = __fmaf_rn(p, t, 0.37409196f);
        p = __fmaf_rn(p, t, 1.00002368f);
        p = __fmaf_rn(p, t, -1.26551223f);
        tail = __fmul_rn(0.5f * t, fast_exp2(__fmul_rn(__fmaf_rn(-x, x, p), kLog2e)));
    } else {
        tail = __fmul_rn(normal_tail_over_e(z), e);
    }
    return z < 0.f ? tail : __fsub_rn(1.f, tail);
}

// f(z), and its slope in s
template <int ACT, bool ACCURATE>
__device__ __forceinline__ float act_value(float z)
{
    if constexpr (ACT == OGQ_ACT_RELU) return z > 0.f ? z : z == z ? 0.f : z;
    if constexpr (ACT == OGQ_ACT_SILU) {
        float rest;
        return __fmul_rn(z, sigmoid<ACCURATE>(z, rest));
    }
    if constexpr (ACT == OGQ_ACT_GELU) {
        float e;
        return z * normal_cdf<ACCURATE>(z, e);
    }
    return z;
}

template <int ACT, bool ACCURATE>
__device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == OGQ_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
    if constexpr (ACT == OGQ_ACT_SILU) {
        float rest;
        const float s = sigmoid<ACCURATE>(z, rest);
        return __fmaf_rn(__fmul_rn(z, s), rest, s);  // (s + t - t s, t = z s, would be 0 where s + t is rounded to t, from 2^24 on)
    }
    if constexpr (ACT == OGQ_ACT_GELU) {
        if constexpr (ACCURATE) {
            float e;
            const float p = normal_cdf<true>(z, e);
            return __fmaf_rn(z * kDensity, e, p);
        } else {  // Phi and z times the density have the same exponential
            const float t = __fmul_rn(__fmaf_rn(fabsf(z), -kDensity, normal_tail_over_e(z)), normal_e(z));
            return z < 0.f ? t : __fsub_rn(1.f, t);
        }
    }
    return 1.f;
}

// Both at once (the backward pass of a gate needs them).
template <int ACT, bool ACCURATE>
__device__ __forceinline__ float act_both(float z, float& slope)
{
    if constexpr (ACT == OGQ_ACT_SILU) {
        float rest;
        const float s = sigmoid<ACCURATE>(z, rest), t = __fmul_rn(z, s);
        slope = __fmaf_rn(t, rest, s);
        return t;
    }
    if constexpr (ACT == OGQ_ACT_GELU) {
        float e;
        const float p = normal_cdf<ACCURATE>(z, e);
        slope = __fmaf_rn(z * kDensity, e, p);
        return z * p;
    }
    slope = act_slope<ACT, ACCURATE>(z);
    return act_value<ACT, ACCURATE>(z);
}

constexpr int kAct8Ctas = 16;  // per SM, at most, of the kernels that stream a matrix

// g / d = hi(g * mul) >> shift for every g below 2^31 and d of 2 and more (d = 1 is not divided by).
inline void act8_divisor(uint32_t d, uint32_t& mul, uint32_t& shift)
{
    mul = shift = 0;
    if (d < 2) return;
    shift = 0;
    while ((2u << shift) < d) ++shift;  // 2^shift < d <= 2^(shift+1)
    mul = (uint32_t)((((uint64_t)1 << (32 + shift)) + d - 1) / d);
}

// The row of group g.
template <class A>
__device__ __forceinline__ uint32_t act8_row(const A& a, uint32_t g)
{
    return a.groups == a.all_groups ? 0u : a.groups == 1 ? g : __umulhi(g, a.div_mul) >> a.div_shift;
}

// Calls f(std::integral_constant) for a run-time choice.
template <class F>
inline cudaError_t with_act(int act, F f)
{
    switch (act) {
        case OGQ_ACT_NONE: return f(std::integral_constant<int, OGQ_ACT_NONE>{});
        case OGQ_ACT_RELU: return f(std::integral_constant<int, OGQ_ACT_RELU>{});
        case OGQ_ACT_SILU: return f(std::integral_constant<int, OGQ_ACT_SILU>{});
        default: return f(std::integral_constant<int, OGQ_ACT_GELU>{});
    }
}
template <class F>
inline cudaError_t with_dtype(int dtype, F f)
{
    switch (dtype) {
        case OGQ_F32: return f(float{});
        case OGQ_F16: return f(__half{});
        default: return f(__nv_bfloat16{});
    }
}
template <class F>
inline cudaError_t with_bool(bool b, F f)
{
    return b ? f(std::true_type{}) : f(std::false_type{});
}

}  // namespace ogq
