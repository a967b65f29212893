// Device arithmetic of the dense and gated layers: 16-bit values, activations
// and their slopes, and the 8-bit checkpoint code.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "../../include/emtk.h"

namespace emtk {
namespace {

template <bool F16>
__device__ __forceinline__ float from16(uint32_t h) {
    if (F16) return __half2float(__ushort_as_half((unsigned short)h));
    return __uint_as_float(h << 16);
}
template <bool F16>
__device__ __forceinline__ uint32_t to16(float v) {
    if (F16) return __half_as_ushort(__float2half_rn(v));
    return __bfloat16_as_ushort(__float2bfloat16_rn(v));
}
// Two values in one word, lo in the low half.
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t d;
    if (F16)
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// exp(z) and 1 / v with flushed subnormals; exp overflows to infinity, whose
// reciprocal is 0.  The reciprocal is good to 1 ulp, the power of two to 2; the product
// z log2(e) is rounded before it, which makes exp off by up to |z| 2^-24 of itself more.
__device__ __forceinline__ float exp_f(float z) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(z * 1.4426950408889634f));
    return r;
}
__device__ __forceinline__ float reciprocal_f(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// 1 / (1 + exp(-z)): 0 where exp(-z) overflows (z < -88), the limit.
__device__ __forceinline__ float sigmoid_f(float z) { return reciprocal_f(1.f + exp_f(-z)); }

// The normal distribution function and e = exp(-z^2 / 2), which is both the tail of the
// one and the derivative's density: 1 - Phi(|z|) = e t (c0 + t (c1 + ..)) with
// t = 1 / (1 + p |z|).  p and the coefficients are a fit to the smallest largest relative
// error for |z| <= 13.5 (least squares in 64 bits, reweighted until level: 8.3e-8), beyond
// which e is 0.  In fp32, for z < 0: 6e-7 of the value to z = -2, 2e-6 to -6 and 8e-6 to
// -12, where the exponent's rounding shows; for z > 0 half an ulp of 1 more.
__device__ __forceinline__ void normal_f(float z, float &phi, float &e) {
    const float t = reciprocal_f(fmaf(fabsf(z), 0.30400993f, 1.f));
    e = exp_f(-0.5f * z * z);
    float s = fmaf(t, 0.03686058f, -0.15529062f);
    s = fmaf(t, s, 0.19214864f);
    s = fmaf(t, s, -0.043099944f);
    s = fmaf(t, s, 0.1235393f);
    s = fmaf(t, s, 0.10242923f);
    s = fmaf(t, s, 0.122174196f);
    s = fmaf(t, s, 0.12123867f);
    s = t * s * e;
    phi = z < 0.f ? s : 1.f - s;
}

template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == EMTK_ACT_RELU) return z > 0.f ? z : (z == z ? 0.f : z);  // NaN stays
    if (ACT == EMTK_ACT_GELU) {
        float phi, e;
        normal_f(z, phi, e);
        return z * phi;
    }
    if (ACT == EMTK_ACT_SILU) return z * sigmoid_f(z);
    if (ACT == EMTK_ACT_SIGMOID) return sigmoid_f(z);
    return z;
}

// act(z) and act'(z), which share their transcendental.
template <int ACT>
__device__ __forceinline__ void act_slope(float z, float &a, float &d) {
    a = z;
    d = 1.f;
    if (ACT == EMTK_ACT_RELU) {
        a = act_of<ACT>(z);
        d = z > 0.f ? 1.f : (z == z ? 0.f : z);
    } else if (ACT == EMTK_ACT_GELU) {
        float phi, e;
        normal_f(z, phi, e);
        a = z * phi;
        d = fmaf(z * 0.39894228f, e, phi);
    } else if (ACT == EMTK_ACT_SILU) {
        const float p = sigmoid_f(z);
        a = z * p;
        d = p * (1.f + z * (1.f - p));
    } else if (ACT == EMTK_ACT_SIGMOID) {
        const float p = sigmoid_f(z);
        a = p;
        d = p * (1.f - p);
    }
}

// act of every element, the choice made once.
template <int N>
__device__ __forceinline__ void apply_act(int act, float (&v)[N]) {
    switch (act) {
#define EMTK_ACT_CASE(A)                                      \
    case A: {                                                 \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = act_of<A>(v[i]); \
        break;                                                \
    }
        EMTK_ACT_CASE(EMTK_ACT_RELU)
        EMTK_ACT_CASE(EMTK_ACT_GELU)
        EMTK_ACT_CASE(EMTK_ACT_SILU)
        EMTK_ACT_CASE(EMTK_ACT_SIGMOID)
#undef EMTK_ACT_CASE
        default: break;
    }
}

// ---- slopes held in fp16 for the products of a backward call
// Power of two by which they are stored, from the bits of the largest finite |dz| (or
// |dg| and |du|): 1 where fp16 holds that to full precision with room below it (an
// element is off by 2^-25 beside its rounding: 2^-19 of the largest or less), or it is 0.
// Else the larger is brought to 2^14 .. 2^15, as far as the power and its inverse are
// normal numbers.
__device__ __forceinline__ float slope_scale(uint32_t peak0, uint32_t peak1) {
    const uint32_t low = __float_as_uint(0.015625f), high = __float_as_uint(65504.f);
    if ((peak0 == 0u || (peak0 >= low && peak0 <= high)) && (peak1 == 0u || (peak1 >= low && peak1 <= high))) return 1.f;
    return __uint_as_float(min(127u + 14u + 127u - (max(peak0, peak1) >> 23), 127u + 112u) << 23);
}
// 1 / slope_scale.
__device__ __forceinline__ float slope_unscale(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }

// ---- 8-bit checkpoints (emtk_matrix in include/emtk.h)
// Scale byte of a block whose largest finite magnitude is `top`: with
// 2^(byte - 127) <= top / 64 < 2^(byte - 126) the quotient is in [64, 128);
// from 127.5 on (mantissa bits 0x7f0000 and up) it would round to 128, so
// those take the next power: adding 0x10000 carries exactly there.
__device__ __forceinline__ uint32_t q8_scale(float top) {
    const int b = (int)((__float_as_uint(top) + 0x10000u) >> 23) - 6;
    return (uint32_t)max(b, 1);
}
__device__ __forceinline__ float q8_step(uint32_t b) { return __uint_as_float(b << 23); }         // 2^(b - 127)
__device__ __forceinline__ float q8_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }  // b <= 249

// The largest finite magnitude of N values, and whether any is not finite: v * 0
// is NaN exactly then, and stays NaN in the sum.
template <int N>
__device__ __forceinline__ float finite_top(const float (&v)[N], bool &all_finite) {
    float top = 0.f, zero = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        top = fmaxf(top, fabsf(v[i]));
        zero = fmaf(v[i], 0.f, zero);
    }
    all_finite = zero == 0.f;
    if (!all_finite) {  // rare
        top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]) < __int_as_float(0x7f800000) ? fabsf(v[i]) : 0.f);
    }
    return top;
}
// Codes of four values in one word.  Adding 1.5 * 2^23 rounds v / step (at most
// 127 in magnitude) to a whole number, ties to even, in the low mantissa bits:
// the quotient by a power of two is exact and the addition rounds once.
__device__ __forceinline__ uint32_t q8_codes4(const float *v, float inverse, bool all_finite) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(fmaf(v[i], inverse, 12582912.f));
    uint32_t w = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    if (!all_finite) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!(fabsf(v[i]) < __int_as_float(0x7f800000))) w = (w & ~(0xffu << (8 * i))) | (0x80u << (8 * i));
    }
    return w;
}
// Two sums or products at once.
__device__ __forceinline__ void add_mul2(float &a, float &b, float add, float mul) {
    uint64_t v, t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("mov.b64 %0, {%1, %1};" : "=l"(t) : "f"(add));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(t));
    asm("mov.b64 %0, {%1, %1};" : "=l"(t) : "f"(mul));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(t));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
// Values of the four codes of a word.  A byte with its sign bit flipped is code +
// 128; below the bits of 2^23 it is 2^23 + 128 + code, from which a subtraction and
// a product by the power of two leave the value, both exact.  Returns not 0 if some
// code is -128 (read as a number here).
__device__ __forceinline__ uint32_t q8_values4_finite(uint32_t w, float step, float *v) {
    const uint32_t x = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7440 + i));
    add_mul2(v[0], v[1], -8388736.f, step);
    add_mul2(v[2], v[3], -8388736.f, step);
    return (x - 0x01010101u) & ~x & 0x80808080u;  // some byte of x is 0
}
__device__ __forceinline__ void q8_values4(uint32_t w, float step, float *v) {
    if (q8_values4_finite(w, step, v)) {  // rare
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (((w >> (8 * i)) & 0xffu) == 0x80u) v[i] = __int_as_float(0x7fffffff);
    }
}
// The value as an operand of the products: bf16 holds it exactly, fp16 saturates.
template <bool F16>
__device__ __forceinline__ float q8_operand(float v) {
    if (!F16) return v;
    return fabsf(v) > 65504.f ? copysignf(65504.f, v) : v;  // NaN compares false and stays
}

}  // namespace
}  // namespace emtk
