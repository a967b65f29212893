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

// 1 / (1 + exp(-z)): 0 where exp(-z) overflows (z < -88), the limit.
__device__ __forceinline__ float sigmoid_f(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

__device__ __forceinline__ float act_f(int act, float z) {
    switch (act) {
        case EMTK_ACT_RELU: return z > 0.f ? z : (z == z ? 0.f : z);  // NaN stays
        case EMTK_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case EMTK_ACT_SILU: return z * sigmoid_f(z);
        case EMTK_ACT_SIGMOID: return sigmoid_f(z);
        default: return z;
    }
}

// act(z) and act'(z), which share their transcendental.
__device__ __forceinline__ void act_slope(int act, float z, float &a, float &d) {
    switch (act) {
        case EMTK_ACT_RELU:
            a = z > 0.f ? z : (z == z ? 0.f : z);
            d = z > 0.f ? 1.f : (z == z ? 0.f : z);
            break;
        case EMTK_ACT_GELU: {
            const float p = 0.5f * (1.f + erff(z * 0.70710678118654752f));
            a = z * p;
            d = p + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
            break;
        }
        case EMTK_ACT_SILU: {
            const float p = sigmoid_f(z);
            a = z * p;
            d = p * (1.f + z * (1.f - p));
            break;
        }
        case EMTK_ACT_SIGMOID: {
            const float p = sigmoid_f(z);
            a = p;
            d = p * (1.f - p);
            break;
        }
        default: a = z; d = 1.f;
    }
}

// ---- 8-bit checkpoints (emtk_matrix in include/emtk.h)
// |v| if finite, else 0: what the block maximum is taken over.
__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a < __int_as_float(0x7f800000) ? a : 0.f;
}
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
__device__ __forceinline__ uint32_t q8_code(float v, float inverse) {
    const uint32_t q = (uint32_t)__float2int_rn(v * inverse) & 0xffu;
    return fabsf(v) < __int_as_float(0x7f800000) ? q : 0x80u;
}
__device__ __forceinline__ float q8_value(uint32_t byte, float step) {
    const int q = (int)(int8_t)byte;
    return q == -128 ? __int_as_float(0x7fffffff) : (float)q * step;
}
// The value as an operand of the products: bf16 holds it exactly, fp16 saturates.
template <bool F16>
__device__ __forceinline__ float q8_operand(float v) {
    if (!F16) return v;
    return fabsf(v) > 65504.f ? copysignf(65504.f, v) : v;  // NaN compares false and stays
}

}  // namespace
}  // namespace emtk
