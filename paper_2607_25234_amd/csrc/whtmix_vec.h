// Device helpers of the feed-forward sublayer's kernels: 16-byte accesses of
// float32 and bf16 rows, block-scaled 8-bit rounding, activations.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "whtmix_layer.h"

namespace whtmix {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// Two floats as bf16, rounded to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, b2));
}

// Rows are moved in chunks of 16 bytes: Chunk<T>::N elements.  Rows of any
// width start at any multiple of the element's size, so accesses carry only the
// element's alignment (global accesses of the hardware need no more); the last
// chunk of a row, of fewer elements, is moved element by element.
template <typename T> struct Chunk;

template <> struct Chunk<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void load(const float *p, int n, float (&v)[4])
    {
        if (n >= 4) {
            __builtin_memcpy(v, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : 0.f;
        }
    }
    static __device__ __forceinline__ void store(float *p, int n, const float (&v)[4])
    {
        if (n >= 4) {
            __builtin_memcpy(p, v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) p[i] = v[i];
        }
    }
};

template <> struct Chunk<__bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void load(const __bf16 *p, int n, float (&v)[8])
    {
        if (n >= 8) {
            uint32_t u[4];
            __builtin_memcpy(u, p, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bits_f32(u[i] << 16);
                v[2 * i + 1] = bits_f32(u[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.f;
        }
    }
    static __device__ __forceinline__ void store(__bf16 *p, int n, const float (&v)[8])
    {
        if (n >= 8) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(p, u, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = (__bf16)v[i];
        }
    }
};

// The value of the lane whose number differs in bit 0 or 1 (within a quad, no LDS).
template <int BIT> __device__ __forceinline__ uint32_t quad_xor(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, BIT == 0 ? 0xB1 : 0x4E, 0xf, 0xf, true);
}

// ---- block-scaled 8 bits ----
// Magnitude of a finite value as ordered bits; 0 for Inf and NaN, which do not
// count for a block's scale (they are stored as e4m3's NaN).
__device__ __forceinline__ uint32_t mx_magnitude(float v)
{
    const uint32_t b = f32_bits(v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// The scale's byte for a block whose largest magnitude has the bits `top`:
// the least e with top <= 448 * 2^e, 448 = 1.75 * 2^8 being e4m3's largest
// value, in [-126, 120] so that 2^e and 2^-e are both normal.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top)
{
    const int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(min(max(e, -126), 120) + 127);
}

__device__ __forceinline__ float mx_inverse(uint32_t byte) { return bits_f32((254u - byte) << 23); }

// Four values as e4m3, rounded to nearest even; inv = 2^-e makes the product
// exact.  Inf and NaN become NaN.
__device__ __forceinline__ uint32_t mx_pack(float a, float b, float c, float d, float inv)
{
    const float nan = bits_f32(0x7fc00000u);
    auto fin = [&](float v) { return (f32_bits(v) & 0x7f800000u) != 0x7f800000u ? v * inv : nan; };
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(fin(a), fin(b), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(fin(c), fin(d), r, true);
    return (uint32_t)r;
}

// ---- activations ----
__device__ __forceinline__ float fast_exp(float x)   // 2^(x log2 e), about 2 ulp + |x| 2^-24
{
    return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
}

// (1 - erf(|z| / sqrt 2)) / 2, the gaussian's tail beyond |z|, by Abramowitz & Stegun
// 7.1.26 (erf off by 1.5e-7 at most), with e = exp(-z^2 / 2), which the density shares.
__device__ __forceinline__ float gauss_tail(float z, float e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
    float p = fmaf(0.5f * 1.061405429f, t, -0.5f * 1.453152027f);
    p = fmaf(p, t, 0.5f * 1.421413741f);
    p = fmaf(p, t, -0.5f * 0.284496736f);
    p = fmaf(p, t, 0.5f * 0.254829592f);
    return p * t * e;
}
__device__ __forceinline__ float gauss(float z)      // exp(-z^2 / 2)
{
    return __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.44269504088896341f));
}

// z * sigmoid(u): 0 for u = -Inf with z finite, NaN for z = -Inf as the formula.
__device__ __forceinline__ float gated(float z, float u)
{
    return z * __builtin_amdgcn_rcpf(1.f + fast_exp(-u));
}

constexpr float kGeluC = 1.5957691216057308f;     // 2 sqrt(2 / pi): tanh(a) = 2 sigmoid(2a) - 1

template <int ACT> __device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == ACT_RELU) return z > 0.f || z != z ? z : 0.f;
    // z for z > 0, less |z| times the tail (which is 0 long before 64: no Inf * 0)
    if constexpr (ACT == ACT_GELU)
        return fmaf(-fminf(fabsf(z), 64.f), gauss_tail(z, gauss(z)), fmaxf(z, 0.f));
    if constexpr (ACT == ACT_GELU_TANH)
        return gated(z, kGeluC * z * fmaf(0.044715f * z, z, 1.f));
    if constexpr (ACT == ACT_SILU) return gated(z, z);
    return z;
}

template <int ACT> __device__ __forceinline__ float act_grad(float z)
{
    if constexpr (ACT == ACT_RELU) return z > 0.f ? 1.f : z != z ? z : 0.f;
    if constexpr (ACT == ACT_GELU) {
        const float e = gauss(z), q = gauss_tail(z, e);
        return fmaf(fminf(fmaxf(z, -64.f), 64.f) * 0.39894228040143268f, e, z < 0.f ? q : 1.f - q);
    }
    if constexpr (ACT == ACT_GELU_TANH) {
        const float s = __builtin_amdgcn_rcpf(
            1.f + fast_exp(-kGeluC * z * fmaf(0.044715f * z, z, 1.f)));
        // beyond 64, where s (1 - s) is 0, the square would overflow: no 0 * Inf
        const float c = fminf(fmaxf(z, -64.f), 64.f);
        return fmaf(c * s * (1.f - s), kGeluC * fmaf(0.134145f * c, c, 1.f), s);
    }
    if constexpr (ACT == ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + fast_exp(-z));
        return fmaf(z * s, 1.f - s, s);
    }
    return 1.f;
}

// Both at once, by the same operations: the exponential and the reciprocal are shared.
template <int ACT> __device__ __forceinline__ void act_both(float z, float &a, float &da)
{
    if constexpr (ACT == ACT_GELU) {
        const float e = gauss(z), q = gauss_tail(z, e);
        a = fmaf(-fminf(fabsf(z), 64.f), q, fmaxf(z, 0.f));
        da = fmaf(fminf(fmaxf(z, -64.f), 64.f) * 0.39894228040143268f, e, z < 0.f ? q : 1.f - q);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        const float s = __builtin_amdgcn_rcpf(
            1.f + fast_exp(-kGeluC * z * fmaf(0.044715f * z, z, 1.f)));
        const float c = fminf(fmaxf(z, -64.f), 64.f);
        a = z * s;
        da = fmaf(c * s * (1.f - s), kGeluC * fmaf(0.134145f * c, c, 1.f), s);
    } else if constexpr (ACT == ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + fast_exp(-z));
        a = z * s;
        da = fmaf(a, 1.f - s, s);
    } else {
        a = act_of<ACT>(z);
        da = act_grad<ACT>(z);
    }
}

// f<ACT>() for the run-time activation (uniform over the grid).
template <typename F> __device__ __forceinline__ void with_act(int act, F f)
{
    switch (act) {
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>{}); break;
    case ACT_GELU: f(std::integral_constant<int, ACT_GELU>{}); break;
    case ACT_GELU_TANH: f(std::integral_constant<int, ACT_GELU_TANH>{}); break;
    case ACT_SILU: f(std::integral_constant<int, ACT_SILU>{}); break;
    default: f(std::integral_constant<int, ACT_NONE>{}); break;
    }
}

}  // namespace whtmix
