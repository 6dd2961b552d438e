// Activations of the dense operators and their derivatives in fp32, and 16-bit values to fp32 and back.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "../../include/dlfusion.h"

namespace dlf {

__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values rounded, the first one in the lower half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }

// Two values at a time: sums and products of pairs are single instructions.
__device__ __forceinline__ unsigned long long pair_bits(float2 v) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 pair_of(unsigned long long r) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
    return v;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// 2^v and 1 / v to 2^-22, without the scaling that subnormal values would need (2^v below 2^-126 is 0, and so is 1 / v above 2^126).
__device__ __forceinline__ float2 exp2_2(float2 v) {
    float2 r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(v.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 rcp2(float2 v) {
    float2 r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(v.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(v.y));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float2 sigmoid2(float2 v) { return rcp2(add2(exp2_2(mul2(v, both(-kLog2e))), both(1.0f))); }   // 1 / (1 + e^-v)

constexpr float kGeluC = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// The normal distribution's density at v and its integral up to v.  The integral up to -a is e^(-a^2 / 2) t Q(t) with t = 1 / (1 + 0.306 a), Q
// the polynomial of degree 7 with the least largest relative error over a from 0 to 15, 1.1e-7 (fitted by reweighted least squares): it
// shares its exponential with the density, and is as exact in the tail, where it is small, as in the middle (with the exponential's
// argument rounded, 6e-7 of the value down to -3, 2e-6 to -6, 8e-6 to -13).
__device__ __forceinline__ void normal2(float2 v, float2* density, float2* integral) {
    const float2 a = make_float2(fabsf(v.x), fabsf(v.y));
    const float2 e = exp2_2(mul2(mul2(v, v), both(-0.5f * kLog2e)));
    const float2 t = rcp2(fma2(a, both(0.306f), both(1.0f)));
    float2 s = fma2(t, both(0.03653757f), both(-0.15069884f));
    s = fma2(t, s, both(0.17938326f));
    s = fma2(t, s, both(-0.033034489f));
    s = fma2(t, s, both(0.11862855f));
    s = fma2(t, s, both(0.104367666f));
    s = fma2(t, s, both(0.12277222f));
    s = fma2(t, s, both(0.1220441f));
    const float2 tail = mul2(mul2(t, e), s), rest = fma2(tail, both(-1.0f), both(1.0f));
    *integral = make_float2(v.x < 0.0f ? tail.x : rest.x, v.y < 0.0f ? tail.y : rest.y);
    *density = mul2(e, both(0.3989422804014327f));
}

// act(v).  GELU by tanh: v (1 + tanh(t)) / 2 = v sigmoid(2 t) with t = c (v + a v^3).  A NaN is 0 behind ReLU and ReLU6, as in the
// other kernels.
template <int ACT>
__device__ __forceinline__ float2 act2(float2 v) {
    if (ACT == DLF_ACT_RELU) return make_float2(fmaxf(v.x, 0.0f), fmaxf(v.y, 0.0f));
    if (ACT == DLF_ACT_RELU6) return make_float2(fminf(fmaxf(v.x, 0.0f), 6.0f), fminf(fmaxf(v.y, 0.0f), 6.0f));
    if (ACT == DLF_ACT_GELU) {
        float2 density, integral;
        normal2(v, &density, &integral);
        return mul2(v, integral);
    }
    if (ACT == DLF_ACT_GELU_TANH) return mul2(v, sigmoid2(mul2(v, fma2(mul2(v, v), both(2.0f * kGeluC * kGeluA), both(2.0f * kGeluC)))));
    if (ACT == DLF_ACT_SILU) return mul2(v, sigmoid2(v));
    return v;
}
// act(v) and its derivative (0 at the corners of ReLU and ReLU6).
template <int ACT>
__device__ __forceinline__ void act_grad2(float2 v, float2* value, float2* slope) {
    *value = v;
    *slope = both(1.0f);
    if (ACT == DLF_ACT_RELU) {
        *value = act2<ACT>(v);
        *slope = make_float2(v.x > 0.0f ? 1.0f : 0.0f, v.y > 0.0f ? 1.0f : 0.0f);
    }
    if (ACT == DLF_ACT_RELU6) {
        *value = act2<ACT>(v);
        *slope = make_float2(v.x > 0.0f && v.x < 6.0f ? 1.0f : 0.0f, v.y > 0.0f && v.y < 6.0f ? 1.0f : 0.0f);
    }
    if (ACT == DLF_ACT_GELU) {
        float2 density, integral;
        normal2(v, &density, &integral);
        *value = mul2(v, integral);
        *slope = fma2(v, density, integral);
    }
    if (ACT == DLF_ACT_GELU_TANH || ACT == DLF_ACT_SILU) {
        // v s(t), s the sigmoid: s + v s (1 - s) t'.  (Beyond 16 the sigmoid of GELU_TANH is 0 or 1, and v^2 need not be finite.)
        const float2 c = ACT == DLF_ACT_SILU ? v : make_float2(fminf(fmaxf(v.x, -16.0f), 16.0f), fminf(fmaxf(v.y, -16.0f), 16.0f)), q = mul2(c, c);
        const float2 t = ACT == DLF_ACT_SILU ? v : mul2(c, fma2(q, both(2.0f * kGeluC * kGeluA), both(2.0f * kGeluC)));
        const float2 s = sigmoid2(t), w = fma2(s, both(-1.0f), both(1.0f));
        *value = mul2(v, s);
        const float2 dt = ACT == DLF_ACT_SILU ? w : mul2(w, fma2(q, both(6.0f * kGeluC * kGeluA), both(2.0f * kGeluC)));
        *slope = fma2(*value, dt, s);
    }
}
// A gradient behind act: d slope.  At a corner or beyond, ReLU and ReLU6 are constant and nothing comes through: 0 whatever d is, infinities
// and NaN too (as in automatic differentiation; a product would make a NaN of them, and that a row of dx and of dw).
template <int ACT>
__device__ __forceinline__ float2 behind2(float2 d, float2 slope) {
    if (ACT == DLF_ACT_RELU || ACT == DLF_ACT_RELU6) return make_float2(slope.x != 0.0f ? d.x : 0.0f, slope.y != 0.0f ? d.y : 0.0f);
    return mul2(d, slope);
}
template <int ACT>
__device__ __forceinline__ float act_f(float v) { return act2<ACT>(make_float2(v, v)).x; }

// Calls f with the activation as a compile-time constant: one branch for a run of values.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case DLF_ACT_RELU: f(std::integral_constant<int, DLF_ACT_RELU>{}); break;
        case DLF_ACT_RELU6: f(std::integral_constant<int, DLF_ACT_RELU6>{}); break;
        case DLF_ACT_GELU: f(std::integral_constant<int, DLF_ACT_GELU>{}); break;
        case DLF_ACT_GELU_TANH: f(std::integral_constant<int, DLF_ACT_GELU_TANH>{}); break;
        case DLF_ACT_SILU: f(std::integral_constant<int, DLF_ACT_SILU>{}); break;
        default: f(std::integral_constant<int, DLF_ACT_NONE>{}); break;
    }
}

}  // namespace dlf
