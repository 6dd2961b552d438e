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

// 1 / (1 + e^-v).  The quotient's denominator is above 2^126 only where the value is below 2^-126; 0 then.
__device__ __forceinline__ float sigmoid_f(float v) { return __fdividef(1.0f, 1.0f + __expf(-v)); }

constexpr float kGeluC = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// The normal distribution's density at v and its integral up to v: erfc by the rational approximation 7.1.26 of Abramowitz and Stegun,
// "Handbook of Mathematical Functions" (off by at most 1.5e-7, half of that here), which shares its exponential with the density
// and takes a third of the instructions of erff.
__device__ __forceinline__ float2 normal_f(float v) {
    const float a = fabsf(v) * 0.7071067811865476f, e = __expf(-0.5f * v * v), t = __fdividef(1.0f, fmaf(0.3275911f, a, 1.0f));
    const float tail = 0.5f * e * (t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f));
    return make_float2(e * 0.3989422804014327f, v < 0.0f ? tail : 1.0f - tail);
}

// act(v).  GELU by tanh: v (1 + tanh(t)) / 2 = v sigmoid(2 t) with t = c (v + a v^3).  A NaN is 0 behind ReLU and ReLU6, as in the
// other kernels.
template <int ACT>
__device__ __forceinline__ float act_f(float v) {
    if (ACT == DLF_ACT_RELU) return fmaxf(v, 0.0f);
    if (ACT == DLF_ACT_RELU6) return fminf(fmaxf(v, 0.0f), 6.0f);
    if (ACT == DLF_ACT_GELU) return v * normal_f(v).y;
    if (ACT == DLF_ACT_GELU_TANH) return v * sigmoid_f(2.0f * kGeluC * (v + kGeluA * v * v * v));
    if (ACT == DLF_ACT_SILU) return v * sigmoid_f(v);
    return v;
}
// act(v) and its derivative (0 at the corners of ReLU and ReLU6).
template <int ACT>
__device__ __forceinline__ float2 act_grad_f(float v) {
    if (ACT == DLF_ACT_RELU) return make_float2(fmaxf(v, 0.0f), v > 0.0f ? 1.0f : 0.0f);
    if (ACT == DLF_ACT_RELU6) return make_float2(fminf(fmaxf(v, 0.0f), 6.0f), v > 0.0f && v < 6.0f ? 1.0f : 0.0f);
    if (ACT == DLF_ACT_GELU) {
        const float2 n = normal_f(v);
        return make_float2(v * n.y, fmaf(v, n.x, n.y));
    }
    if (ACT == DLF_ACT_GELU_TANH) {
        const float s = sigmoid_f(2.0f * kGeluC * (v + kGeluA * v * v * v));
        return make_float2(v * s, s + v * s * (1.0f - s) * (2.0f * kGeluC * (1.0f + 3.0f * kGeluA * v * v)));
    }
    if (ACT == DLF_ACT_SILU) {
        const float s = sigmoid_f(v);
        return make_float2(v * s, s * (1.0f + v * (1.0f - s)));
    }
    return make_float2(v, 1.0f);
}

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
