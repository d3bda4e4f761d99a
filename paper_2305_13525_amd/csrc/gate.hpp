// The activations of a gated block, in fp32.
#pragma once
#include <type_traits>

#include "axo_common.hpp"

namespace axo {

// v sigmoid(v): one exp2 and one reciprocal, as gelu_tanh.  Below v = -87 exp(-v) passes 2^126 and the result is zero (it is smaller than 2^-119).
__device__ __forceinline__ float silu(float v) {
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
}
template <int GATE>
__device__ __forceinline__ float gate_value(float v) {
    return GATE == GATE_SILU ? silu(v) : GATE == GATE_GELU_TANH ? gelu_tanh(v) : gelu_erf(v);
}
// The value and its derivative.
template <int GATE>
__device__ __forceinline__ float2 gate_both(float v) {
    if (GATE == GATE_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
        return float2{v * s, s * __builtin_fmaf(v, 1.0f - s, 1.0f)};
    }
    // beyond 16 the derivative is that of 16 (1 or 0, and nothing overflows on the way); NaN stays NaN
    if (GATE == GATE_GELU_TANH) return float2{gelu_tanh(v), dgelu_tanh(v > 16.0f ? 16.0f : v < -16.0f ? -16.0f : v)};
    return float2{gelu_erf(v), dgelu_erf(v)};
}

// f of the gate as a compile-time constant.
template <typename F>
__device__ __forceinline__ void with_gate(int gate, F f) {
    if (gate == GATE_SILU) f(std::integral_constant<int, GATE_SILU>{});
    else if (gate == GATE_GELU_TANH) f(std::integral_constant<int, GATE_GELU_TANH>{});
    else f(std::integral_constant<int, GATE_GELU_ERF>{});
}

}  // namespace axo
