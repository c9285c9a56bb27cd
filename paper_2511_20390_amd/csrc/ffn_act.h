// The activations of the gated feed-forward block and their derivatives.  Device code.
#pragma once

#include "free_internal.h"

namespace freemi {

namespace {

// act(v), act'(v) with the hardware's exponential and reciprocal (1 ulp each): both activations are v s with s = 1 / (1 + 2^-t),
// t = v log2(e) for SiLU and v (a + b v^2) for the tanh form of GELU
__device__ __forceinline__ void act_fast(float v, int act, float* f, float* df) {
    constexpr float kLog2e = 1.4426950408889634f, kA = 2.0f * 0.7978845608028654f, kB = kA * 0.044715f;
    const float v2 = v * v;
    const float t = act == FREE_ACT_SILU ? -v * kLog2e : -v * fmaf(v2, kB * kLog2e, kA * kLog2e);
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
    const float slope = act == FREE_ACT_SILU ? v : v * fmaf(v2, 3.0f * kB, kA);      // v dt / dv
    *f = v * s;
    // s (1 - s): where slope is infinite s is 0 or 1 exactly
    *df = s == 0.f || s == 1.f ? s : fmaf(s * (1.0f - s), slope, s);
}

// fp32: the library's exponential and tanh in place of the hardware's
__device__ __forceinline__ void act_exact(float v, int act, float* f, float* df) {
    if (act == FREE_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-v));
        *f = v * s;
        *df = s == 0.f || s == 1.f ? s : s * (1.0f + v * (1.0f - s));
    } else {
        const float k = 0.7978845608028654f;
        const float v2 = v * v, t = tanhf(k * (v + 0.044715f * v2 * v));
        *f = 0.5f * v * (1.0f + t);
        // (1 - t^2) times what grows with v^3: 0 where t is one to the last bit
        *df = fabsf(t) == 1.f ? 0.5f * (1.0f + t) : 0.5f * (1.0f + t) + 0.5f * v * (1.0f - t * t) * k * (1.0f + 3.0f * 0.044715f * v2);
    }
}

}  // namespace
}  // namespace freemi
