// Activations of a linear layer's epilogue (kq_linear.hip, kq_matvec.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kq_linear.h"

namespace kq {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

// act(p).  The exponentials and reciprocals are the hardware's (1 ulp each).
template <Act A>
__device__ __forceinline__ float activate(float p) {
    if (A == Act::Relu) return p <= 0.0f ? 0.0f : p;  // NaN stays NaN, as in the other activations
    if (A == Act::Silu || A == Act::Swiglu) return p * sigmoid(p);
    if (A == Act::GeluTanh) {
        // p (1 + tanh z) / 2 = p sigmoid(2 z), z = sqrt(2 / pi) (p + 0.044715 p^3)
        constexpr float c = -2.0f * kLog2e * 0.797884560802865356f;
        return p * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(p * fmaf(c * 0.044715f, p * p, c)));
    }
    if (A == Act::Gelu) {
        // p Phi(p), Phi(-a) = exp(-a^2 / 2) q(t) with t = 1 / (1 + 0.35 a): the polynomial q is a
        // minimax fit of exp(a^2 / 2) Phi(-a) in relative error, 3.1e-7 for a <= 13.5 (Phi(-a) = 0 beyond)
        const float a = fabsf(p), t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
        float q = 0.048942483961582184f;
        q = fmaf(q, t, -0.20211942493915558f);
        q = fmaf(q, t, 0.2406410276889801f);
        q = fmaf(q, t, -0.01702360063791275f);
        q = fmaf(q, t, 0.1559615582227707f);
        q = fmaf(q, t, 0.13335508108139038f);
        q = fmaf(q, t, 0.14027033746242523f);
        q = fmaf(q, t, -2.731548374867998e-05f);
        q *= __builtin_amdgcn_exp2f(-0.5f * kLog2e * a * a);
        const float m = a >= 13.5f ? 0.0f : p * q;
        return p > 0.0f ? p - m : m;
    }
    return p;
}

// f with the call's activation as a compile-time constant.
template <class F>
__device__ __forceinline__ void with_act(Act a, F f) {
    switch (a) {
        case Act::None: f(std::integral_constant<Act, Act::None>{}); break;
        case Act::Gelu: f(std::integral_constant<Act, Act::Gelu>{}); break;
        case Act::GeluTanh: f(std::integral_constant<Act, Act::GeluTanh>{}); break;
        case Act::Silu: f(std::integral_constant<Act, Act::Silu>{}); break;
        case Act::Relu: f(std::integral_constant<Act, Act::Relu>{}); break;
        case Act::Swiglu: f(std::integral_constant<Act, Act::Swiglu>{}); break;
    }
}

}  // namespace

}  // namespace kq
