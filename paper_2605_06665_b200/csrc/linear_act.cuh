// Activations of the dense products and their derivatives.  kFast: through the special-function unit (errors of a few 2^-22, gelu's slope
// 2^-18, far below the rounding to bf16); otherwise CUDA's expf and divisions.
#pragma once

#include "common.cuh"

namespace unipool {

// 1 / (1 + 2^z)
__device__ __forceinline__ float rcp_1_ex2(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;
template <bool kFast> __device__ __forceinline__ float logistic(float a) {
  if constexpr (kFast) return rcp_1_ex2(-kLog2e * a);
  else return 1.f / (1.f + expf(-a));
}

// gelu (tanh form): 0.5 p (1 + tanh(u)) = p logistic(2 u), u = sqrt(2 / pi) (p + 0.044715 p^3); as a product with the
// logistic function it keeps its relative accuracy where the tanh nears -1.
constexpr float kGeluTwice = 1.5957691216057308f, kGeluCube = 0.044715f;

template <bool kFast> __device__ __forceinline__ float act_value(float p, int act) {
  switch (act) {
    case UNIPOOL_ACT_RELU: return max_nan(p, 0.f);
    case UNIPOOL_ACT_SILU: return p * logistic<kFast>(p);
    case UNIPOOL_ACT_GELU:
      if constexpr (kFast) return p * rcp_1_ex2(p * fmaf(p * p, -kLog2e * kGeluTwice * kGeluCube, -kLog2e * kGeluTwice));
      else return p * logistic<false>(kGeluTwice * (p + kGeluCube * p * p * p));
    default: return p;
  }
}

// The logistic function and what it lacks to 1, both to fp32's relative accuracy (1 - s where s nears 1 would keep its absolute error of 2^-25 only,
// which gelu's slope multiplies by 40: 2e-6 at 5).
struct Logistic { float s, rest; };
__device__ __forceinline__ Logistic logistic_both(float a) {
  const float e = expf(-fabsf(a)), r = 1.f / (1.f + e), er = e * r;
  return a >= 0.f ? Logistic{r, er} : Logistic{er, r};
}

template <bool kFast> __device__ __forceinline__ float act_slope(float p, int act) {
  switch (act) {
    case UNIPOOL_ACT_RELU: return p > 0.f ? 1.f : p <= 0.f ? 0.f : p;
    case UNIPOOL_ACT_SILU: {
      if constexpr (kFast) {
        const float s = logistic<true>(p);
        return s * (1.f + p * (1.f - s));
      } else {
        const Logistic l = logistic_both(p);
        return l.s * (1.f + p * l.rest);
      }
    }
    case UNIPOOL_ACT_GELU: {
      const float q = fminf(fmaxf(p, -30.f), 30.f), q2 = q * q;     // 0 or 1 from there on; the square would overflow
      float s, both;                                                // s (1 - s); (p itself carries a NaN into s)
      if constexpr (kFast) {
        s = rcp_1_ex2(p * fmaf(q2, -kLog2e * kGeluTwice * kGeluCube, -kLog2e * kGeluTwice));
        both = fmaf(-s, s, s);
      } else {
        const Logistic l = logistic_both(kGeluTwice * (p + kGeluCube * p * q2));
        s = l.s;
        both = l.s * l.rest;
      }
      return fmaf(both, q * fmaf(q2, 3.f * kGeluTwice * kGeluCube, kGeluTwice), s);
    }
    default: return 1.f;
  }
}

}  // namespace unipool
