// What the 8-bit product does with z = t u sum + bias before it is rounded: y = act(z), times the product of the next row of the
// weights where the rows alternate between gate and up projection, plus a residual.
#pragma once

#include "common.cuh"

namespace tlq {

struct Epilogue {
  int act;                    // TLQ_ACT_*
  int gated;                  // rows 2j and 2j + 1 of the weights make channel j of the result
  const uint16_t* residual;   // rows ldr apart, or null
  int64_t ldr;
};

__device__ __forceinline__ float exp_of_minus(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * -1.4426950408889634f));
  return y;
}
// The normal distribution's integral from a >= 0 on: t P(t) e^(-a^2/2) with t = 1 / (1 + 0.4 a), which turns all of a into (0, 1].  P is a
// fit of lowest relative error to the quotient of both sides, 2^-17 over the whole range; CUDA's own erfc takes three times as long.
__device__ __forceinline__ float normal_tail(float a) {
  const float t = __fdividef(1.f, fmaf(0.4f, a, 1.f));
  float p = 0.0498208738f;
  p = fmaf(p, t, -0.139627426f);
  p = fmaf(p, t, 0.0594341829f);
  p = fmaf(p, t, 0.0772080421f);
  p = fmaf(p, t, 0.1339580267f);
  p = fmaf(p, t, 0.1596342176f);
  p = fmaf(p, t, 0.1595757305f);
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a * a * -0.72134752044448170f));
  return p * t * e;
}
// SiLU: z / (1 + e^-z).  GELU: z times the normal distribution's integral up to z.  GELU by tanh: z / (1 + e^-2a) = 0.5 z (1 + tanh a).
// Forms without a difference of near numbers, so that results stay exact where they are small; errors of 2^-17 for a result of 8 bits.
template <int kAct>
__device__ __forceinline__ float activate(float z) {
  if constexpr (kAct == TLQ_ACT_SILU) return __fdividef(z, 1.f + exp_of_minus(z));
  if constexpr (kAct == TLQ_ACT_GELU) {
    const float tail = z * normal_tail(fabsf(z));
    return z > 0.f ? z - tail : tail;
  }
  if constexpr (kAct == TLQ_ACT_GELU_TANH) return __fdividef(z, 1.f + exp_of_minus(1.5957691216057308f * fmaf(0.044715f * z * z, z, z)));
  return z;
}
// The first n of v, or with `gated` n / 2 products of pairs; one decision for all of them.
template <int kAct, int n>
__device__ __forceinline__ void activate_as(bool gated, float (&v)[n]) {
  if (gated) {
#pragma unroll
    for (int j = 0; j < n / 2; ++j) v[j] = activate<kAct>(v[2 * j]) * v[2 * j + 1];
  } else {
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = activate<kAct>(v[j]);
  }
}
template <int n>
__device__ __forceinline__ void activate_all(int act, bool gated, float (&v)[n]) {
  switch (act) {
    case TLQ_ACT_SILU: return activate_as<TLQ_ACT_SILU>(gated, v);
    case TLQ_ACT_GELU: return activate_as<TLQ_ACT_GELU>(gated, v);
    case TLQ_ACT_GELU_TANH: return activate_as<TLQ_ACT_GELU_TANH>(gated, v);
    default: return activate_as<TLQ_ACT_NONE>(gated, v);
  }
}

}  // namespace tlq
