// What the 8-bit product does with z = t u sum + bias before it is rounded: y = act(z), times the product of the next row of the
// weights where the rows alternate between gate and up projection, plus a residual.
#pragma once

#include "common.cuh"
#include "pairs.cuh"

namespace tlq {

struct Epilogue {
  int act;                    // TLQ_ACT_*
  int gated;                  // rows 2j and 2j + 1 of the weights make channel j of the result
  const uint16_t* residual;   // rows ldr apart, or null
  int64_t ldr;
};

__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float one_over(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ pair2 exp2_of(pair2 x) {
  const float2 v = halves(x);
  return pair_of(exp2_of(v.x), exp2_of(v.y));
}
__device__ __forceinline__ pair2 one_over(pair2 x) {
  const float2 v = halves(x);
  return pair_of(one_over(v.x), one_over(v.y));
}
__device__ __forceinline__ pair2 both(float x) { return pair_of(x, x); }
__device__ __forceinline__ float size_to(float z, float most) {         // |z|, no larger than `most`; a NaN stays one
  float a;
  asm("{\n\t.reg .f32 n;\n\tabs.f32 n, %1;\n\tmin.NaN.f32 %0, n, %2;\n\t}" : "=f"(a) : "f"(z), "f"(most));
  return a;
}
__device__ __forceinline__ float is_positive(float z) { return __saturatef(z * 1.7014118346046923e38f); }   // 1, or 0 where z is negative or a NaN

// Two at a time, in forms without a difference of near numbers where the result is small:
//  SiLU          z / (1 + e^-z)
//  GELU by tanh  z / (1 + e^-2a) = 0.5 z (1 + tanh a)
//  GELU          max(z, 0) - |z| tail(|z|), with the normal distribution's integral from a on, tail(a) = t P(t) e^(-a^2/2), t = 1 / (1 + 0.398 a),
//                which turns all of a >= 0 into (0, 1].  P is a fit of lowest relative error to the quotient of both sides: off by
//                2^-13.4 at most, a sixteenth of the rounding of the result to 8 bits.  From 2^64 on a stands still, where the tail is 0, and
//                max(z, 0) is z times 1 or 0: so infinity is infinity, and -infinity no number, as the infinity times 0 that it stands for.
// (1025 tokens, 1280 -> 5120 with GELU: 52 us with CUDA's erfc, one at a time; 19 so; 15.5 without an activation.)
template <int kAct>
__device__ __forceinline__ pair2 activate(pair2 z) {
  if constexpr (kAct == TLQ_ACT_SILU) return pmul(z, one_over(padd(both(1.f), exp2_of(pmul(z, both(-1.4426950408889634f))))));
  if constexpr (kAct == TLQ_ACT_GELU_TANH) {
    // 2 a log2 e = z (k + 0.044715 k z^2), k = 2 sqrt(2 / pi) log2 e
    const pair2 inner = pfma(pmul(z, z), both(-0.10294324f), both(-2.3022082f));
    return pmul(z, one_over(padd(both(1.f), exp2_of(pmul(z, inner)))));
  }
  if constexpr (kAct == TLQ_ACT_GELU) {
    const float2 v = halves(z);
    const pair2 a = pair_of(size_to(v.x, 18446744073709551616.f), size_to(v.y, 18446744073709551616.f)), t = one_over(pfma(a, both(0.39800000190734863f), both(1.f)));
    pair2 p = both(0.08496466279029846f);
    p = pfma(p, t, both(-0.1475699543952942f));
    p = pfma(p, t, both(-0.11862977594137192f));
    p = pfma(p, t, both(-0.15996518731117249f));
    p = pfma(p, t, both(-0.1587645411491394f));
    const pair2 e = exp2_of(pmul(pmul(a, a), both(-0.72134752044448170f)));
    return pfma(z, pair_of(is_positive(v.x), is_positive(v.y)), pmul(pmul(a, pmul(p, t)), e));
  }
  return z;
}
// All n of v, or with `gated` n / 2 products of pairs; one decision for all of them.
template <int kAct, int n>
__device__ __forceinline__ void activate_as(bool gated, float (&v)[n]) {
  if (gated) {
#pragma unroll
    for (int j = 0; j < n / 2; j += 2) {
      const int k = n > 2 ? 2 * j + 2 : 0;
      const float2 y = halves(pmul(activate<kAct>(pair_of(v[2 * j], v[k])), pair_of(v[2 * j + 1], v[k + 1])));
      v[j] = y.x;
      if (n > 2) v[j + 1] = y.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < n; j += 2) {
      const float2 y = halves(activate<kAct>(pair_of(v[j], v[j + 1])));
      v[j] = y.x;
      v[j + 1] = y.y;
    }
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
