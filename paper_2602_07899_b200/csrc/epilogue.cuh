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
// z / (1 + e^-z), 0.5 z erfc(-z / sqrt 2), and z / (1 + e^-2a) = 0.5 z (1 + tanh a): forms without a difference of near numbers,
// so that results stay exact where they are small.  The approximate exponential and quotient are off by 2^-21, for a result of 8 bits.
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case TLQ_ACT_SILU: return __fdividef(z, 1.f + exp_of_minus(z));
    case TLQ_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678118654752f);
    case TLQ_ACT_GELU_TANH: return __fdividef(z, 1.f + exp_of_minus(1.5957691216057308f * fmaf(0.044715f * z * z, z, z)));
    default: return z;
  }
}

}  // namespace tlq
