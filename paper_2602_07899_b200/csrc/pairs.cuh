// Two floats in one 64-bit register, for the instructions that work on both at a time.
#pragma once

namespace tlq {

using pair2 = unsigned long long;
__device__ __forceinline__ pair2 pair_of(float lo, float hi) {
  pair2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 halves(pair2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ pair2 padd(pair2 a, pair2 b) {
  pair2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ pair2 pmul(pair2 a, pair2 b) {
  pair2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ pair2 pfma(pair2 a, pair2 b, pair2 c) {
  pair2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

}  // namespace tlq
