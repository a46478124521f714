// Y[n,o] = bf16( t[n] u[o] sum_c Xq[n,c] Wq[o,c] + bias[o] ) from kept 8-bit codes.
//
// Few tokens: the weights' bytes are the bound (2 N operations per weight byte), and every weight is read once, straight
// from global memory into the registers of the lane that feeds it to the matrix instruction m16n8k32 (weights on the
// m side: 16 output channels, tokens on the n side).  Which channel of C1 a matrix index means is free as long as both
// operands agree, so a lane's operands are whole 16-byte pieces of a row.  A CTA owns 16 output channels and its eight
// warps share C1; the 32-bit integer partial sums are exact in any order.
#include "serve.cuh"

namespace tlq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;

__device__ __forceinline__ uint4 ld_weights(const int8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma_i8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int NT>
__global__ void __launch_bounds__(kThreads)
linear_i8_few_kernel(const int8_t* __restrict__ X, const float* __restrict__ t, const int8_t* __restrict__ W,
                     const float* __restrict__ u, const uint16_t* __restrict__ bias, int64_t N, int C1, int64_t C2,
                     uint16_t* __restrict__ Y) {
  __shared__ int s_acc[kWarps][NT * 8][17];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, q = lane & 3;
  const int64_t o0 = (int64_t)blockIdx.x * 16, n0 = (int64_t)blockIdx.y * (8 * NT);
  // rows beyond the end read the last one; their results are not stored
  const int8_t* w0 = W + min(o0 + g, C2 - 1) * C1;
  const int8_t* w1 = W + min(o0 + g + 8, C2 - 1) * C1;
  const int8_t* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = X + min(n0 + n * 8 + g, N - 1) * C1;
  int acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[n][j] = 0;
  const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll 4
  for (int c = (warp * 4 + q) * 16; c - q * 16 < C1; c += kWarps * 64) {
    const bool in = c < C1;                        // C1 is a multiple of 16: a piece is in or out as a whole
    const uint4 a = in ? ld_weights(w0 + c) : zero, b = in ? ld_weights(w1 + c) : zero;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4 v = in ? __ldg(reinterpret_cast<const uint4*>(x[n] + c)) : zero;
      mma_i8(acc[n], a.x, b.x, a.y, b.y, v.x, v.y);
      mma_i8(acc[n], a.z, b.z, a.w, b.w, v.z, v.w);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) s_acc[warp][n * 8 + 2 * q + (j & 1)][g + (j >> 1) * 8] = acc[n][j];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * 16; e += kThreads) {
    const int r = e & 15, n = e >> 4;
    if (n0 + n >= N || o0 + r >= C2) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += s_acc[w][n][r];
    float y = (float)sum * (t[n0 + n] * u[o0 + r]);
    if (bias != nullptr) y += bf16_bits_to_float(bias[o0 + r]);
    const __nv_bfloat16 v = __float2bfloat16_rn(y);
    Y[(n0 + n) * C2 + o0 + r] = *reinterpret_cast<const uint16_t*>(&v);
  }
}

}  // namespace

int launch_linear_i8(const int8_t* Xq, const float* t, const int8_t* Wq, const float* u, const uint16_t* bias, int64_t N,
                     int64_t C1, int64_t C2, uint16_t* Y, WorkspaceHeader* hdr, cudaStream_t st) {
  (void)hdr;
  const unsigned rows = (unsigned)ceil_div(C2, 16);
  if (N <= 8) {
    linear_i8_few_kernel<1><<<dim3(rows, 1), kThreads, 0, st>>>(Xq, t, Wq, u, bias, N, (int)C1, C2, Y);
  } else if (N <= 16) {
    linear_i8_few_kernel<2><<<dim3(rows, 1), kThreads, 0, st>>>(Xq, t, Wq, u, bias, N, (int)C1, C2, Y);
  } else {
    if (ceil_div(N, 32) > 65535) return TLQ_ERR_SHAPE;
    linear_i8_few_kernel<4><<<dim3(rows, (unsigned)ceil_div(N, 32)), kThreads, 0, st>>>(Xq, t, Wq, u, bias, N, (int)C1, C2, Y);
  }
  return after_launch();
}

}  // namespace tlq
