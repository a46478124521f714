// h = bf16(x + r); y = h / sqrt(mean h^2 + eps) * w; v = y / s; step = max(|v|max, 1e-5) / qpos; code = rint(v / step).
//
// One pass over the data: a CTA takes whole rows, a thread keeps its pieces of 8 channels of the row as 16-bit floats in registers
// between the sum of squares, the maximum and the codes, and the factors w / s of its channels in 32 bits for all rows of the CTA.
// Bound by memory for many rows, by one trip to memory and two sums over the CTA for a few.
#include "serve.cuh"

namespace tlq {
namespace {

constexpr int kNormThreads = 512;         // at most; 8 pieces of 8 channels each: rows of up to 32768 channels
constexpr int kNormWarps = kNormThreads / 32;
constexpr float kRoundMagic = 12582912.f; // 1.5 2^23: adding it rounds to the nearest integer, ties to even, in the lowest bits

struct NormArgs {
  const uint16_t* x;          // rows ldx apart
  const uint16_t* r;          // rows ldr apart, or null
  const uint16_t* w;          // [C] or null
  const uint16_t* s;          // [C] or null
  uint16_t* h;                // rows ldh apart, or null
  int8_t* codes;              // [N,C] or null
  float* steps;               // [N], with codes
  uint16_t* values;           // [N,C] or null
  uint16_t* y;                // [N,C] or null
  int64_t N, ldx, ldr, ldh;
  int pieces;                 // C / 8
  float inv_c, eps, qpos;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int kPieces>
__global__ void __launch_bounds__(kNormThreads)
norm_quantize_kernel(const NormArgs a) {
  __shared__ float s_sum[2][kNormWarps];
  __shared__ uint32_t s_max[2][kNormWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const uint4 none = make_uint4(0, 0, 0, 0);
  after_previous();
  float g[kPieces][8];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
    const int i = p * blockDim.x + threadIdx.x;
#pragma unroll
    for (int j = 0; j < 8; ++j) g[p][j] = 1.f;
    if (i < a.pieces && a.w != nullptr) unpack8(load_near(reinterpret_cast<const uint4*>(a.w) + i), g[p]);
    if (i < a.pieces && a.s != nullptr) {
      float s[8];
      unpack8(load_near(reinterpret_cast<const uint4*>(a.s) + i), s);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[p][j] *= __frcp_rn(s[j]);
    }
  }
  int parity = 0;
  for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x, parity ^= 1) {
    const uint4* x = reinterpret_cast<const uint4*>(a.x + n * a.ldx);
    uint4 h[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int i = p * blockDim.x + threadIdx.x;
      h[p] = i < a.pieces ? load_once(x + i) : none;
    }
    if (a.r != nullptr) {
      const uint4* r = reinterpret_cast<const uint4*>(a.r + n * a.ldr);
      uint4 q[kPieces];
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const int i = p * blockDim.x + threadIdx.x;
        q[p] = i < a.pieces ? load_once(r + i) : none;
      }
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {      // the sum is what the residual stream holds from here on, rounded to its 16 bits
        float u[8], v[8];
        unpack8(h[p], u);
        unpack8(q[p], v);
        h[p] = make_uint4(pack_bf16(u[0] + v[0], u[1] + v[1]), pack_bf16(u[2] + v[2], u[3] + v[3]),
                          pack_bf16(u[4] + v[4], u[5] + v[5]), pack_bf16(u[6] + v[6], u[7] + v[7]));
      }
    }
    if (a.h != nullptr) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const int i = p * blockDim.x + threadIdx.x;
        if (i < a.pieces) reinterpret_cast<uint4*>(a.h + n * a.ldh)[i] = h[p];
      }
    }
    // Sum of the squares of f h over the row, the same in every thread.
    auto squares = [&](float f) {
      float sum = 0.f;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        float u[8];
        unpack8(h[p], u);
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) part = fmaf(u[j] * f, u[j] * f, part);
        sum += part;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      if (lane == 0) s_sum[parity][warp] = sum;
      __syncthreads();
      float all = 0.f;
      for (int k = 0; k < warps; ++k) all += s_sum[parity][k];
      return all;
    };
    float f = 1.f, total = squares(1.f);
    if (!(total < INFINITY)) {                 // squares beyond the 32-bit range (or a row that is not finite): once more, scaled
      f = 1.2621774483536189e-29f;             // 2^-96: the sum of 32768 squares of the largest number is 2^79 then
      __syncthreads();
      total = squares(f);
    }
    const bool finite = total < INFINITY;
    const float root = rsqrtf(total * a.inv_c + a.eps * f * f);
    if (a.y != nullptr) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const int i = p * blockDim.x + threadIdx.x;
        if (i >= a.pieces) continue;
        float u[8], w[8];
        unpack8(h[p], u);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.f;
        if (a.w != nullptr) unpack8(load_near(reinterpret_cast<const uint4*>(a.w) + i), w);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = finite ? u[j] * root * w[j] * f : NAN;
        reinterpret_cast<uint4*>(a.y)[n * a.pieces + i] =
            make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(u[4], u[5]), pack_bf16(u[6], u[7]));
      }
    }
    if (a.codes == nullptr) continue;
    uint32_t top = 0;                          // of the bits of |v|, which order as the values do, with NaN above infinity
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      float u[8];
      unpack8(h[p], u);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(fabsf(u[j] * root * g[p][j] * f)));
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (lane == 0) s_max[parity][warp] = top;
    __syncthreads();
    for (int k = 0; k < warps; ++k) top = max(top, s_max[parity][k]);
    const bool good = finite && top < 0x7F800000u;
    const float step = good ? __fdiv_rn(fmaxf(__uint_as_float(top), TLQ_RANGE_FLOOR), a.qpos) : NAN;
    const float inv = good ? __fdiv_rn(1.f, step) : 0.f;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int i = p * blockDim.x + threadIdx.x;
      if (i >= a.pieces) continue;
      float u[8];
      unpack8(h[p], u);
      uint32_t c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float q = good ? u[j] * root * g[p][j] * f * inv + kRoundMagic : kRoundMagic;
        c[j] = __float_as_uint(q);
        u[j] = (q - kRoundMagic) * step;
      }
      const uint32_t lo = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
      const uint32_t hi = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
      reinterpret_cast<uint2*>(a.codes)[n * a.pieces + i] = make_uint2(lo, hi);
      if (a.values != nullptr)
        reinterpret_cast<uint4*>(a.values)[n * a.pieces + i] =
            make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(u[4], u[5]), pack_bf16(u[6], u[7]));
    }
    if (threadIdx.x == 0) a.steps[n] = step;
  }
}

}  // namespace

int launch_norm_quantize(const uint16_t* x, int64_t N, int64_t C, int64_t ldx, const uint16_t* r, int64_t ldr, const uint16_t* w,
                         float eps, const uint16_t* s, int a_bits, uint16_t* h, int64_t ldh, int8_t* codes, float* steps,
                         uint16_t* values, uint16_t* y, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  NormArgs a{};
  a.x = x; a.r = r; a.w = w; a.s = s; a.h = h; a.codes = codes; a.steps = steps; a.values = values; a.y = y;
  a.N = N; a.ldx = ldx; a.ldr = ldr; a.ldh = ldh;
  a.pieces = (int)(C / 8);
  a.inv_c = 1.f / (float)C;
  a.eps = eps;
  a.qpos = (float)((1 << (a_bits - 1)) - 1);
  // Few rows: as many threads to a row as there are pieces, the shortest way through it.  Many rows: up to four pieces to a thread,
  // so that a sum over the CTA serves more bytes, but two warps at least.
  const int want = N <= 2 * sms ? (int)ceil_div(a.pieces, kNormThreads) : a.pieces / 64;
  int per = 1;
  while (per < want && per < 4) per *= 2;
  while (per * kNormThreads < a.pieces) per *= 2;
  const int threads = (int)ceil_div(ceil_div(a.pieces, per), 32) * 32;
  const int64_t resident = (int64_t)sms * (per > 4 ? 1 : 1024 / threads);
  auto run = [&](auto kernel) {
    return launch_next(kernel, dim3((unsigned)(N < resident ? N : resident)), threads, 0, 1, st, a);
  };
  switch (per) {
    case 1: return run(norm_quantize_kernel<1>);
    case 2: return run(norm_quantize_kernel<2>);
    case 4: return run(norm_quantize_kernel<4>);
    default: return run(norm_quantize_kernel<8>);
  }
}

}  // namespace tlq
