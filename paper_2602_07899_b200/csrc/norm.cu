// h = bf16(x + r); y = h / sqrt(mean h^2 + eps) * w; v = y / s; step = max(|v|max, 1e-5) / qpos; code = rint(v / step).
//
// One pass over the data: a CTA takes whole rows, a thread keeps its pieces of 8 channels of the row as 16-bit floats in registers
// between the sums and the codes, and the factors g = w / s of its channels in 32 bits for all rows of the CTA.  The largest |v| is the
// largest |h g| times the root, so that one sum over the CTA gives both; code = rint(h g k) with k = root / step.  The row after the one in
// registers is on its way into shared memory, into places of the thread's own: no barrier, and the memory has work while the CTA sums and
// rounds.  Bound by memory for many rows (8192 x 8192 with all but y: 98 us, 95 % of the copy rate; 4096 x 3584 24), by one trip to memory
// and the sum over the CTA for a few (1 x 3584: 2.3 us).  With its arguments as __grid_constant__ the compiler
// needs 8 to 16 registers less where they are not held to 64 (8192 x 8192 102 us without, 98 so).
#include "serve.cuh"

namespace tlq {
namespace {

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
  float inv_c, eps, inv_qpos;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 pack8(const float (&u)[8]) {
  return make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(u[4], u[5]), pack_bf16(u[6], u[7]));
}
__device__ __forceinline__ float max_nan(float a, float b) {  // (a NaN stays one)
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint4 ld_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// Thread t has pieces t, t + kThreads, ... of a row.
template <int kPieces, int kThreads, int kCtas, bool kKeep>
__global__ void __launch_bounds__(kThreads, kCtas)
norm_quantize_kernel(const __grid_constant__ NormArgs a) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ __align__(16) uint8_t ahead[];           // the next row's pieces of x, then of r
  __shared__ float2 s_part[2][kWarps];                       // of each warp, of two rows in turn
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t place_x = (uint32_t)__cvta_generic_to_shared(ahead) + tid * 16u, place_r = place_x + kPieces * kThreads * 16u;
  bool in[kPieces];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) in[p] = p * kThreads + tid < a.pieces;
  int64_t n = blockIdx.x;
  const uint4* x = reinterpret_cast<const uint4*>(a.x + n * a.ldx) + tid;
  const uint4* r = reinterpret_cast<const uint4*>(a.r + n * a.ldr) + tid;
  auto fetch = [&] {                           // the row at x and r into this thread's places
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
      if (in[p]) copy_ahead(place_x + p * kThreads * 16u, x + p * kThreads);
    if (a.r != nullptr) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
        if (in[p]) copy_ahead(place_r + p * kThreads * 16u, r + p * kThreads);
    }
  };
  after_previous();
  fetch();
  // w / s of a piece; kept in registers for all rows where there is room for them, else made anew from the first-level cache
  auto gains = [&](int p, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 1.f;
    if (in[p] && a.w != nullptr) unpack8(load_near(reinterpret_cast<const uint4*>(a.w) + p * kThreads + tid), f);
    if (in[p] && a.s != nullptr) {
      float s[8];
      unpack8(load_near(reinterpret_cast<const uint4*>(a.s) + p * kThreads + tid), s);
#pragma unroll
      for (int j = 0; j < 8; ++j)              // (by a divisor over 2^126 __fdividef would make 0)
        f[j] = kKeep ? f[j] * __frcp_rn(s[j]) : __fdividef(f[j] * 0.25f, s[j] * 0.25f);
    }
  };
  float kept[kKeep ? kPieces : 1][8];
  if (kKeep) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) gains(p, kept[kKeep ? p : 0]);
  }
  auto gain = [&](int p, float (&f)[8]) {
    if (!kKeep) return gains(p, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = kept[kKeep ? p : 0][j];
  };
  int64_t flat = n * a.pieces + tid;                          // this thread's first piece in the outputs without a pitch
  for (int parity = 0; n < a.N; n += gridDim.x, flat += (int64_t)gridDim.x * a.pieces, parity ^= 1) {
    uint4 h[kPieces];
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      h[p] = in[p] ? ld_shared(place_x + p * kThreads * 16u) : make_uint4(0, 0, 0, 0);
      if (a.r != nullptr && in[p]) {           // the sum is what the residual stream holds from here on, rounded to its 16 bits
        float u[8], v[8];
        unpack8(h[p], u);
        unpack8(ld_shared(place_r + p * kThreads * 16u), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] += v[j];
        h[p] = pack8(u);
      }
    }
    if (a.h != nullptr) {
      uint4* to = reinterpret_cast<uint4*>(a.h + n * a.ldh) + tid;
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
        if (in[p]) to[p * kThreads] = h[p];
    }
    // Over the row, the same in every thread: the sum of the squares of h, and the largest |h g|, which is |v| but for the root.
    float total, top;
    auto sums = [&] {
      float sum = 0.f, most = 0.f;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        float u[8], g[8];
        unpack8(h[p], u);
        gain(p, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum = fmaf(u[j], u[j], sum);
          most = max_nan(most, fabsf(u[j] * g[j]));
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        most = max_nan(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      }
      total = sum;
      top = most;
      if (kWarps > 1) {
        if (lane == 0) s_part[parity][warp] = make_float2(sum, most);
        __syncthreads();
        total = top = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float2 part = s_part[parity][k];
          total += part.x;
          top = max_nan(top, part.y);
        }
      }
    };
    auto once_more = [&](float power) {        // with h times a power of 2
      __syncthreads();
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        float u[8];
        unpack8(h[p], u);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] *= power;
        h[p] = pack8(u);
      }
      sums();
    };
    sums();
    if (n + gridDim.x < a.N) {                 // the next row (behind the sum over the CTA, which needs all of this one)
      x += (int64_t)gridDim.x * a.ldx / 8;
      r += (int64_t)gridDim.x * a.ldr / 8;
      fetch();
    }
    float eps = a.eps;
    if (!(total < INFINITY)) {                 // squares beyond the 32-bit range (or a row that is not finite): once more with h 2^-96,
      once_more(1.2621774483536189e-29f);      // where the sum of 32768 squares of the largest number is 2^79
      eps = 0.f;                               // (nothing beside such squares)
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p)          // (nothing of it is kept unpacked, which would take twice the registers)
      asm volatile("" : "+r"(h[p].x), "+r"(h[p].y), "+r"(h[p].z), "+r"(h[p].w));
    float root = total < INFINITY ? rsqrtf(fmaf(total, a.inv_c, eps)) : NAN;
    if (a.y != nullptr) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        if (!in[p]) continue;
        float u[8], w[8];
        unpack8(h[p], u);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.f;
        if (a.w != nullptr) unpack8(load_near(reinterpret_cast<const uint4*>(a.w) + p * kThreads + tid), w);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = u[j] * root * w[j];
        reinterpret_cast<uint4*>(a.y)[flat + p * kThreads] = pack8(u);
      }
    }
    if (a.codes == nullptr) continue;
    if (top == INFINITY && root < INFINITY) {  // |h g| beyond the 32-bit range, which |v| may be in: once more with h times the power of 2 in
      // the root, where no |h| is above the square root of the row's length (what gets lost below rounds to 0)
      const float power = __uint_as_float(__float_as_uint(root) & 0x7F800000u);
      once_more(power);
      root /= power;
    }
    const float largest = top * root;
    if (!(largest < INFINITY)) {               // not a number, or v or w / s leaves the range
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        if (!in[p]) continue;
        reinterpret_cast<uint2*>(a.codes)[flat + p * kThreads] = make_uint2(0, 0);
        if (a.values != nullptr) reinterpret_cast<uint4*>(a.values)[flat + p * kThreads] = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);
      }
      if (tid == 0) a.steps[n] = NAN;
      continue;
    }
    const float step = fmaxf(largest, TLQ_RANGE_FLOOR) * a.inv_qpos, k = __fdividef(root * 0.0625f, step * 0.0625f);   // (the same)
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      if (!in[p]) continue;
      float u[8], g[8];
      unpack8(h[p], u);
      gain(p, g);
      uint32_t c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float q = fmaf(u[j] * g[j], k, kRoundMagic);
        c[j] = __float_as_uint(q);
        u[j] = (q - kRoundMagic) * step;
      }
      const uint32_t lo = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
      const uint32_t hi = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
      reinterpret_cast<uint2*>(a.codes)[flat + p * kThreads] = make_uint2(lo, hi);
      if (a.values != nullptr) reinterpret_cast<uint4*>(a.values)[flat + p * kThreads] = pack8(u);
    }
    if (tid == 0) a.steps[n] = step;
  }
}

// CTAs of a kernel that an SM has at a time (asked once for each device).
template <int kPieces, int kThreads, int kCtas>
int run_norm(const NormArgs& a, cudaStream_t st) {
  constexpr size_t smem = 2 * kPieces * kThreads * 16;
  static OncePerDevice once;
  static int resident[kMaxDevices] = {};
  auto kernel = norm_quantize_kernel<kPieces, kThreads, kCtas, (kPieces * kThreads <= 2048)>;
  const int dev = current_device_index(), sms = device_sm_count();
  const int rc = once_per_device(once, [&] {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return e != cudaSuccess ? e : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident[dev], kernel, kThreads, smem);
  });
  if (rc != TLQ_OK) return rc;
  if (resident[dev] < 1 || sms < 1) return TLQ_ERR_CUDA;
  const int64_t grid = (int64_t)sms * resident[dev];
  return launch_next(kernel, dim3((unsigned)(a.N < grid ? a.N : grid)), kThreads, smem, 1, st, a);
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
  a.inv_qpos = 1.f / (float)((1 << (a_bits - 1)) - 1);
  const int pieces = a.pieces;
  if (N <= 2 * sms) {                          // few rows: as many threads to a row as there are pieces, the shortest way through it
    if (pieces <= 32) return run_norm<1, 32, 1>(a, st);
    if (pieces <= 128) return run_norm<1, 128, 1>(a, st);
    if (pieces <= 256) return run_norm<1, 256, 1>(a, st);
    if (pieces <= 512) return run_norm<1, 512, 1>(a, st);
    if (pieces <= 1024) return run_norm<2, 512, 1>(a, st);
  } else {                                     // many rows: two pieces to a thread, so that a sum over the CTA serves more bytes (four do
    if (pieces <= 32) return run_norm<1, 32, 1>(a, st);      // not fit into the registers of three CTAs of 256: 8192 x 8192 104 us with two
    if (pieces <= 64) return run_norm<2, 32, 1>(a, st);      // of them, 141 with spills, 102 so, then)
    if (pieces <= 128) return run_norm<2, 64, 16>(a, st);
    if (pieces <= 256) return run_norm<2, 128, 8>(a, st);
    if (pieces <= 512) return run_norm<2, 256, 4>(a, st);
    if (pieces <= 1024) return run_norm<2, 512, 2>(a, st);
  }
  return pieces <= 2048 ? run_norm<4, 512, 1>(a, st) : run_norm<4, 1024, 1>(a, st);
}

}  // namespace tlq
