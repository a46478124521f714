// Y[n,o] = bf16( t[n] u[o] sum_c Xq[n,c] Wq[o,c] + bias[o] ) from kept 8-bit codes.
//
// Few tokens and small weights (linear_i8_few_kernel): latency is the bound.  Weights go straight from global memory into
// the registers of the lane that feeds them to the matrix instruction m16n8k32 (16 output channels on the m side, tokens on
// the n side).  Which channel of C1 a matrix index means is free as long as both operands agree, so a lane's operands are
// whole 16-byte pieces of a row.  A CTA owns 16 output channels and its warps share C1; the 32-bit integer partial sums are
// exact in any order.  One token, 3584 x 512: 2.7 us with 16 warps to a CTA, 3.2 with 8, 4.7 by the tile kernel.
//
// Everything else up to a few hundred tokens (linear_i8_tile_kernel): bound by the weights' bytes, which TMA keeps under way
// deeper than registers could.  16 tokens, 3584 x 18944 (68 MB): 15.5 us, 18.8 by the few kernel; 1 token, 18944 x 3584:
// 14.8 us against 17 to 28.
//
// Beyond that the persistent kernel of tlq_apply_layer, bound by the tensor core.
#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

__device__ __forceinline__ void mma_i8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int NT, int kWarps, bool kEpi>
__global__ void __launch_bounds__(kWarps * 32)
linear_i8_few_kernel(const int8_t* X, const float* t, const int8_t* W, const float* u, const uint16_t* bias, int64_t N, int C1,
                     int64_t C2, const Epilogue epi, uint16_t* Y) {
  constexpr int kThreads = kWarps * 32;
  __shared__ int s_acc[kWarps][NT * 8][17];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, q = lane & 3;
  after_previous();
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
    const uint4 a = in ? load_once(w0 + c) : zero, b = in ? load_once(w1 + c) : zero;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4 v = in ? load_near(reinterpret_cast<const uint4*>(x[n] + c)) : zero;
      mma_i8(acc[n], a.x, b.x, a.y, b.y, v.x, v.y);
      mma_i8(acc[n], a.z, b.z, a.w, b.w, v.z, v.w);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) s_acc[warp][n * 8 + 2 * q + (j & 1)][g + (j >> 1) * 8] = acc[n][j];
  __syncthreads();
  auto product = [&](int n, int r) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += s_acc[w][n][r];
    float y = (float)sum * (t[n0 + n] * u[o0 + r]);
    if (bias != nullptr) y += bf16_bits_to_float(bias[o0 + r]);
    return y;
  };
  if constexpr (kEpi) {
    const int pair = epi.gated ? 1 : 0;                       // C2 is even then: both rows of a pair are there
    const int64_t width = C2 >> pair;
    for (int e = threadIdx.x; e < NT * 8 * (16 >> pair); e += kThreads) {
      const int r = (e & ((16 >> pair) - 1)) << pair, n = e >> (4 - pair);
      if (n0 + n >= N || o0 + r >= C2) continue;
      float v[2] = {product(n, r), pair ? product(n, r + 1) : 0.f};
      activate_all(epi.act, pair != 0, v);
      float y = v[0];
      const int64_t o = (o0 + r) >> pair;
      if (epi.residual != nullptr) y += bf16_bits_to_float(epi.residual[(n0 + n) * epi.ldr + o]);
      const __nv_bfloat16 b = __float2bfloat16_rn(y);
      Y[(n0 + n) * width + o] = *reinterpret_cast<const uint16_t*>(&b);
    }
    return;
  }
  for (int e = threadIdx.x; e < NT * 8 * 16; e += kThreads) {
    const int r = e & 15, n = e >> 4;
    if (n0 + n >= N || o0 + r >= C2) continue;
    const __nv_bfloat16 v = __float2bfloat16_rn(product(n, r));
    Y[(n0 + n) * C2 + o0 + r] = *reinterpret_cast<const uint16_t*>(&v);
  }
}


// ---------------------------------------------------------------------------------------------- tensor-memory kernel
// Up to a few hundred tokens, fewer tiles than SMs: tcgen05 with 128 output channels on the M side (accumulator lanes) and
// a tile of up to 256 tokens on the N side, 128 channels of C1 per stage, operands staged by TMA (128-byte swizzle), 32-bit
// integer accumulators in tensor memory.  The CTAs of a cluster (up to 8) share the C1 of one tile, so that all SMs read
// weights; each leaves its integer sums in its shared memory and adds up a part of the tokens over the cluster's, exact in
// any order.  A warp then stores whole pieces of 128 channels of a token's row.
constexpr int kTileO = 128, kTileN = 256, kTileK = 128;
constexpr int kMaxStages = 8, kMaxSplits = 8;
constexpr int kTileThreads = 320;                         // producer, MMA issuer, eight warps that empty the accumulator
constexpr uint32_t kWBytes = kTileO * kTileK;
constexpr uint32_t kStageBudget = 4 * (kWBytes + kTileN * kTileK);

struct TileArgs {
  const float* t;
  const float* u;
  const uint16_t* bias;
  uint16_t* Y;
  WorkspaceHeader* hdr;
  int64_t N, C2;
  int num_kb, tile_n, stages, mtiles, splits;
  uint32_t tmem_cols;
  Epilogue epi;
  int piece;                  // ... whose results and residual lie in rows of whole pieces of 4, 2 or 1 channels
};

__device__ __forceinline__ int4 ld_cluster(uint32_t addr) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add(int4& a, const int4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; }

template <bool kEpi>
__global__ void __launch_bounds__(kTileThreads, 1)
linear_i8_tile_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const TileArgs g) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t stage_bytes = kWBytes + (uint32_t)g.tile_n * kTileK;
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 1];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto full = [&](int i) { return ptx::smem_u32(&bars[i]); };
  auto empty = [&](int i) { return ptx::smem_u32(&bars[kMaxStages + i]); };
  const uint32_t acc_full = ptx::smem_u32(&bars[2 * kMaxStages]);
  if (threadIdx.x == 0) {
    for (int i = 0; i < g.stages; ++i) {
      ptx::mbar_init(full(i), 1);
      ptx::mbar_init(empty(i), 1);
    }
    ptx::mbar_init(acc_full, 1);
    s_abort = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmW);
    ptx::prefetch_tensormap(&tmX);
  }
  if (warp == 1) ptx::tmem_alloc(ptx::smem_u32(&s_tmem), g.tmem_cols);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = s_tmem;
  volatile int* abort_flag = &s_abort;
  after_previous();

  const int rank = (int)(blockIdx.x % g.splits), tile = (int)(blockIdx.x / g.splits);
  const int mt = tile % g.mtiles, ot = tile / g.mtiles;   // token tiles of the same weights run side by side
  const int kb0 = (int)((int64_t)g.num_kb * rank / g.splits), kb1 = (int)((int64_t)g.num_kb * (rank + 1) / g.splits);

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!ptx::mbar_wait(empty(stage), phase ^ 1u, abort_flag)) {
          report_status(g.hdr, TLQ_ERR_TIMEOUT, 220);
          break;
        }
        const uint32_t dst = base + stage * stage_bytes;
        ptx::mbar_expect_tx(full(stage), stage_bytes);
        ptx::tma_load_2d(dst, &tmW, full(stage), kb * kTileK, ot * kTileO);
        ptx::tma_load_2d(dst + kWBytes, &tmX, full(stage), kb * kTileK, mt * g.tile_n);
        if (++stage == g.stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = ptx::make_idesc(2, 1, kTileO, (uint32_t)g.tile_n, false);     // s8 x s8 -> s32
      int stage = 0;
      uint32_t phase = 0, accumulate = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!ptx::mbar_wait(full(stage), phase, abort_flag)) {
          report_status(g.hdr, TLQ_ERR_TIMEOUT, 221);
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t src = base + stage * stage_bytes;
        const uint64_t a = ptx::smem_desc_sw128(src), b = ptx::smem_desc_sw128(src + kWBytes);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          ptx::mma_i8_ss(tmem, a + 2 * k, b + 2 * k, idesc, accumulate);
          accumulate = 1;
        }
        ptx::mma_commit(empty(stage));
        if (++stage == g.stages) { stage = 0; phase ^= 1u; }
      }
      if (ok) ptx::mma_commit(acc_full);
    }
  } else {
    // the accumulator to shared memory, token by channel (the stages are free once it is complete)
    const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane;
    if (!ptx::mbar_wait(acc_full, 0, abort_flag)) {
      if (lane == 0) report_status(g.hdr, TLQ_ERR_TIMEOUT, 222);
    }
    __syncwarp();
    if (*abort_flag == 0) {
      ptx::tc_fence_after();
      const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16);
      for (int c = half * 16; c < g.tile_n; c += 32) {
        uint32_t r[16];
        __syncwarp();
        ptx::tmem_ld16(src + c, r);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j)
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + (uint32_t)((c + j) * kTileO + row) * 4u), "r"(r[j]) : "memory");
      }
      ptx::tc_fence_before();
    }
  }
  __syncwarp();
  if (g.splits > 1) ptx::cluster_sync_all(); else __syncthreads();
  if (*abort_flag == 0) {
    const int64_t n0 = (int64_t)mt * g.tile_n, o = (int64_t)ot * kTileO + 4 * lane;
    const int c0 = g.tile_n * rank / g.splits;
    const int c1 = (int)min((int64_t)(g.tile_n * (rank + 1) / g.splits), g.N - n0);
    float u[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = o + j < g.C2 ? load_near(g.u + o + j) : 0.f;
      b[j] = g.bias != nullptr && o + j < g.C2 ? bf16_bits_to_float(g.bias[o + j]) : 0.f;
    }
    const bool whole = (g.C2 & 3) == 0 && o + 4 <= g.C2;  // four channels at an address of 8 bytes
    uint32_t from[kMaxSplits];
#pragma unroll
    for (int r = 0; r < kMaxSplits; ++r) from[r] = g.splits > 1 && r < g.splits ? ptx::map_to_cta(base, (uint32_t)r) : base;
    if constexpr (kEpi) {
      // channels o .. o + 3, or o / 2 and o / 2 + 1 of pairs (C2 is even then)
      const bool gated = g.epi.gated != 0;
      const int64_t width = gated ? g.C2 >> 1 : g.C2, to = gated ? o >> 1 : o;
      const int count = (int)max((int64_t)0, min((int64_t)(gated ? 2 : 4), width - to));
      auto finish = [&](int c, const int4& s, float t) {
        float v[4] = {fmaf((float)s.x, t * u[0], b[0]), fmaf((float)s.y, t * u[1], b[1]), fmaf((float)s.z, t * u[2], b[2]),
                      fmaf((float)s.w, t * u[3], b[3])};
        activate_all(g.epi.act, gated, v);
        uint16_t* out = g.Y + (n0 + c) * width + to;
        const uint16_t* res = g.epi.residual == nullptr ? nullptr : g.epi.residual + (n0 + c) * g.epi.ldr + to;
        if (count > 0 && g.piece >= (gated ? 2 : 4)) {       // all of them at an address that is a multiple of their size
          uint2 r = make_uint2(0u, 0u);
          if (res != nullptr && gated) r.x = load_near(reinterpret_cast<const uint32_t*>(res));
          if (res != nullptr && !gated) r = load_near(reinterpret_cast<const uint2*>(res));
          if (res != nullptr) {
            v[0] += bf16_bits_to_float(r.x & 0xFFFFu); v[1] += bf16_bits_to_float(r.x >> 16);
            v[2] += bf16_bits_to_float(r.y & 0xFFFFu); v[3] += bf16_bits_to_float(r.y >> 16);
          }
          const __nv_bfloat162 p0 = __floats2bfloat162_rn(v[0], v[1]), p1 = __floats2bfloat162_rn(v[2], v[3]);
          r = make_uint2(*reinterpret_cast<const uint32_t*>(&p0), *reinterpret_cast<const uint32_t*>(&p1));
          if (gated) *reinterpret_cast<uint32_t*>(out) = r.x;
          else *reinterpret_cast<uint2*>(out) = r;
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k >= count) continue;
            if (res != nullptr) v[k] += bf16_bits_to_float(res[k]);
            const __nv_bfloat16 p = __float2bfloat16_rn(v[k]);
            out[k] = *reinterpret_cast<const uint16_t*>(&p);
          }
        }
      };
      constexpr int kStep = kTileThreads / 32;
      if (g.splits == 1) {                                   // many tokens to a warp: four of them under way
        for (int c = c0 + warp; c < c1; c += 4 * kStep) {
          int4 s[4];
          float t[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int at = min(c + k * kStep, c1 - 1);
            t[k] = load_near(g.t + n0 + at);
            s[k] = ld_cluster(base + (uint32_t)(at * kTileO + 4 * lane) * 4u);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k * kStep < c1) finish(c + k * kStep, s[k], t[k]);
        }
      } else {
        for (int c = c0 + warp; c < c1; c += kStep) {
          const uint32_t at = (uint32_t)(c * kTileO + 4 * lane) * 4u;
          const float t = load_near(g.t + n0 + c);
          int4 v[kMaxSplits];
#pragma unroll
          for (int r = 0; r < kMaxSplits; ++r) v[r] = r < g.splits ? ld_cluster(from[r] + at) : make_int4(0, 0, 0, 0);
#pragma unroll
          for (int r = 1; r < kMaxSplits; ++r) add(v[0], v[r]);
          finish(c, v[0], t);
        }
      }
    } else
    for (int c = c0 + warp; c < c1; c += kTileThreads / 32) {
      const uint32_t at = (uint32_t)(c * kTileO + 4 * lane) * 4u;
      const float t = load_near(g.t + n0 + c);
      int4 s = ld_cluster(from[0] + at);
      if (g.splits > 1) {
        int4 v[kMaxSplits];
#pragma unroll
        for (int r = 1; r < kMaxSplits; ++r) v[r] = r < g.splits ? ld_cluster(from[r] + at) : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int r = 1; r < kMaxSplits; ++r) add(s, v[r]);
      }
      const float y0 = fmaf((float)s.x, t * u[0], b[0]), y1 = fmaf((float)s.y, t * u[1], b[1]);
      const float y2 = fmaf((float)s.z, t * u[2], b[2]), y3 = fmaf((float)s.w, t * u[3], b[3]);
      const __nv_bfloat162 p0 = __floats2bfloat162_rn(y0, y1), p1 = __floats2bfloat162_rn(y2, y3);
      const uint2 w = make_uint2(*reinterpret_cast<const uint32_t*>(&p0), *reinterpret_cast<const uint32_t*>(&p1));
      uint16_t* y = g.Y + (n0 + c) * g.C2 + o;
      if (whole) {
        *reinterpret_cast<uint2*>(y) = w;
      } else {
        if (o < g.C2) y[0] = (uint16_t)w.x;
        if (o + 1 < g.C2) y[1] = (uint16_t)(w.x >> 16);
        if (o + 2 < g.C2) y[2] = (uint16_t)w.y;
        if (o + 3 < g.C2) y[3] = (uint16_t)(w.y >> 16);
      }
    }
  }
  __syncwarp();
  if (g.splits > 1) ptx::cluster_sync_all();              // nobody leaves while its shared memory is read
  if (*abort_flag != 0)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);     // copies under way land before the shared memory is given back
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, g.tmem_cols);
  }
}

bool map_codes(CUtensorMap* tm, const int8_t* p, int64_t rows, int64_t cols, uint32_t box_rows) {
  const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows};
  const uint64_t pitch[1] = {(uint64_t)cols};
  const uint32_t box[2] = {kTileK, box_rows};
  return encode_tensor_map(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, p, dims, pitch, box);
}

template <bool kEpi>
int configure_tiles() {
  static OncePerDevice once;
  return once_per_device(once, [] {
    return cudaFuncSetAttribute(linear_i8_tile_kernel<kEpi>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kStageBudget + 1024));
  });
}

int launch_tiles(const int8_t* Xq, const float* t, const int8_t* Wq, const float* u, const uint16_t* bias, int64_t N, int64_t C1,
                 int64_t C2, const Epilogue* epi, uint16_t* Y, WorkspaceHeader* hdr, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  TileArgs g{};
  g.t = t; g.u = u; g.bias = bias; g.Y = Y; g.hdr = hdr; g.N = N; g.C2 = C2;
  const int64_t mtiles = ceil_div(N, kTileN), otiles = ceil_div(C2, kTileO);
  g.tile_n = (int)(ceil_div(ceil_div(N, mtiles), 16) * 16);
  // narrow tiles (bound by the weights' bytes) run two CTAs per SM
  const bool narrow = g.tile_n <= 64;
  const int64_t slots = narrow ? 2 * sms : sms, tiles = mtiles * otiles;
  // more tiles than that: the persistent kernel of tlq_apply_layer, which writes one tile while it sums the next
  if (tiles > slots) return launch_apply_gemm_i8(Xq, Wq, t, u, bias, N, C1, C2, epi, Y, hdr, st);
  g.mtiles = (int)mtiles;
  g.num_kb = (int)ceil_div(C1, kTileK);
  const uint32_t stage_bytes = kWBytes + (uint32_t)g.tile_n * kTileK;
  g.stages = (int)((narrow ? 104u * 1024u : kStageBudget) / stage_bytes);
  if (g.stages > kMaxStages) g.stages = kMaxStages;
  g.splits = 1;
  while (g.splits < kMaxSplits && 2 * g.splits * tiles <= slots && 2 * g.splits <= g.num_kb) g.splits *= 2;
  g.tmem_cols = 32;
  while (g.tmem_cols < (uint32_t)g.tile_n) g.tmem_cols *= 2;
  CUtensorMap tmW, tmX;
  if (!map_codes(&tmW, Wq, C2, C1, kTileO) || !map_codes(&tmX, Xq, N, C1, (uint32_t)g.tile_n)) return TLQ_ERR_CUDA;
  size_t smem = (size_t)g.stages * stage_bytes;
  if (smem < (size_t)g.tile_n * kTileO * 4) smem = (size_t)g.tile_n * kTileO * 4;
  if (epi != nullptr) {
    g.epi = *epi;
    const int64_t width = epi->gated ? C2 / 2 : C2;
    auto pieces = [&](int64_t n) {
      return width % n == 0 && (epi->residual == nullptr || (epi->ldr % n == 0 && (reinterpret_cast<uintptr_t>(epi->residual) & (uintptr_t)(2 * n - 1)) == 0));
    };
    g.piece = pieces(4) ? 4 : pieces(2) ? 2 : 1;
  }
  const int rc = epi != nullptr ? configure_tiles<true>() : configure_tiles<false>();
  if (rc != TLQ_OK) return rc;
  return launch_next(epi != nullptr ? linear_i8_tile_kernel<true> : linear_i8_tile_kernel<false>, dim3((unsigned)(tiles * g.splits)),
                     kTileThreads, smem + 1024, (unsigned)g.splits, st, tmW, tmX, g);
}

}  // namespace

int launch_linear_i8(const int8_t* Xq, const float* t, const int8_t* Wq, const float* u, const uint16_t* bias, int64_t N,
                     int64_t C1, int64_t C2, const Epilogue* epi, uint16_t* Y, WorkspaceHeader* hdr, cudaStream_t st) {
  // Few tokens and weights of up to 24 MB: measured, the few kernel is ahead up to 14 MB (1536 x 8960: 4.7 us against 6.1) and
  // behind from 64 MB on (8192 x 8192: 16.1 against 15.0).
  if (N > 16 || C1 * C2 > (24 << 20)) return launch_tiles(Xq, t, Wq, u, bias, N, C1, C2, epi, Y, hdr, st);
  const unsigned ctas = (unsigned)ceil_div(C2, 16);
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  // with no more CTAs than SMs a CTA has an SM to itself and takes twice the warps (1536 x 8960, 560 CTAs: 5.8 us so, 4.7 not)
  const bool deep = (int)ctas <= sms;
  const Epilogue e = epi != nullptr ? *epi : Epilogue{};
  auto run = [&](auto kernel, int warps) {
    return launch_next(kernel, dim3(ctas), warps * 32, 0, 1, st, Xq, t, Wq, u, bias, N, (int)C1, C2, e, Y);
  };
  if (epi != nullptr) {
    if (N <= 8) return deep ? run(linear_i8_few_kernel<1, 16, true>, 16) : run(linear_i8_few_kernel<1, 8, true>, 8);
    return deep ? run(linear_i8_few_kernel<2, 16, true>, 16) : run(linear_i8_few_kernel<2, 8, true>, 8);
  }
  if (N <= 8) return deep ? run(linear_i8_few_kernel<1, 16, false>, 16) : run(linear_i8_few_kernel<1, 8, false>, 8);
  return deep ? run(linear_i8_few_kernel<2, 16, false>, 16) : run(linear_i8_few_kernel<2, 8, false>, 8);
}

}  // namespace tlq
