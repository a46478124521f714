// A model's logits, read once: log probabilities of given tokens with entropy and the largest alternatives, and the distillation loss
// on a teacher's top logits with its gradient.
//
//   d_v = scale log2(e) z_v - m',  S = sum 2^d_v,  T = sum 2^d_v d_v   (m': the largest of scale log2(e) z_v, rounded)
//   lse = ln2 (m' + log2 S),  ln p_v = ln2 (d_v - log2 S),  entropy = ln S - ln2 T / S,
//   grad_v = w scale (2^d_v / S - sum of the teacher's p at v).
//
// Maximum and sums run along in one pass (each thread with a maximum of its own, looked at once for a batch of loads), so that the
// row is read from memory once; the loss then takes K logits of it.  The gradient reads the row a second time, from the second-level
// cache: the rows under way at one time are kept to what stays there by giving a row to a cluster of CTAs.  The largest K: at the end of
// the pass every thread knows the largest logit it has seen; the K-th largest of these is a bound below which nothing is wanted, and
// only the threads above it look through their logits again.  Bound by memory; the exponentials take 3/4 of that time (16 bits).
//
// Rows may begin at any element: vectors of 16 bytes lie on the memory's own grid, those at a row's ends are read element by element.
#include <type_traits>

#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kMaxTop = TLQ_MAX_TOP;
constexpr int kBatch = 4;                 // vectors of a thread under way at a time
constexpr int kCandidates = 2048;         // logits that may be among the largest, as keys
constexpr float kMasked = -1.2676506002282294e30f;       // -2^100: logits from here down have probability 0
constexpr uint32_t kMaskedPair = 0xF180F180u;            // the same, twice in bf16

using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 halves(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 padd(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 pfma(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {   // (a NaN stays one)
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// ---------------------------------------------------------------------------------------------- elements and rows
template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int kVec = 8, kPairs = 4;
  __device__ static float load(const uint16_t* p) {
    uint16_t v;
    asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
    return bf16_bits_to_float(v);
  }
  __device__ static void store(uint16_t* p, float f) {
    const __nv_bfloat16 v = __float2bfloat16_rn(f);
    *p = *reinterpret_cast<const uint16_t*>(&v);
  }
  // Four words of a vector, each no less than the mask's value.
  __device__ static uint4 clamp(const uint4& v) {
    return make_uint4(max_bf16x2(v.x, kMaskedPair), max_bf16x2(v.y, kMaskedPair), max_bf16x2(v.z, kMaskedPair), max_bf16x2(v.w, kMaskedPair));
  }
  __device__ static float largest(const uint4 (&v)[kBatch]) {
    uint32_t m = max_bf16x2(max_bf16x2(v[0].x, v[0].y), max_bf16x2(v[0].z, v[0].w));
#pragma unroll
    for (int u = 1; u < kBatch; ++u) m = max_bf16x2(m, max_bf16x2(max_bf16x2(v[u].x, v[u].y), max_bf16x2(v[u].z, v[u].w)));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  __device__ static void pairs(const uint4& v, f32x2 (&x)[kPairs]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  __device__ static uint32_t masked() { return kMaskedPair; }
  __device__ static uint4 pack(const float (&f)[kVec]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static void put(uint4& v, int j, float f) {
    const uint32_t bits = __float_as_uint(f) >> 16;
    uint32_t* w = &v.x + (j >> 1);
    *w = (j & 1) ? (*w & 0xFFFFu) | (bits << 16) : (*w & 0xFFFF0000u) | bits;
  }
};
template <>
struct Elem<float> {
  static constexpr int kVec = 4, kPairs = 2;
  __device__ static float load(const float* p) { return load_near(p); }
  __device__ static void store(float* p, float f) { *p = f; }
  __device__ static uint4 clamp(const uint4& v) {
    auto c = [](uint32_t w) { return __float_as_uint(max_nan(__uint_as_float(w), kMasked)); };
    return make_uint4(c(v.x), c(v.y), c(v.z), c(v.w));
  }
  __device__ static float largest(const uint4 (&v)[kBatch]) {
    float m = kMasked;
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[u].x), __uint_as_float(v[u].y)), fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
    return m;
  }
  __device__ static void pairs(const uint4& v, f32x2 (&x)[kPairs]) {
    x[0] = pair_of(__uint_as_float(v.x), __uint_as_float(v.y));
    x[1] = pair_of(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  __device__ static uint32_t masked() { return __float_as_uint(kMasked); }
  __device__ static uint4 pack(const float (&f)[kVec]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  __device__ static void put(uint4& v, int j, float f) { (&v.x)[j] = __float_as_uint(f); }
};

// A CTA's part of a row: vectors [lo, hi) of the 16-byte grid, of which vector i holds elements i kVec - off and on.
template <typename T>
struct Row {
  const T* z;                 // element 0
  int off, V, lo, hi;
  __device__ Row(const T* logits, int64_t n, int64_t ld, int V_, int rank, int ctas) : z(logits + n * ld), V(V_) {
    off = (int)((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
    const int vectors = (off + V + Elem<T>::kVec - 1) / Elem<T>::kVec, per = (vectors + ctas - 1) / ctas;
    lo = min(vectors, rank * per);
    hi = min(vectors, lo + per);
  }
  __device__ int first(int i) const { return i * Elem<T>::kVec - off; }
  __device__ bool whole(int i) const { return first(i) >= 0 && first(i) + Elem<T>::kVec <= V; }
  __device__ uint4 none() const { return make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked()); }
  __device__ uint4 load(int i) const {
    if (whole(i)) return load_once(z + first(i));
    uint4 v = none();
#pragma unroll
    for (int j = 0; j < Elem<T>::kVec; ++j)
      if (first(i) + j >= 0 && first(i) + j < V) Elem<T>::put(v, j, Elem<T>::load(z + first(i) + j));
    return v;
  }
};

// ---------------------------------------------------------------------------------------------- maximum and sums
struct Stat {
  float m, mc;                // the largest logit, and that times scale log2(e), rounded
  float s, t;                 // sums of 2^d and of 2^d d
};
__device__ __forceinline__ Stat empty_stat(float c2) { return Stat{kMasked, kMasked * c2, 0.f, 0.f}; }

// Over the lanes of a warp, in a fixed order; every lane gets the same.
__device__ __forceinline__ Stat merge_warp(const Stat& a, float c2) {
  Stat r;
  r.m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.m = fmaxf(r.m, __shfl_xor_sync(0xFFFFFFFFu, r.m, o));
  r.mc = r.m * c2;
  const float d = a.mc - r.mc, f = exp2_fast(d);
  r.s = a.s * f;
  r.t = f * fmaf(a.s, d, a.t);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, o);
    r.t += __shfl_xor_sync(0xFFFFFFFFu, r.t, o);
  }
  return r;
}

struct RowShared {
  Stat warps[16];
  float cta[4];               // what the other CTAs of the cluster read
};
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// Maximum and sums of the whole row, the same in every thread of every CTA of it; `mine`: the largest logit of this thread's vectors.
template <typename T, bool kEntropy, int kThreads>
__device__ __forceinline__ Stat row_stat(const Row<T>& row, float c2, int ctas, RowShared& sh, float& mine) {
  constexpr int kWarps = kThreads / 32, kPairs = Elem<T>::kPairs;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Stat a = empty_stat(c2);
  const f32x2 cc = pair_of(c2, c2);
  f32x2 s = pair_of(0.f, 0.f), t = s;
  for (int i0 = row.lo + (int)threadIdx.x; i0 < row.hi; i0 += kBatch * kThreads) {
    uint4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = i0 + u * kThreads < row.hi ? row.load(i0 + u * kThreads) : row.none();
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = Elem<T>::clamp(v[u]);
    const float m = fmaxf(a.m, Elem<T>::largest(v));          // (a NaN passes by here and shows in the sum)
    if (m > a.m) {
      const float mc = m * c2, d = a.mc - mc, f = exp2_fast(d);
      const float2 s2 = halves(s), t2 = halves(t);
      if (kEntropy) t = pair_of(f * fmaf(s2.x, d, t2.x), f * fmaf(s2.y, d, t2.y));
      s = pair_of(s2.x * f, s2.y * f);
      a.m = m;
      a.mc = mc;
    }
    const f32x2 minus = pair_of(-a.mc, -a.mc);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      f32x2 x[kPairs];
      Elem<T>::pairs(v[u], x);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const f32x2 d = pfma(x[j], cc, minus);
        const float2 d2 = halves(d);
        const f32x2 e = pair_of(exp2_fast(d2.x), exp2_fast(d2.y));
        s = padd(s, e);
        if (kEntropy) t = pfma(e, d, t);
      }
    }
  }
  mine = a.m;
  a.s = halves(s).x + halves(s).y;
  a.t = halves(t).x + halves(t).y;
  a = merge_warp(a, c2);
  if (lane == 0) sh.warps[warp] = a;
  __syncthreads();
  a = merge_warp(lane < kWarps ? sh.warps[lane] : empty_stat(c2), c2);
  if (ctas > 1) {
    if (threadIdx.x == 0) {
      sh.cta[0] = a.m; sh.cta[1] = a.mc; sh.cta[2] = a.s; sh.cta[3] = a.t;
    }
    __syncwarp();
    ptx::cluster_sync_all();
    a = empty_stat(c2);
    if (lane < ctas) {
      const uint32_t from = ptx::map_to_cta(ptx::smem_u32(sh.cta), (uint32_t)lane);
      a.m = ld_cluster_f32(from); a.mc = ld_cluster_f32(from + 4); a.s = ld_cluster_f32(from + 8); a.t = ld_cluster_f32(from + 12);
    }
    __syncwarp();
    a = merge_warp(a, c2);
  }
  return a;
}

// ---------------------------------------------------------------------------------------------- the largest K
// Keys order as the logits do, and equal logits by their index, the lower one first; 0 is none.
__device__ __forceinline__ uint32_t in_order(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);                // (-0 is 0)
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ unsigned long long key_of(float x, int index) {
  return ((unsigned long long)in_order(x) << 32) | (0xFFFFFFFFu - (uint32_t)index);
}

struct TopShared {
  unsigned long long keys[kCandidates];
  unsigned long long top[kMaxTop];        // of this CTA's part, largest first
  unsigned long long all[kMaxTop];        // of the row
  uint16_t threads[512];
  int n_keys, n_threads;
};

// The K-th largest of the first n keys (n >= K).
template <int kThreads>
__device__ unsigned long long kth_key(const TopShared& sh, int n, int K) {
  unsigned long long bound = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const unsigned long long next = bound | (1ull << bit);
    int count = 0;
    for (int i = 0; i < n; i += kThreads) count += __syncthreads_count(i + (int)threadIdx.x < n && sh.keys[min(i + (int)threadIdx.x, n - 1)] >= next);
    if (count >= K) bound = next;
  }
  return bound;
}

// The largest K of this CTA's part of the row into sh.top.  `mine`: the largest logit of this thread's vectors.
template <typename T, int kThreads>
__device__ __forceinline__ void top_of_part(const Row<T>& row, int K, float mine, TopShared& sh) {
  const int tid = threadIdx.x;
  const bool any = row.lo + tid < row.hi;
  const uint32_t own = any ? in_order(mine) : 0u;
  // a bound that K threads at least reach (none where fewer have anything; the part is small then); the 16 lower bits of a bf16 say nothing
  uint32_t bound = 0;
  for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {
    const uint32_t next = bound | (1u << bit);
    if (__syncthreads_count(own >= next) >= K) bound = next;
  }
  if (tid == 0) sh.n_threads = 0;
  if (tid < K) sh.top[tid] = 0;
  __syncthreads();
  if (any && own >= bound) sh.threads[atomicAdd(&sh.n_threads, 1)] = (uint16_t)tid;
  __syncthreads();
  const int listed = sh.n_threads, columns = (row.hi - row.lo + kThreads - 1) / kThreads;
  unsigned long long least = (unsigned long long)bound << 32;
  int n;
  while (true) {
    if (tid == 0) sh.n_keys = 0;
    __syncthreads();
    for (int k = tid; k < listed * columns; k += kThreads) {
      const int i = row.lo + sh.threads[k % listed] + k / listed * kThreads;
      if (i >= row.hi) continue;
      const uint4 v = Elem<T>::clamp(row.load(i));
      f32x2 x[Elem<T>::kPairs];
      Elem<T>::pairs(v, x);
#pragma unroll
      for (int j = 0; j < Elem<T>::kVec; ++j) {
        const float2 h = halves(x[j >> 1]);
        const int e = row.first(i) + j;
        const unsigned long long key = key_of((j & 1) ? h.y : h.x, e);
        if (key >= least && e >= 0 && e < row.V) {
          const int at = atomicAdd(&sh.n_keys, 1);
          if (at < kCandidates) sh.keys[at] = key;
        }
      }
    }
    __syncthreads();
    n = sh.n_keys;
    if (n <= kCandidates) break;
    least = kth_key<kThreads>(sh, kCandidates, K);            // more than there is room for: a higher bound, from those there was room for
    __syncthreads();
  }
  // each key's place is the number of larger ones; with many of them only the largest K are placed
  if (n > kThreads / 2 && n > K) least = kth_key<kThreads>(sh, n, K);
  for (int i = tid; i < n; i += kThreads) {
    const unsigned long long key = sh.keys[i];
    if (key < least) continue;
    int place = 0;
    for (int j = 0; j < n; ++j) place += sh.keys[j] > key;
    if (place < K) sh.top[place] = key;
  }
  __syncthreads();
}

// The row's from its CTAs' lists, into sh.all of the first CTA.
template <int kThreads>
__device__ __forceinline__ void join_tops(int K, int ctas, int rank, TopShared& sh) {
  ptx::cluster_sync_all();
  if (rank == 0) {
    for (int i = threadIdx.x; i < ctas * K; i += kThreads) {
      const uint32_t from = ptx::map_to_cta(ptx::smem_u32(sh.top), (uint32_t)(i / K)) + (uint32_t)(i % K) * 8u;
      unsigned long long key;
      asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(key) : "r"(from) : "memory");
      sh.keys[i] = key;
    }
    if (threadIdx.x < K) sh.all[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < ctas * K; i += kThreads) {
      const unsigned long long key = sh.keys[i];
      if (key == 0) continue;
      int place = i % K;                                      // larger ones in its own list, and in the others
      for (int r = 0; r < ctas; ++r) {
        if (r == i / K) continue;
        int above = 0;
        for (int step = kMaxTop; step > 0; step >>= 1)
          if (above + step <= K && sh.keys[r * K + above + step - 1] > key) above += step;
        place += above;
      }
      if (place < K) sh.all[place] = key;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------- log probabilities
struct LogprobArgs {
  const void* z;
  int64_t ld;
  int V, ctas, K;
  float c2;                   // scale log2(e)
  const int32_t* ids;
  float* logp;
  float* entropy;
  float* lse;
  int32_t* top_ids;
  float* top_logp;
};

// ln p of a logit; nothing is left of a row whose largest logit is masked.
__device__ __forceinline__ float log_p(float x, const Stat& a, float c2, float log2_s) {
  if (isnan(a.s)) return NAN;
  if (!(x > kMasked)) return isnan(x) ? NAN : -INFINITY;
  return kLn2 * (fmaf(x, c2, -a.mc) - log2_s);
}

template <typename T, bool kEntropy, bool kTop, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
logprobs_kernel(const LogprobArgs g) {
  __shared__ RowShared sh;
  __shared__ typename std::conditional<kTop, TopShared, int>::type top;
  after_previous();
  const int rank = (int)(blockIdx.x % (unsigned)g.ctas);
  const int64_t n = blockIdx.x / (unsigned)g.ctas;
  const Row<T> row(reinterpret_cast<const T*>(g.z), n, g.ld, g.V, rank, g.ctas);
  int id = -1;
  float z_id = 0.f;
  if (rank == 0 && threadIdx.x == 0 && g.ids != nullptr) {
    id = load_near(g.ids + n);
    if (id >= 0 && id < g.V) z_id = Elem<T>::load(row.z + id);
  }
  float mine;
  const Stat a = row_stat<T, kEntropy, kThreads>(row, g.c2, g.ctas, sh, mine);
  const float log2_s = log2f(a.s);
  if (rank == 0 && threadIdx.x == 0) {
    const bool none = a.m <= kMasked && !isnan(a.s);
    if (g.ids != nullptr) g.logp[n] = id < 0 ? 0.f : id >= g.V ? NAN : log_p(z_id, a, g.c2, log2_s);
    if (g.lse != nullptr) g.lse[n] = none ? -INFINITY : isnan(a.s) ? NAN : kLn2 * (a.mc + log2_s);
    if (kEntropy) g.entropy[n] = none ? 0.f : kLn2 * (log2_s - a.t / a.s);
  }
  if constexpr (kTop) {
    const bool bad = isnan(a.s);                              // (the same in all CTAs of the row)
    if (!bad) {
      top_of_part<T, kThreads>(row, g.K, mine, top);
      if (g.ctas > 1) join_tops<kThreads>(g.K, g.ctas, rank, top);
    }
    if (rank == 0 && (int)threadIdx.x < g.K) {
      const unsigned long long key = bad ? 0 : g.ctas > 1 ? top.all[threadIdx.x] : top.top[threadIdx.x];
      const int64_t at = n * g.K + threadIdx.x;
      g.top_ids[at] = key == 0 ? -1 : (int)(0xFFFFFFFFu - (uint32_t)key);
      g.top_logp[at] = bad ? NAN : key == 0 ? -INFINITY : log_p(of_order((uint32_t)(key >> 32)), a, g.c2, log2_s);
    }
  }
  if (g.ctas > 1) {
    __syncwarp();
    ptx::cluster_sync_all();                                  // nobody leaves while its shared memory is read
  }
}

// ---------------------------------------------------------------------------------------------- distillation
struct DistillArgs {
  const void* z;
  int64_t ld;
  int V, ctas, K;
  float c2, scale;
  const int32_t* ids;
  const float* top;
  const float* weights;
  float* loss;
  void* grad;
  int64_t ldg;
};

struct DistillShared {
  int id[kMaxTop];
  float t[kMaxTop], z[kMaxTop], p[kMaxTop];
  float loss;
  int teacher;                // 0: the row has none, 1: it has, 2: an id outside of the vocabulary
};

template <typename T, bool kGrad, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
distill_kernel(const DistillArgs g) {
  constexpr int kVec = Elem<T>::kVec;
  __shared__ RowShared sh;
  __shared__ DistillShared d;
  after_previous();
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = (int)(blockIdx.x % (unsigned)g.ctas);
  const int64_t n = blockIdx.x / (unsigned)g.ctas;
  const Row<T> row(reinterpret_cast<const T*>(g.z), n, g.ld, g.V, rank, g.ctas);
  T* grad = kGrad ? reinterpret_cast<T*>(g.grad) + n * g.ldg : nullptr;
  const bool aligned = kGrad && ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.z)) & 15u) == 0;
  auto store = [&](int i, const float (&f)[kVec]) {
    if (aligned && row.whole(i)) {
      *reinterpret_cast<uint4*>(grad + row.first(i)) = Elem<T>::pack(f);
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (row.first(i) + j >= 0 && row.first(i) + j < row.V) Elem<T>::store(grad + row.first(i) + j, f[j]);
    }
  };
  auto store_zeros = [&]() {
    float f[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) f[j] = 0.f;
    for (int i = row.lo + tid; i < row.hi; i += kThreads) store(i, f);
  };
  const float w = g.weights != nullptr ? load_near(g.weights + n) : 1.f;
  if (w == 0.f) {                                             // the same for all CTAs of the row
    if (rank == 0 && tid == 0) g.loss[n] = 0.f;
    if (kGrad) store_zeros();
    return;
  }
  // the teacher's places, and the student's logits there: read before a gradient may be written over them
  if (tid < g.K) {
    const int id = load_near(g.ids + n * g.K + tid);
    d.id[tid] = id;
    d.t[tid] = load_near(g.top + n * g.K + tid);
    d.z[tid] = id >= 0 && id < g.V ? Elem<T>::load(row.z + id) : kMasked;
  }
  float mine;
  const Stat a = row_stat<T, false, kThreads>(row, g.c2, g.ctas, sh, mine);
  if (tid < 32) {
    // p = softmax over the places: a lane has every 32nd
    constexpr int kPer = kMaxTop / 32;
    const float log2_s = log2f(a.s);
    float x[kPer], top = kMasked;
    bool outside = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = lane + 32 * k, id = i < g.K ? d.id[i] : -1;
      outside |= id >= g.V;
      x[k] = id >= 0 ? max_nan(d.t[i], kMasked) : kMasked;
      top = fmaxf(top, x[k]);
    }
    bool any = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) any |= !(x[k] <= kMasked);  // (a NaN counts)
    const int teacher = __any_sync(0xFFFFFFFFu, outside) ? 2 : __any_sync(0xFFFFFFFFu, any) ? 1 : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float tc = top * g.c2;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) sum += x[k] <= kMasked ? 0.f : exp2_fast(fmaf(x[k], g.c2, -tc));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const float log2_t = log2f(sum);
    float loss = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = lane + 32 * k;
      if (i >= g.K) continue;
      const float dt = fmaf(x[k], g.c2, -tc), p = x[k] <= kMasked ? 0.f : __fdiv_rn(exp2_fast(dt), sum);
      d.p[i] = p;
      if (p == 0.f) continue;
      const float z = d.z[i];
      loss += z <= kMasked ? INFINITY : p * ((dt - fmaf(z, g.c2, -a.mc)) + (log2_s - log2_t));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xFFFFFFFFu, loss, o);
    if (lane == 0) {
      d.teacher = teacher;
      if (rank == 0) g.loss[n] = teacher == 0 ? 0.f : teacher == 2 || isnan(a.s) ? NAN : w * (kLn2 * loss);
    }
  }
  if constexpr (kGrad) {
    __syncthreads();
    const bool bad = d.teacher == 2 || isnan(a.s);
    if (d.teacher == 0 || (!bad && a.m <= kMasked)) {
      store_zeros();
    } else {
      const float gp = w * g.scale, gq = bad ? NAN : gp / a.s;
      const f32x2 cc = pair_of(g.c2, g.c2), minus = pair_of(-a.mc, -a.mc);
      for (int i0 = row.lo + tid; i0 < row.hi; i0 += kBatch * kThreads) {
        uint4 v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) v[u] = i0 + u * kThreads < row.hi ? row.load(i0 + u * kThreads) : row.none();
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (i0 + u * kThreads >= row.hi) continue;
          f32x2 x[Elem<T>::kPairs];
          Elem<T>::pairs(Elem<T>::clamp(v[u]), x);
          float f[kVec];
#pragma unroll
          for (int j = 0; j < Elem<T>::kPairs; ++j) {
            const float2 e = halves(pfma(x[j], cc, minus));
            f[2 * j] = exp2_fast(e.x) * gq;
            f[2 * j + 1] = exp2_fast(e.y) * gq;
          }
          store(i0 + u * kThreads, f);
        }
      }
      __syncthreads();
      // the teacher's places of this CTA's part, after the barrier: each with all of its p, in the order of the places
      if (tid < g.K && d.id[tid] >= 0 && d.id[tid] < g.V) {
        const int id = d.id[tid], i = (id + row.off) / kVec;
        if (i >= row.lo && i < row.hi) {
          float p = 0.f;
          for (int k = 0; k < g.K; ++k) p += d.id[k] == id ? d.p[k] : 0.f;
          Elem<T>::store(grad + id, exp2_fast(fmaf(max_nan(d.z[tid], kMasked), g.c2, -a.mc)) * gq - gp * p);
        }
      }
    }
  }
  if (g.ctas > 1) {
    __syncwarp();
    ptx::cluster_sync_all();                                  // nobody leaves while its shared memory is read
  }
}

// ---------------------------------------------------------------------------------------------- launches
// CTAs of 128 threads for rows of up to 32 KB, of which an SM runs eight at a time, of 512 for longer ones, two at a time.  Rows that
// are too few for all SMs are shared by the CTAs of a cluster, as long as each thread has a vector; and with `again` (the row is read
// a second time) so that the rows under way at one time take no more than a third of the second-level cache.
constexpr int64_t kShortRow = 32 << 10, kRowsUnderWay = 40 << 20;
struct Plan {
  int threads, ctas;
};
Plan plan_rows(int64_t N, int64_t V, int64_t size, bool again, int sms) {
  Plan p;
  p.threads = V * size <= kShortRow ? 128 : 512;
  p.ctas = 1;
  const int64_t slots = (int64_t)sms * (1024 / p.threads), row = V * size;
  auto wanted = [&] {
    return N * p.ctas * 2 <= slots || (again && (N * p.ctas < slots ? N : slots / p.ctas) * row > kRowsUnderWay);
  };
  while (p.ctas < kMaxCluster && row >= (int64_t)2 * p.ctas * p.threads * 16 && wanted()) p.ctas *= 2;
  return p;
}

}  // namespace

int launch_token_logprobs(const void* logits, int f32, int64_t N, int64_t V, int64_t ld, float scale, const int32_t* ids, int K,
                          float* logp, float* entropy, float* lse, int32_t* top_ids, float* top_logp, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  const Plan p = plan_rows(N, V, f32 ? 4 : 2, false, sms);
  LogprobArgs g{};
  g.z = logits; g.ld = ld; g.V = (int)V; g.ctas = p.ctas; g.K = K; g.c2 = scale * kLog2e;
  g.ids = ids; g.logp = logp; g.entropy = entropy; g.lse = lse; g.top_ids = top_ids; g.top_logp = top_logp;
  auto run = [&](auto kernel) { return launch_next(kernel, dim3((unsigned)(N * p.ctas)), p.threads, 0, (unsigned)p.ctas, st, g); };
  auto of_type = [&](auto type, auto threads) {
    using T = decltype(type);
    constexpr int kThreads = decltype(threads)::value;
    if (entropy != nullptr) return K > 0 ? run(logprobs_kernel<T, true, true, kThreads>) : run(logprobs_kernel<T, true, false, kThreads>);
    return K > 0 ? run(logprobs_kernel<T, false, true, kThreads>) : run(logprobs_kernel<T, false, false, kThreads>);
  };
  const std::integral_constant<int, 128> few;
  const std::integral_constant<int, 512> many;
  if (f32) return p.threads == 128 ? of_type(0.f, few) : of_type(0.f, many);
  return p.threads == 128 ? of_type((uint16_t)0, few) : of_type((uint16_t)0, many);
}

int launch_distill_loss(const void* logits, int f32, int64_t N, int64_t V, int64_t ld, float scale, const int32_t* top_ids,
                        const float* top_logits, int K, const float* weights, float* loss, void* grad, int64_t ldg, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  const Plan p = plan_rows(N, V, f32 ? 4 : 2, grad != nullptr, sms);
  DistillArgs g{};
  g.z = logits; g.ld = ld; g.V = (int)V; g.ctas = p.ctas; g.K = K; g.c2 = scale * kLog2e; g.scale = scale;
  g.ids = top_ids; g.top = top_logits; g.weights = weights; g.loss = loss; g.grad = grad; g.ldg = ldg;
  auto run = [&](auto kernel) { return launch_next(kernel, dim3((unsigned)(N * p.ctas)), p.threads, 0, (unsigned)p.ctas, st, g); };
  auto of_type = [&](auto type) {
    using T = decltype(type);
    if (grad != nullptr) return p.threads == 128 ? run(distill_kernel<T, true, 128>) : run(distill_kernel<T, true, 512>);
    return p.threads == 128 ? run(distill_kernel<T, false, 128>) : run(distill_kernel<T, false, 512>);
  };
  return f32 ? of_type(0.f) : of_type((uint16_t)0);
}

}  // namespace tlq
