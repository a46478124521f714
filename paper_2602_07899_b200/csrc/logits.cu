// A model's logits, read once: log probabilities of given tokens with entropy and the largest alternatives, and the distillation loss
// on a teacher's top logits with its gradient.
//
//   d_v = scale log2(e) (z_v - m),  S = sum 2^d_v,  T = sum 2^d_v d_v   (m: the largest z_v)
//   lse = scale m + ln S,  ln p_v = ln2 (d_v - log2 S),  entropy = ln S - ln2 T / S,
//   grad_v = w scale (2^d_v / S - sum of the teacher's p at v).
//
// Maximum and sums run along in one pass (each thread with a maximum of its own, looked at once for a batch of vectors), so that a row is
// read from memory once.  Bound by memory; the exponentials take 3/4 of that time (16 bits).  4096 x 131072 of 16 bits, which a copy's rate
// reads in 166 us: log probabilities 177, with 64 alternatives 226, the distillation loss 175, with the gradient (333) 405.
//  - Every warp has slots of shared memory of its own, into which it has pieces of the rows copied ahead of time, the next row's too, so
//    that the memory has work while the CTA joins its sums, looks for the largest or writes; no warp waits for another but at a row's end.
//  - The gradient needs the row a second time, and gets it from the second-level cache: a CTA has an SM to itself, and rows are shared by
//    the CTAs of a cluster where those under way at one time would not stay there.  Both times come through the same slots.
//  - The largest K: every thread notes the largest of each run of its vectors.  The K-th largest of what the threads have seen is a bound
//    below which nothing is wanted, and only the runs that reach it are looked through again: little more than K of them.
//
// Rows may begin at any element: vectors of 16 bytes lie on the memory's own grid, and what belongs to a neighbour is masked.  (16 bytes
// at a multiple of 16 that hold an element of the row lie in the row's own memory page.)
#include <type_traits>

#include "pairs.cuh"
#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kMaxTop = TLQ_MAX_TOP;
constexpr int kBatch = 4;                 // vectors that a thread works on at a time
// Rows over 16 KB: CTAs of 256 threads, four to an SM, or of 256 to 1024 for the gradient; a warp has slots of kBatch vectors for each lane.
constexpr int kShort = 128, kLong = 256;
constexpr int kSlotsOnce = 2, kSlotsTwice = 3;            // (the latter for CTAs of 1024 threads: 405 us against 412; of 256 and 512 two are better)
constexpr int kRuns = 16;                 // a thread's batches b, b + kRuns, ... are a run, which has a maximum of its own
constexpr int kCandidates = kMaxCluster * kMaxTop;       // logits that may be among the largest: those of eight lists at least
constexpr int64_t kShortRow = 16 << 10;   // bytes of rows that CTAs of kShort threads read straight from memory
constexpr int kShortVectors = kShortRow / 16 + 1;
constexpr float kMasked = -1.2676506002282294e30f;       // -2^100: logits from here down have probability 0
constexpr uint32_t kMaskedPair = 0xF180F180u;            // the same, twice in bf16

using f32x2 = pair2;
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
// All ones in the halves of a that are no less than those of b, as bf16; b of the upper half of a float, twice.
__device__ __forceinline__ uint32_t at_least(uint32_t a, uint32_t b) {
  return __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
}
__device__ __forceinline__ uint32_t reach_word(float least) { return (__float_as_uint(least) >> 16) * 0x10001u; }

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
  __device__ static float get(uint16_t v) { return bf16_bits_to_float(v); }
  __device__ static void store(uint16_t* p, float f) {
    const __nv_bfloat16 v = __float2bfloat16_rn(f);
    *p = *reinterpret_cast<const uint16_t*>(&v);
  }
  // Four words of a vector, each no less than the mask's value.
  __device__ static uint4 clamp(const uint4& v) {
    return make_uint4(max_bf16x2(v.x, kMaskedPair), max_bf16x2(v.y, kMaskedPair), max_bf16x2(v.z, kMaskedPair), max_bf16x2(v.w, kMaskedPair));
  }
  template <int n>
  __device__ static float largest(const uint4 (&v)[n]) {
    uint32_t m = max_bf16x2(max_bf16x2(v[0].x, v[0].y), max_bf16x2(v[0].z, v[0].w));
#pragma unroll
    for (int u = 1; u < n; ++u) m = max_bf16x2(m, max_bf16x2(max_bf16x2(v[u].x, v[u].y), max_bf16x2(v[u].z, v[u].w)));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  __device__ static void pairs(const uint4& v, f32x2 (&x)[kPairs]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  // A bit for each element that is no less than `least`, and which element (of all in v) a bit stands for.
  template <int n>
  __device__ static uint32_t reach(const uint4 (&v)[n], float least) {
    const uint32_t b = reach_word(least);
    uint32_t hit = 0;
#pragma unroll
    for (int u = 0; u < n; ++u) {
      hit |= at_least(v[u].x, b) & (0x10001u << (4 * u));
      hit |= at_least(v[u].y, b) & (0x10001u << (4 * u + 1));
      hit |= at_least(v[u].z, b) & (0x10001u << (4 * u + 2));
      hit |= at_least(v[u].w, b) & (0x10001u << (4 * u + 3));
    }
    return hit;
  }
  __device__ static int element(int bit) { return 2 * (bit & 15) + (bit >> 4); }
  __device__ static float value(uint32_t word, int bit) { return __uint_as_float(bit < 16 ? word << 16 : word & 0xFFFF0000u); }
  __device__ static void mask(uint32_t addr) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"((uint16_t)kMaskedPair) : "memory"); }
  __device__ static uint32_t masked() { return kMaskedPair; }
  __device__ static uint4 pack(const f32x2 (&x)[kPairs]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = halves(x[i]);
      const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static void put_into(uint16_t* p, const uint4& v, int j) { *p = (uint16_t)((&v.x)[j >> 1] >> (j & 1) * 16); }
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
  __device__ static float get(float v) { return v; }
  __device__ static void store(float* p, float f) { *p = f; }
  __device__ static uint4 clamp(const uint4& v) {
    auto c = [](uint32_t w) { return __float_as_uint(max_nan(__uint_as_float(w), kMasked)); };
    return make_uint4(c(v.x), c(v.y), c(v.z), c(v.w));
  }
  template <int n>
  __device__ static float largest(const uint4 (&v)[n]) {
    float m = kMasked;
#pragma unroll
    for (int u = 0; u < n; ++u)
      m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[u].x), __uint_as_float(v[u].y)), fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
    return m;
  }
  __device__ static void pairs(const uint4& v, f32x2 (&x)[kPairs]) {
    x[0] = pair_of(__uint_as_float(v.x), __uint_as_float(v.y));
    x[1] = pair_of(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  template <int n>
  __device__ static uint32_t reach(const uint4 (&v)[n], float least) {
    uint32_t hit = 0;
#pragma unroll
    for (int u = 0; u < n; ++u) {
      hit |= __uint_as_float(v[u].x) >= least ? 1u << (4 * u) : 0u;
      hit |= __uint_as_float(v[u].y) >= least ? 2u << (4 * u) : 0u;
      hit |= __uint_as_float(v[u].z) >= least ? 4u << (4 * u) : 0u;
      hit |= __uint_as_float(v[u].w) >= least ? 8u << (4 * u) : 0u;
    }
    return hit;
  }
  __device__ static int element(int bit) { return bit; }
  __device__ static float value(uint32_t word, int) { return __uint_as_float(word); }
  __device__ static void mask(uint32_t addr) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(kMasked) : "memory"); }
  __device__ static uint32_t masked() { return __float_as_uint(kMasked); }
  __device__ static uint4 pack(const f32x2 (&x)[kPairs]) {
    const float2 a = halves(x[0]), b = halves(x[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
  __device__ static void put_into(float* p, const uint4& v, int j) { *p = __uint_as_float((&v.x)[j]); }
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
  // A piece from vector p on has no end of the row in it.
  __device__ bool inside(int p) const { return first(p) >= 0 && p + 32 * kBatch < hi; }
  // Vector i as it came, with what does not belong to the row masked.
  __device__ uint4 own(uint4 v, int i) const {
    if (!whole(i)) {
#pragma unroll
      for (int j = 0; j < Elem<T>::kVec; ++j)
        if (first(i) + j < 0 || first(i) + j >= V) Elem<T>::put(v, j, kMasked);
    }
    return v;
  }
  __device__ uint4 load(int i) const { return own(load_once(z + first(i)), i); }
};

struct Rows {                 // of one CTA: first, first + step, ...
  const void* z;
  int64_t ld, first, step, N;
  int V, rank, ctas;
  const float* weights;       // rows of weight 0 are not read, or null
};
// A warp's pieces of 32 kBatch vectors, row after row, in slots of its own: of each part of a row every (warps)th piece; with kAgain every row
// a second time before the next.
constexpr int kPiece = 32 * kBatch;
constexpr uint32_t kPieceBytes = kPiece * 16;
template <typename T, int kThreads, int kSlots, bool kAgain>
struct Pieces {
  const Rows& r;
  int64_t n;                  // what comes next: `left` vectors from src on, of row n
  const T* src;
  int left;
  bool second;
  float w, w_next;            // (read a row ahead)
  int slot;                   // what is read next
  uint32_t data, bar, phase;  // ... this lane's first vector of it, its barrier, how often it was read

  __device__ Pieces(const Rows& rows, const void* smem, uint64_t* barriers, int* abort)
      : r(rows), n(r.first), left(0), second(false), w(1.f), w_next(1.f), slot(0), phase(0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    data = ptx::smem_u32(smem) + (uint32_t)(warp * kSlots) * kPieceBytes + lane * 16u;
    bar = ptx::smem_u32(barriers + warp * kSlots);
    if (lane == 0) {
      for (int k = 0; k < kSlots; ++k) ptx::mbar_init(bar + 8u * k, 1);
      ptx::fence_barrier_init();
    }
    if (threadIdx.x == 0) *abort = 0;
    __syncthreads();
    begin();
    if (r.weights != nullptr) {
      // whether the first row counts is a trip to memory away: its first pieces are sent for meanwhile, as far as the second-level cache
      const int there = left - lane * kThreads * kBatch;
      if (lane < kSlots && there > 0)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;"
                     ::"l"(src + lane * kThreads * kBatch * Elem<T>::kVec), "r"((uint32_t)min(kPiece, there) * 16u) : "memory");
      w = load_near(r.weights + n);
      if (n + r.step < r.N) w_next = load_near(r.weights + n + r.step);
      if (w == 0.f) left = 0;
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) fill(data + k * kPieceBytes, bar + 8u * k);
  }
  __device__ void begin() {
    const Row<T> row(reinterpret_cast<const T*>(r.z), n, r.ld, r.V, r.rank, r.ctas);
    const int first = row.lo + (int)(threadIdx.x >> 5) * kPiece;
    src = row.z + row.first(first);
    left = w == 0.f ? 0 : row.hi - first;
  }
  // On to the row that comes next, or to the same one again; false where there is none.
  __device__ bool go_on() {
    do {
      if (n >= r.N) return false;
      if (kAgain && !second && w != 0.f) {
        second = true;
      } else {
        second = false;
        n += r.step;
        if (n >= r.N) return false;
        if (r.weights != nullptr) {
          w = w_next;
          if (n + r.step < r.N) w_next = load_near(r.weights + n + r.step);
        }
      }
      begin();
    } while (left <= 0);
    return true;
  }
  // The next piece into a slot; nothing where there is none.
  __device__ void fill(uint32_t to, uint32_t to_bar) {
    if (left <= 0 && !go_on()) return;
    if ((threadIdx.x & 31) == 0) {
      const uint32_t bytes = (uint32_t)min(kPiece, left) * 16u;
      ptx::mbar_expect_tx(to_bar, bytes);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   ::"r"(to), "l"(src), "r"(bytes), "r"(to_bar) : "memory");
    }
    src += kThreads * kBatch * Elem<T>::kVec;
    left -= kThreads * kBatch;
  }
  // The lane's vectors of the piece that is read next, whose slot then takes another one; false when it did not come within the limit of
  // a wait, which no correct run reaches.  (A load from shared memory that is still on its way may be overtaken by a copy into the same
  // place: the fence waits for it.)
  // With `row`, what is not the row's is masked: in its place in shared memory, so that the pieces inside of a row, which are almost all, are
  // not held up by it.
  __device__ bool next(uint4 (&v)[kBatch], int* abort, const Row<T>* row, int i) {
    const bool ok = ptx::mbar_try_wait(bar, phase) || ptx::mbar_wait(bar, phase, abort);
    if (row != nullptr && !row->inside(i - (int)(threadIdx.x & 31))) {
      for (int u = 0; u < kBatch; ++u) {
        const int k = i + u * 32;
        if (k < row->hi && row->whole(k)) continue;
        for (int j = 0; j < Elem<T>::kVec; ++j)
          if (k >= row->hi || row->first(k) + j < 0 || row->first(k) + j >= row->V) Elem<T>::mask(data + u * 512u + j * (uint32_t)sizeof(T));
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[u].x), "=r"(v[u].y), "=r"(v[u].z), "=r"(v[u].w)
                   : "r"(data + u * 512u) : "memory");
    ptx::fence_proxy_async();
    __syncwarp();
    fill(data, bar);
    data += kPieceBytes;
    bar += 8u;
    if (++slot == kSlots) {
      slot = 0;
      phase ^= 1u;
      data -= kSlots * kPieceBytes;
      bar -= 8u * kSlots;
    }
    return ok;
  }
};
// Where a thread's vectors of a row are: the first of its batch number b, and how far apart those of a batch are.
template <int kThreads>
__device__ __forceinline__ int first_vector(int lo, int b) {
  return lo + b * kThreads * kBatch + (kThreads == kShort ? (int)threadIdx.x : (int)(threadIdx.x >> 5) * 32 * kBatch + (int)(threadIdx.x & 31));
}
template <int kThreads>
__device__ __forceinline__ constexpr int vector_step() { return kThreads == kShort ? kShort : 32; }

// ---------------------------------------------------------------------------------------------- maximum and sums
// The factor of a logit's distance from the row's largest, m, to the exponent of 2: c = scale log2(e).  d = fma(z, c, -mc) with mc = m c rounded
// is off by that rounding, the same for all logits of the row, which drops out of everything as long as 2^d stays in range: up to
// |m c| = 2^31, where it is 64.  Beyond, any other logit is 2^-24 m away from m, over 128 in the exponent, and counts nothing; with
// the power of 2 above c for the factor m c is exact, and d is 0 for m itself.  (A quarter of that where m c would leave the 32-bit range, which
// scale m does not.)
// Sums whose largest logits have different factors are joined with the larger one's: their logits are 2^-24 2^31 apart at least, so that the
// sum of the smaller one, rounded by 64 or not, counts nothing.
struct Factors {
  float near, far;            // c, and the power of 2 above it
};
Factors factors_of(float scale) {
  const float c = scale * kLog2e;
  int e;
  frexpf(c, &e);              // c = [0.5, 1) 2^e
  return Factors{c, ldexpf(1.f, e)};
}
__device__ __forceinline__ bool is_near(float m, const Factors& f) { return fabsf(m * f.near) < 2147483648.f; }
__device__ __forceinline__ float factor(float m, const Factors& f) {
  float c = f.near;
  if (__builtin_expect(!is_near(m, f), 0)) c = m * f.far < INFINITY ? f.far : 0.25f * f.far;
  return c;
}
constexpr float kFar = -16384.f;          // 2^kFar is 0, and no product with it leaves the range
struct Stat {
  float m, mc;                // the largest logit, and that times its factor, rounded
  float s, t;                 // sums of 2^d and of 2^d d
};
__device__ __forceinline__ Stat empty_stat(const Factors& f) { return Stat{kMasked, kMasked * f.far, 0.f, 0.f}; }
// log2 of the sum of 2^((z - m) c): without the rounding of mc.
__device__ __forceinline__ float log2_sum(const Stat& a, const Factors& f) { return log2f(a.s) - fmaf(a.m, factor(a.m, f), -a.mc); }

// Over the lanes of a warp, in a fixed order; every lane gets the same.
__device__ __forceinline__ Stat merge_warp(const Stat& a, const Factors& of) {
  Stat r;
  r.m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.m = fmaxf(r.m, __shfl_xor_sync(0xFFFFFFFFu, r.m, o));
  const float c = factor(r.m, of);
  r.mc = __fmul_rn(r.m, c);               // (rounded as it is everywhere else, not within the difference)
  const float d = fmaxf(__fmul_rn(a.m, c) - r.mc, kFar), f = exp2_fast(d);
  r.s = a.s * f;
  r.t = fmaf(r.s, d, a.t * f);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, o);
    r.t += __shfl_xor_sync(0xFFFFFFFFu, r.t, o);
  }
  return r;
}

struct RowShared {            // of two rows in turn: a warp may be a row ahead of one that still reads
  Stat warps[2][32];
  float cta[2][4];            // what the other CTAs of the cluster read
};
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// A thread's own maximum and sums as its vectors come.
template <typename T, bool kEntropy>
struct Running {
  const Factors& of;
  float m, mc;
  f32x2 cc, s, t;
  __device__ explicit Running(const Factors& f) : of(f), m(kMasked), mc(kMasked * f.far), cc(pair_of(f.far, f.far)), s(pair_of(0.f, 0.f)), t(s) {}
  // Returns the vectors' largest.
  template <int n>
  __device__ float add(const uint4 (&v)[n]) {
    const float largest = Elem<T>::largest(v), top = fmaxf(m, largest);        // (a NaN passes by here and shows in the sum)
    if (top > m) {
      const float of_top = factor(top, of), c = __fmul_rn(top, of_top), d = fmaxf(__fmul_rn(m, of_top) - c, kFar), f = exp2_fast(d);
      cc = pair_of(of_top, of_top);
      s = pmul(s, pair_of(f, f));
      if (kEntropy) t = pfma(s, pair_of(d, d), pmul(t, pair_of(f, f)));
      m = top;
      mc = c;
    }
    const f32x2 minus = pair_of(-mc, -mc);
#pragma unroll
    for (int u = 0; u < n; ++u) {
      f32x2 x[Elem<T>::kPairs];
      Elem<T>::pairs(v[u], x);
#pragma unroll
      for (int j = 0; j < Elem<T>::kPairs; ++j) {
        const f32x2 d = pfma(x[j], cc, minus);
        const float2 d2 = halves(d);
        const f32x2 e = pair_of(exp2_fast(d2.x), exp2_fast(d2.y));
        s = padd(s, e);
        if (kEntropy) t = pfma(e, d, t);
      }
    }
    return largest;
  }
  __device__ Stat stat() const { return Stat{m, mc, halves(s).x + halves(s).y, halves(t).x + halves(t).y}; }
};

// A batch of vectors from i on, from the warp's slot or from memory, with what is not the row's masked, and with kClamp no value below the
// mask's (which the entropy's terms 0 x -infinity need; without them the sums take any).
template <typename T, int kThreads, bool kClamp, typename P, typename R>
__device__ __forceinline__ void read_batch(const Row<T>& row, int i, P& pieces, int* abort, uint4 (&v)[kBatch], R& run) {
  constexpr int kStep = vector_step<kThreads>();
  if constexpr (kThreads != kShort) {
    if (!pieces.next(v, abort, &row, i)) run.s = pair_of(NAN, NAN);
  } else {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = i + u * kStep < row.hi ? row.load(i + u * kStep) : row.none();
  }
  if (kClamp) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = Elem<T>::clamp(v[u]);
  }
}

// Maximum and sums of the whole row from those of the threads, the same in every thread of every CTA of it.  The sum is no number where the
// row has no distribution: where it has a NaN or +infinity, or its largest logit leaves the range when multiplied by scale.
template <int kThreads>
__device__ __forceinline__ Stat join_row(Stat a, const Factors& f, float scale, int ctas, RowShared& sh, int parity) {
  constexpr int kWarps = kThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  a = merge_warp(a, f);
  if (lane == 0) sh.warps[parity][warp] = a;
  __syncthreads();
  a = merge_warp(lane < kWarps ? sh.warps[parity][lane] : empty_stat(f), f);
  if (ctas > 1) {
    if (threadIdx.x == 0) {
      sh.cta[parity][0] = a.m; sh.cta[parity][1] = a.mc; sh.cta[parity][2] = a.s; sh.cta[parity][3] = a.t;
    }
    __syncwarp();
    ptx::cluster_sync_all();
    a = empty_stat(f);
    if (lane < ctas) {
      const uint32_t from = ptx::map_to_cta(ptx::smem_u32(sh.cta[parity]), (uint32_t)lane);
      a.m = ld_cluster_f32(from); a.mc = ld_cluster_f32(from + 4); a.s = ld_cluster_f32(from + 8); a.t = ld_cluster_f32(from + 12);
    }
    __syncwarp();
    a = merge_warp(a, f);
  }
  if (!(a.m * scale < INFINITY)) a.s = NAN;
  return a;
}

// ---------------------------------------------------------------------------------------------- the largest K
// Keys order as the logits do, and equal logits by their index, the lower one first; 0 is none.
__device__ __forceinline__ uint32_t in_order(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);                // (-0 is 0)
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o); }
// A bound, in the order of logits, that none masked reaches, and the logit that stands there.
__device__ __forceinline__ uint32_t above_mask(uint32_t order) { return max(order, in_order(kMasked) + 1u); }
__device__ __forceinline__ float least_of(uint32_t order) { return of_order(above_mask(order)); }
__device__ __forceinline__ unsigned long long key_of(float x, int index) {
  return ((unsigned long long)in_order(x) << 32) | (0xFFFFFFFFu - (uint32_t)index);
}

// What logits have to reach for a key of `least` or more: that key's logit up to its index, a larger one behind it.
template <typename T>
struct KeyBound {
  float least, larger;
  int last;
  __device__ explicit KeyBound(unsigned long long key)
      : least(least_of((uint32_t)(key >> 32))), larger(least_of((uint32_t)(key >> 32) + (sizeof(T) == 2 ? 0x10000u : 1u))),
        last((int)min(0xFFFFFFFFu - (uint32_t)key, 0x7FFFFFFFu)) {}
  __device__ float from(int index) const { return index > last ? larger : least; }
};

template <int kThreads>
struct TopShared {
  static constexpr bool kShortRows = kThreads == kShort;
  union {
    unsigned long long keys[kCandidates];
    uint32_t runs[kShortRows ? 1 : kRuns / 2][kThreads]; // upper halves of the largest logit of each thread's runs 2 j and 2 j + 1, until they are listed
  };
  unsigned long long top[kMaxTop];        // of this CTA's part, largest first
  unsigned long long all[kShortRows ? 1 : kMaxTop];      // of the row
  uint32_t bounds[kThreads / 32];
  uint4 row[kShortRows ? kShortVectors : 1];             // a short row
  uint16_t listed[kShortRows ? 1 : kCandidates];         // runs that reach the bound: run kThreads + thread
  int n_keys, n_listed;
};

// The K-th largest of the first n keys (n >= K).
template <int kThreads>
__device__ unsigned long long kth_key(const TopShared<kThreads>& sh, int n, int K) {
  unsigned long long bound = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const unsigned long long next = bound | (1ull << bit);
    int count = 0;
    for (int i = 0; i < n; i += kThreads) count += __syncthreads_count(i + (int)threadIdx.x < n && sh.keys[min(i + (int)threadIdx.x, n - 1)] >= next);
    if (count >= K) bound = next;
  }
  return bound;
}

// The largest K of n keys to their places, largest first: 32 at a time are put in order by a warp; a key's place is then the number of larger
// ones in every such list.
template <int kThreads>
__device__ __forceinline__ void place_keys(unsigned long long* keys, int n, int K, unsigned long long* places) {
  const int tid = threadIdx.x, lane = tid & 31, lists = (n + 31) / 32;
  for (int l = tid >> 5; l < lists; l += kThreads / 32) {
    unsigned long long key = l * 32 + lane < n ? keys[l * 32 + lane] : 0;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
      for (int step = size >> 1; step > 0; step >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, key, step);
        key = ((lane & step) == 0) == ((lane & size) == 0) ? max(key, other) : min(key, other);
      }
    keys[l * 32 + lane] = key;
  }
  __syncthreads();
  for (int i = tid; i < lists * 32; i += kThreads) {
    const unsigned long long key = keys[i];
    int place = i & 31;
    if (key == 0 || place >= K) continue;
    for (int l = 0; l < lists; ++l) {
      if (l == i >> 5) continue;
      int above = 0;
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
        if (keys[l * 32 + above + step - 1] > key) above += step;
      above += keys[l * 32 + above] > key;                    // (31 at most before this)
      place += above;
      if (place >= K) break;
    }
    if (place < K) places[place] = key;
  }
}

// Word `i` of four vectors, without a detour through memory.
__device__ __forceinline__ uint32_t word_of(const uint4 (&v)[4], int i) {
  auto pick = [](bool second, const uint4& a, const uint4& b) { return make_uint4(second ? b.x : a.x, second ? b.y : a.y, second ? b.z : a.z, second ? b.w : a.w); };
  const uint4 w = pick(i & 8, pick(i & 4, v[0], v[1]), pick(i & 4, v[2], v[3]));
  return (i & 2) ? ((i & 1) ? w.w : w.z) : ((i & 1) ? w.y : w.x);
}

// A bound that `share` lanes at least reach: the largest that is left, and with it all lanes that have it, until there are enough.
__device__ __forceinline__ uint32_t bound_of_lanes(uint32_t own, int share) {
  uint32_t bound = 0;
  for (int have = 0; have < share;) {
    bound = __reduce_max_sync(0xFFFFFFFFu, own);
    if (bound == 0) break;
    have += __popc(__ballot_sync(0xFFFFFFFFu, own == bound));
    own = own == bound ? 0u : own;
  }
  return bound;
}

// The largest K of this CTA's part of the row into sh.top.  `mine`: the largest logit of this thread's vectors; a run has up to `batches` batches.
template <typename T, int kThreads>
__device__ __forceinline__ void top_of_part(const Row<T>& row, int K, float mine, int runs, int batches, TopShared<kThreads>& sh) {
  const int tid = threadIdx.x;
  const bool any = first_vector<kThreads>(row.lo, 0) < row.hi;
  const uint32_t own = any ? in_order(mine) >> 16 : 0u;
  // A bound that K threads at least reach: in every warp its share of them does.  (None where fewer have
  // anything; the part is small then.)
  const int vectors = row.hi - row.lo, here = __popc(__ballot_sync(0xFFFFFFFFu, any));
  const int active = min(kThreads / 32, vectors / kPiece) * 32 + min(32, vectors % kPiece) * (vectors < kThreads * kBatch);
  const int share = max(1, (K * here + active - 1) / max(active, 1));
  uint32_t bound = bound_of_lanes(own, share);
  if ((tid & 31) == 0) sh.bounds[tid >> 5] = bound;
  if (tid == 0) sh.n_listed = 0;
  if (tid < K) sh.top[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kThreads / 32; ++k) bound = min(bound, sh.bounds[k]);
  if (any && own >= bound) {
    const uint32_t least = reach_word(least_of(bound << 16));
    uint32_t hit = 0;                                         // run 2 j: bit j, 2 j + 1: bit 16 + j
#pragma unroll
    for (int j = 0; j < kRuns / 2; ++j) hit |= at_least(sh.runs[j][tid], least) & (0x10001u << j);
    hit &= ((1u << (runs + 1) / 2) - 1u) | (((1u << runs / 2) - 1u) << 16);
    for (; hit != 0; hit &= hit - 1) {
      const int at = atomicAdd(&sh.n_listed, 1);
      if (at < kCandidates) sh.listed[at] = (uint16_t)((((__ffs(hit) - 1) & 15) * 2 + ((__ffs(hit) - 1) >> 4)) * kThreads + tid);
    }
  }
  if (tid == 0) sh.n_keys = 0;
  __syncthreads();
  // all of them where there are more than the list holds (equal logits in every run)
  const bool all = sh.n_listed > kCandidates;
  const int total = (all ? runs * kThreads : sh.n_listed) * batches;
  unsigned long long least = (unsigned long long)above_mask(bound << 16) << 32;
  // Where the bound is no higher than the mask, fewer than K may be above it: the part's first masked logits are wanted then, which
  // are among its first K.
  if (bound << 16 <= in_order(kMasked) && tid < K) {
    const int at = max(0, row.first(row.lo)) + tid;
    if (at < min(row.V, row.first(row.hi)) && !(Elem<T>::load(row.z + at) > kMasked)) sh.keys[atomicAdd(&sh.n_keys, 1)] = key_of(kMasked, at);
  }
  int n;
  while (true) {
    const KeyBound<T> above(least);
    for (int k = tid; k < total; k += kThreads) {
      const int entry = batches == 1 ? k : k / batches, which = all ? entry : sh.listed[entry], t = which % kThreads;
      const int i = row.lo + (which / kThreads + (k - entry * batches) * kRuns) * kThreads * kBatch + (kThreads == kShort ? t : (t >> 5) * kPiece + (t & 31));
      uint4 v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        v[u] = i + u * vector_step<kThreads>() < row.hi ? load_once(row.z + row.first(i + u * vector_step<kThreads>())) : row.none();
      for (uint32_t hit = Elem<T>::reach(v, above.from(row.first(i))); hit != 0; hit &= hit - 1) {
        const int bit = __ffs(hit) - 1, e = Elem<T>::element(bit), from = i + e / Elem<T>::kVec * vector_step<kThreads>(), at = row.first(from) + e % Elem<T>::kVec;
        if (at < 0 || at >= row.V || from >= row.hi) continue;
        const unsigned long long key = key_of(fmaxf(Elem<T>::value(word_of(v, bit & 15), bit), kMasked), at);
        if (key < least) continue;
        const int to = atomicAdd(&sh.n_keys, 1);
        if (to < kCandidates) sh.keys[to] = key;
        else k = total, hit = 1;                              // (no room: enough has been seen)
      }
    }
    __syncthreads();
    n = sh.n_keys;
    if (n <= kCandidates) break;
    least = kth_key<kThreads>(sh, kCandidates, K);            // more than there is room for: a higher bound, from those there was room for
    __syncthreads();
    if (tid == 0) sh.n_keys = 0;
    __syncthreads();
  }
  place_keys<kThreads>(sh.keys, n, K, sh.top);
  __syncthreads();
}

// The same of a short row, which the threads have left in sh.row.  What counts for the bound are the largest of the threads, or where there
// are hardly more of them than K those of the vectors, or else the elements: in every warp its share of them reaches its bound.
template <typename T>
__device__ __forceinline__ void top_of_short_row(const Row<T>& row, int K, float mine, TopShared<kShort>& sh) {
  constexpr int kVec = Elem<T>::kVec, kMine = (kShortVectors + kShort - 1) / kShort, kUnits = kMine > 2 * kVec ? kMine : 2 * kVec;
  static_assert(2 * kMaxTop <= 2 * kShort, "elements of two vectors of each thread at most");
  const int tid = threadIdx.x, vectors = row.hi - row.lo, active = min(vectors, kShort);
  uint32_t bound = 0;
  int units = __popc(__ballot_sync(0xFFFFFFFFu, tid < vectors));     // of the warp
  if (4 * K <= 3 * active) {
    bound = bound_of_lanes(tid < vectors ? in_order(mine) >> 16 : 0u, max(1, (K * units + active - 1) / active));
  } else {
    const bool fine = vectors < 2 * K;
    uint32_t unit[kUnits];
    units = 0;
#pragma unroll
    for (int q = 0; q < kUnits; ++q) unit[q] = 0;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      if (j * kShort >= vectors) continue;
      const bool in = j * kShort + tid < vectors;
      units += __popc(__ballot_sync(0xFFFFFFFFu, in));
      f32x2 x[Elem<T>::kPairs];
      Elem<T>::pairs(in ? sh.row[j * kShort + tid] : row.none(), x);
      float most = kMasked;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float2 h = halves(x[e >> 1]);
        const float z = (e & 1) ? h.y : h.x;
        most = fmaxf(most, z);
        if (fine && j < 2) unit[j < 2 ? j * kVec + e : 0] = in ? in_order(z) >> 16 : 0u;
      }
      if (!fine) unit[j] = in ? in_order(most) >> 16 : 0u;
    }
    const int share = max(1, (K * units + vectors - 1) / vectors), rows = (vectors + kShort - 1) / kShort, count = fine ? min(2, rows) * kVec : rows;
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t next = bound | (1u << bit);
      int reach = 0;
#pragma unroll
      for (int q = 0; q < kUnits; ++q)
        if (q < count) reach += __popc(__ballot_sync(0xFFFFFFFFu, unit[q] >= next));
      if (reach >= share) bound = next;
    }
  }
  if ((tid & 31) == 0) sh.bounds[tid >> 5] = units > 0 ? bound : 0xFFFFu;     // (a warp without any has no say)
  if (tid == 0) sh.n_keys = 0;
  if (tid < K) sh.top[tid] = 0;
  __syncthreads();
  bound = 0xFFFFu;
#pragma unroll
  for (int k = 0; k < kShort / 32; ++k) bound = min(bound, sh.bounds[k]);
  unsigned long long least = (unsigned long long)above_mask(bound << 16) << 32;
  if (bound << 16 <= in_order(kMasked) && tid < min(K, row.V)) {       // the first masked ones, as above
    const int e = tid + row.off;
    if (!(Elem<T>::get(reinterpret_cast<const T*>(sh.row)[e]) > kMasked)) sh.keys[atomicAdd(&sh.n_keys, 1)] = key_of(kMasked, tid);
  }
  int n;
  while (true) {
    const KeyBound<T> above(least);
    for (int j = tid; j < vectors; j += kShort) {
      const uint4 v[1] = {sh.row[j]};
      for (uint32_t hit = Elem<T>::reach(v, above.from(row.first(row.lo + j))); hit != 0; hit &= hit - 1) {
        const int e = Elem<T>::element(__ffs(hit) - 1), at = row.first(row.lo + j) + e;
        if (at < 0 || at >= row.V) continue;
        const unsigned long long key = key_of(Elem<T>::get(reinterpret_cast<const T*>(sh.row + j)[e]), at);
        if (key < least) continue;
        const int to = atomicAdd(&sh.n_keys, 1);
        if (to < kCandidates) sh.keys[to] = key;
        else j = vectors, hit = 1;
      }
    }
    __syncthreads();
    n = sh.n_keys;
    if (n <= kCandidates) break;
    least = kth_key<kShort>(sh, kCandidates, K);
    __syncthreads();
    if (tid == 0) sh.n_keys = 0;
    __syncthreads();
  }
  place_keys<kShort>(sh.keys, n, K, sh.top);
  __syncthreads();
}

// The row's from its CTAs' lists, into sh.all of the first CTA.
template <int kThreads>
__device__ __forceinline__ void join_tops(int K, int ctas, int rank, TopShared<kThreads>& sh) {
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
    place_keys<kThreads>(sh.keys, ctas * K, K, sh.all);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------- log probabilities
struct LogprobArgs {
  const void* z;
  int64_t N, ld;
  int V, ctas, K, batches;    // batches of a run
  float scale;
  Factors f;
  const int32_t* ids;
  float* logp;
  float* entropy;
  float* lse;
  int32_t* top_ids;
  float* top_logp;
};

// ln p of a logit; nothing is left of a row whose largest logit is masked.  (Not by way of log2 p, which may leave the range where ln p does
// not.)
__device__ __forceinline__ float log_p(float x, const Stat& a, float scale, float ln_s) {
  if (isnan(a.s)) return NAN;
  if (!(x > kMasked)) return isnan(x) ? NAN : -INFINITY;
  return fmaf(x - a.m, scale, -ln_s);
}

// Long rows come through slots, short ones straight from memory.
template <typename T, bool kEntropy, bool kTop, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
logprobs_kernel(const LogprobArgs g) {
  constexpr bool kSlots = kThreads != kShort;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ RowShared sh;
  __shared__ typename std::conditional<kTop, TopShared<kThreads>, int>::type top;
  __shared__ uint64_t barriers[kSlots ? kSlotsOnce * kThreads / 32 : 1];
  __shared__ int abort;
  after_previous();
  const int rank = (int)(blockIdx.x % (unsigned)g.ctas);
  const Rows rows{g.z, g.ld, blockIdx.x / (unsigned)g.ctas, gridDim.x / (unsigned)g.ctas, g.N, g.V, rank, g.ctas, nullptr};
  typename std::conditional<kSlots, Pieces<T, kThreads, kSlotsOnce, false>, int>::type pieces = [&] {
    if constexpr (kSlots) return Pieces<T, kThreads, kSlotsOnce, false>(rows, slots, barriers, &abort);
    else return 0;
  }();
  int parity = 0;
  for (int64_t n = rows.first; n < g.N; n += rows.step, parity ^= 1) {
    const Row<T> row(reinterpret_cast<const T*>(g.z), n, g.ld, g.V, rank, g.ctas);
    int id = -1;
    float z_id = 0.f;
    if (rank == 0 && threadIdx.x == 0 && g.ids != nullptr) {
      id = load_near(g.ids + n);
      if (id >= 0 && id < g.V) z_id = Elem<T>::load(row.z + id);
    }
    Running<T, kEntropy> run(g.f);
    int batch = 0;
    for (int i = first_vector<kThreads>(row.lo, 0); i - (kSlots ? (int)(threadIdx.x & 31) : (int)threadIdx.x) < row.hi; i += kBatch * kThreads) {
      uint4 v[kBatch];
      read_batch<T, kThreads, kEntropy>(row, i, pieces, &abort, v, run);
      const float largest = run.add(v);
      if constexpr (kTop && kSlots) {
        uint16_t* const at = reinterpret_cast<uint16_t*>(&top.runs[batch / 2 % (kRuns / 2)][threadIdx.x]) + batch % 2;
        float most = kEntropy ? largest : fmaxf(largest, kMasked);
        if (batch >= kRuns) most = fmaxf(most, bf16_bits_to_float(*at));
        *at = (uint16_t)(__float_as_uint(most) >> 16);
        ++batch;
      }
      if constexpr (kTop && !kSlots) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (i + u * kThreads < row.hi) top.row[i + u * kThreads - row.lo] = kEntropy ? v[u] : Elem<T>::clamp(v[u]);
      }
    }
    const Stat a = join_row<kThreads>(run.stat(), g.f, g.scale, g.ctas, sh, parity);
    const float ln_s = kLn2 * log2_sum(a, g.f);
    if (rank == 0 && threadIdx.x == 0) {
      const bool none = a.m <= kMasked && !isnan(a.s);
      if (g.ids != nullptr) g.logp[n] = id < 0 ? 0.f : id >= g.V ? NAN : log_p(z_id, a, g.scale, ln_s);
      if (g.lse != nullptr) g.lse[n] = none ? -INFINITY : isnan(a.s) ? NAN : fmaf(a.m, g.scale, ln_s);
      // (with the rounding of mc in both; where there is none t is 0, but for terms 0 x -infinity where d itself leaves the range)
      if (kEntropy) g.entropy[n] = none ? 0.f : kLn2 * (log2f(a.s) - (is_near(a.m, g.f) ? a.t / a.s : 0.f));
    }
    if constexpr (kTop) {
      const bool bad = isnan(a.s);                            // (the same in all CTAs of the row)
      if (!bad) {
        if constexpr (kSlots) top_of_part<T, kThreads>(row, g.K, run.m, min(batch, kRuns), g.batches, top);
        else top_of_short_row<T>(row, g.K, run.m, top);
        if constexpr (kSlots)
          if (g.ctas > 1) join_tops<kThreads>(g.K, g.ctas, rank, top);
      }
      if (rank == 0 && (int)threadIdx.x < g.K) {
        const unsigned long long key = bad ? 0 : kSlots && g.ctas > 1 ? top.all[kSlots ? threadIdx.x : 0] : top.top[threadIdx.x];
        const int64_t to = n * g.K + threadIdx.x;
        g.top_ids[to] = key == 0 ? -1 : (int)(0xFFFFFFFFu - (uint32_t)key);
        g.top_logp[to] = bad ? NAN : key == 0 ? -INFINITY : log_p(of_order((uint32_t)(key >> 32)), a, g.scale, ln_s);
      }
    }
  }
  if (g.ctas > 1) {
    __syncwarp();
    ptx::cluster_sync_all();                                  // nobody leaves while its shared memory is read
  }
  if (kSlots && *reinterpret_cast<volatile int*>(&abort) != 0)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);         // copies under way land before the shared memory is given back
}

// ---------------------------------------------------------------------------------------------- distillation
struct DistillArgs {
  const void* z;
  int64_t N, ld;
  int V, ctas, K;
  float scale;
  Factors f;
  const int32_t* ids;
  const float* top;
  const float* weights;
  float* loss;
  void* grad;
  int64_t ldg;
};

struct DistillShared {        // of two rows in turn
  int id[2][kMaxTop];
  float t[2][kMaxTop], z[2][kMaxTop], p[2][kMaxTop];
  uint32_t flags[2][kMaxTop / 32];  // of each warp's places: 1 there is a teacher, 2 an id outside of the vocabulary
};

// p = softmax over the places, and the row's loss: by one warp, a lane has every 32nd place.
__device__ __forceinline__ float teacher_loss(const DistillArgs& g, const Stat& a, DistillShared& d, int parity) {
  constexpr int kPer = kMaxTop / 32;
  const int lane = threadIdx.x & 31;
  float x[kPer], top = kMasked;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 32 * k;
    x[k] = i < g.K ? d.t[parity][i] : kMasked;
    top = fmaxf(top, x[k]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) sum += x[k] <= kMasked ? 0.f : exp2_fast((x[k] - top) * g.f.near);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  const float logs = kLn2 * (log2_sum(a, g.f) - log2f(sum));
  float loss = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 32 * k;
    if (i >= g.K) continue;
    const float p = x[k] <= kMasked ? 0.f : __fdiv_rn(exp2_fast((x[k] - top) * g.f.near), sum);
    d.p[parity][i] = p;
    if (p == 0.f) continue;
    const float z = d.z[parity][i];
    loss += z <= kMasked ? INFINITY : p * fmaf((x[k] - top) - (z - a.m), g.scale, logs);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xFFFFFFFFu, loss, o);
  return loss;
}

// A lane's vector of 32 that follow one another, to an address off the grid: the elements before the grid's next line go with the lane before, and
// the next lane's first ones come here.  `beyond`: what lane 0 gives to lane 31, where there is `more`.  The first vector's first elements
// (`begin`) and the last one's last ones are written one by one.
// (2048 x 131072 with an odd pitch of the gradient: 842 us with all elements one by one, 293 so, 200 where the grids agree.)
template <typename T>
__device__ __forceinline__ void store_off_grid(T* to, const uint4& y, const uint4& beyond, bool begin, bool more) {
  constexpr int kVec = Elem<T>::kVec;
  const int lane = threadIdx.x & 31, ahead = kVec - (int)((reinterpret_cast<uintptr_t>(to) & 15u) / sizeof(T));    // elements before the next line
  const bool give = lane == 0 && more;
  uint32_t w[8] = {y.x, y.y, y.z, y.w};
  w[4] = __shfl_sync(0xFFFFFFFFu, give ? beyond.x : y.x, (lane + 1) & 31);
  w[5] = __shfl_sync(0xFFFFFFFFu, give ? beyond.y : y.y, (lane + 1) & 31);
  w[6] = __shfl_sync(0xFFFFFFFFu, give ? beyond.z : y.z, (lane + 1) & 31);
  w[7] = __shfl_sync(0xFFFFFFFFu, give ? beyond.w : y.w, (lane + 1) & 31);
  const int words = ahead * (int)sizeof(T) / 4;
#pragma unroll
  for (int j = 0; j < 6; ++j) w[j] = (words & 2) ? w[j + 2] : w[j];
#pragma unroll
  for (int j = 0; j < 5; ++j) w[j] = (words & 1) ? w[j + 1] : w[j];
  const uint32_t bits = sizeof(T) == 2 && (ahead & 1) ? 16u : 0u;
  if (lane < 31 || more) {
    *reinterpret_cast<uint4*>(to + ahead) = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                                                       __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
  } else {
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (j >= ahead) Elem<T>::put_into(to + j, y, j);
  }
  if (lane == 0 && begin) {
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (j < ahead) Elem<T>::put_into(to + j, y, j);
  }
}

// kShift: the gradient's rows do not all lie as the logits' do on the memory's grid.
template <typename T, bool kGrad, int kThreads, bool kShift>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
distill_kernel(const DistillArgs g) {
  constexpr bool kSlots = kThreads != kShort;
  constexpr int kVec = Elem<T>::kVec, kStep = vector_step<kThreads>(), kSlotsRow = kThreads == 1024 ? kSlotsTwice : kSlotsOnce;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ RowShared sh;
  __shared__ DistillShared d;
  __shared__ uint64_t barriers[kSlots ? kSlotsRow * kThreads / 32 : 1];
  __shared__ int abort;
  after_previous();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)(blockIdx.x % (unsigned)g.ctas);
  const Rows rows{g.z, g.ld, blockIdx.x / (unsigned)g.ctas, gridDim.x / (unsigned)g.ctas, g.N, g.V, rank, g.ctas, g.weights};
  typename std::conditional<kSlots, Pieces<T, kThreads, kSlotsRow, kGrad>, int>::type pieces = [&] {
    if constexpr (kSlots) return Pieces<T, kThreads, kSlotsRow, kGrad>(rows, slots, barriers, &abort);
    else return 0;
  }();
  int parity = 0;
  float w = g.weights != nullptr ? load_near(g.weights + rows.first) : 1.f, w_next = 1.f;
  for (int64_t n = rows.first; n < g.N; n += rows.step, w = w_next) {
    if (g.weights != nullptr && n + rows.step < g.N) w_next = load_near(g.weights + n + rows.step);
    const Row<T> row(reinterpret_cast<const T*>(g.z), n, g.ld, g.V, rank, g.ctas);
    T* grad = kGrad ? reinterpret_cast<T*>(g.grad) + n * g.ldg : nullptr;
    const bool aligned = kGrad && (!kShift || ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.z)) & 15u) == 0);
    auto store = [&](int i, const uint4& y) {
      if (aligned && row.whole(i)) {
        *reinterpret_cast<uint4*>(grad + row.first(i)) = y;
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (row.first(i) + j >= 0 && row.first(i) + j < row.V) Elem<T>::put_into(grad + row.first(i) + j, y, j);
      }
    };
    auto store_zeros = [&]() {                                // of this CTA's part: on the gradient's own grid, and one by one at its ends
      T* const from = grad + max(0, row.first(row.lo)), * const to = grad + min(g.V, row.first(row.hi));
      const int lead_in = (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(from)) & 15u) / (int)sizeof(T), all = (int)(to - from);
      const int body = all > lead_in ? (all - lead_in) / kVec : 0, rest = min(all, lead_in) + body * kVec;
      for (int i = tid; i < body; i += kThreads) *reinterpret_cast<uint4*>(from + lead_in + i * kVec) = make_uint4(0, 0, 0, 0);
      if (tid < min(all, lead_in)) Elem<T>::store(from + tid, 0.f);
      if (tid < all - rest) Elem<T>::store(from + rest + tid, 0.f);
    };
    if (w == 0.f) {                                           // the same for all CTAs of the row, which is not read
      if (rank == 0 && tid == 0) g.loss[n] = 0.f;
      if (kGrad) store_zeros();
      continue;
    }
    int id = -1;
    float teacher = kMasked, z_id = kMasked;
    if (tid < g.K) {
      id = load_near(g.ids + n * g.K + tid);
      teacher = load_near(g.top + n * g.K + tid);
    }
    Running<T, false> run(g.f);
    const int i0 = first_vector<kThreads>(row.lo, 0), lead = kSlots ? lane : tid;
    for (int i = i0; i - lead < row.hi; i += kBatch * kThreads) {
      uint4 v[kBatch];
      read_batch<T, kThreads, false>(row, i, pieces, &abort, v, run);
      run.add(v);
      // the student's logits at the teacher's places: read before a gradient may be written over them
      if (i == i0 && tid < g.K && id >= 0 && id < g.V) z_id = Elem<T>::load(row.z + id);
    }
    if (i0 - lead >= row.hi && tid < g.K && id >= 0 && id < g.V) z_id = Elem<T>::load(row.z + id);
    if (tid < g.K) {
      d.id[parity][tid] = id;
      d.t[parity][tid] = id >= 0 ? max_nan(teacher, kMasked) : kMasked;
      d.z[parity][tid] = max_nan(z_id, kMasked);
    }
    const bool there = tid < g.K && id >= 0;
    const uint32_t flags = (__any_sync(0xFFFFFFFFu, there && !(teacher <= kMasked)) ? 1u : 0u) | (__any_sync(0xFFFFFFFFu, there && id >= g.V) ? 2u : 0u);
    if (lane == 0 && warp < kMaxTop / 32) d.flags[parity][warp] = flags;
    const Stat a = join_row<kThreads>(run.stat(), g.f, g.scale, g.ctas, sh, parity);
    uint32_t all = 0;
#pragma unroll
    for (int k = 0; k < kMaxTop / 32; ++k) all |= d.flags[parity][k];
    const bool bad = isnan(a.s) || (all & 2u) != 0;           // (an id outside of the vocabulary, or a row that is no number)
    const bool none = all == 0;                               // no teacher
    if (warp == 0 && !none) {
      const float loss = teacher_loss(g, a, d, parity);
      if (rank == 0 && lane == 0) g.loss[n] = bad ? NAN : w * loss;
    }
    if (none && rank == 0 && tid == 0) g.loss[n] = 0.f;
    if constexpr (kGrad) {
      const bool zeros = none || (!bad && a.m <= kMasked);
      const float gp = zeros ? 0.f : w * g.scale;
      const float gq = zeros ? 0.f : bad ? NAN : gp / a.s;
      const float c = factor(a.m, g.f);
      const f32x2 cc = pair_of(c, c), minus = pair_of(-a.mc, -a.mc);
      f32x2 scale2 = pair_of(gq, gq);
      const uint32_t keep = zeros ? 0u : 0xFFFFFFFFu;
      uint4* const out = reinterpret_cast<uint4*>(grad - row.off);      // vector 0, where the gradient lies as the logits do
      for (int i = i0; i - lead < row.hi; i += kBatch * kThreads) {
        uint4 v[kBatch];
        if constexpr (kSlots) {
          if (!pieces.next(v, &abort, nullptr, 0)) scale2 = pair_of(NAN, NAN);       // (a copy that did not come in time)
        } else {
#pragma unroll
          for (int u = 0; u < kBatch; ++u) v[u] = i + u * kStep < row.hi ? row.load(i + u * kStep) : row.none();
        }
        const bool piece = kSlots && row.inside(i - lane), inside = aligned && piece;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          f32x2 x[Elem<T>::kPairs];
          Elem<T>::pairs(v[u], x);
#pragma unroll
          for (int q = 0; q < Elem<T>::kPairs; ++q) {
            const float2 e = halves(pfma(x[q], cc, minus));
            x[q] = pmul(pair_of(exp2_fast(e.x), exp2_fast(e.y)), scale2);
          }
          uint4 y = Elem<T>::pack(x);
          y.x &= keep; y.y &= keep; y.z &= keep; y.w &= keep;
          if constexpr (kShift) v[u] = y;
          else if (inside) out[i + u * kStep] = y;
          else if (i + u * kStep < row.hi) store(i + u * kStep, y);
        }
        if constexpr (kShift) {
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const int k = i + u * kStep;
            if (!aligned && (piece || __all_sync(0xFFFFFFFFu, k < row.hi && row.whole(k)))) {
              const bool joined = piece && u + 1 < kBatch;    // (the lanes' next vectors follow those of lane 31)
              store_off_grid<T>(grad + row.first(k), v[u], v[u + 1 < kBatch ? u + 1 : u], !piece || u == 0, joined);
            } else if (k < row.hi) {
              store(k, v[u]);
            }
          }
        }
      }
      __syncthreads();
      // the teacher's places of this CTA's part, after the barrier: each with all of its p, in the order of the places
      if (!zeros && tid < g.K && id >= 0 && id < g.V) {
        const int i = (id + row.off) / kVec;
        if (i >= row.lo && i < row.hi) {
          float p = 0.f;
          for (int k = 0; k < g.K; ++k) p += d.id[parity][k] == id ? d.p[parity][k] : 0.f;
          Elem<T>::store(grad + id, exp2_fast(fmaf(d.z[parity][tid], c, -a.mc)) * gq - gp * p);
        }
      }
      if (kSlots && !zeros && isnan(halves(scale2).x)) g.loss[n] = NAN;  // (a row that is no number, or part of it came late)
    }
    parity ^= 1;
  }
  if (g.ctas > 1) {
    __syncwarp();
    ptx::cluster_sync_all();                                  // nobody leaves while its shared memory is read
  }
  if (kSlots && *reinterpret_cast<volatile int*>(&abort) != 0)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);         // copies under way land before the shared memory is given back
}

// ---------------------------------------------------------------------------------------------- launches
// Rows of 32-bit logits of which nothing is kept in shared memory are short to half of that (4096 x 4000 with 16 KB: log probabilities
// 26.6 us as short rows, 21.2 as long ones, gradient 61 and 40; 2000 with 8 KB: no difference; of 16 bits, 8000: 21.2 and 25.8, 43 and 44).
constexpr int64_t short_row(int f32) { return f32 ? kShortRow / 2 : kShortRow; }
constexpr int64_t kRowsUnderWay = 48 << 20;  // bytes of rows that are to be found again in the second-level cache

constexpr double kRateSm = 43e3, kRateThread = 117;     // bytes in a us
struct Plan {
  int ctas;                   // of a row
  int64_t rows;               // under way at a time
  size_t smem;
};
// CTAs of a cluster share a row where rows are too few for all SMs, or do not go up evenly in those that can be under way, or where those
// are not to be more than the second-level cache keeps (`again`).  `clusters(c, k)`: how many of c CTAs run at a time with k CTAs to an SM; k is
// no larger than all rows need, or some SMs would get four CTAs and others one (300 x 131072: 21.5 us with 3, 26.7 with room for 4).
// The time of a row's part is estimated by its bytes at the rate that a CTA has, alone or beside others on its SM, and what is around it: 2 us,
// joining with others 1.6 to 2.2, and 0.8 more for their alternatives (1 x 131072 with 1, 2, 4, 8 CTAs: 10.9, 7.8, 5.7, 4.7 us, with 20
// alternatives 14.8, 12.7, 10.7, 10.1; 140 x 50001 with 20: 10.4, 12.1, 13.8).
template <typename F>
int plan_rows(int64_t N, int64_t row /* vectors, at most */, int threads, bool again, bool tops, Plan& p, int& to_sm, F clusters) {
  double best = 0;
  p.ctas = 0;
  for (int c = 1; c <= kMaxCluster; c *= 2) {
    const int64_t part = ceil_div(row, c);
    if (c > 1 && (threads < kLong || part < threads * kBatch)) break;
    for (int k = 1; k <= 1024 / threads; ++k) {
      const int64_t slots = clusters(c, k);
      if (slots < 1) continue;
      const int64_t rows = N < slots ? N : slots;
      const double rate = fmin(kRateSm / k, kRateThread * threads), around = 2.0 + (c > 1 ? (tops ? 2.2 : 1.4) + 0.1 * c : 0.0);
      const double us = (double)ceil_div(N, slots) * ((double)part * 16 * (again ? 2 : 1) / rate + around);
      const bool fits = rows * row * 16 <= kRowsUnderWay;
      if (p.ctas == 0 || us < 0.97 * best || (again && fits && p.rows * row * 16 > kRowsUnderWay)) {
        best = us;
        p.ctas = c;
        p.rows = rows;
        to_sm = k;
      }
      if (slots >= N) break;
    }
  }
  return p.ctas == 0 ? TLQ_ERR_CUDA : TLQ_OK;
}
// Vectors that rows have at most: one more where they do not begin on the vectors' grid.
int64_t row_vectors(const void* z, int64_t N, int64_t V, int64_t ld, int64_t size) {
  return ceil_div(V * size, 16) + (aligned16(z) && (N == 1 || ld * size % 16 == 0) ? 0 : 1);
}

// What is asked once for each kernel and device: its shared memory, and the clusters of c CTAs that run at a time with k to an SM.
struct Resident {
  size_t fixed[kMaxDevices] = {};
  int count[kMaxDevices][4][8] = {};
};
constexpr size_t kSharedOfSm = 228 << 10, kSharedOfCta = 1 << 10;         // (the latter is the system's)
template <int kThreads, typename Kernel>
int plan_launch(Kernel kernel, Resident& known, size_t smem, int64_t N, int64_t row, bool again, bool tops, Plan& p) {
  constexpr int kMost = 1024 / kThreads;
  const int dev = current_device_index();
  if (dev < 0) return TLQ_ERR_CUDA;
  if (known.fixed[dev] == 0) {
    cudaFuncAttributes attr;
    TLQ_CUDA_TRY(cudaFuncGetAttributes(&attr, kernel));
    TLQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(smem > kSharedOfSm / 2 + 1024 ? smem : kSharedOfSm / 2 + 1024)));
    known.fixed[dev] = attr.sharedSizeBytes + kSharedOfCta;
  }
  const size_t fixed = known.fixed[dev];
  auto with = [&](int k) {    // shared memory of which k + 1 CTAs have no room on an SM
    const size_t wanted = align_up(kSharedOfSm / (k + 1) + 1, 128);
    return k >= kMost || wanted < fixed + smem ? smem : wanted - fixed;
  };
  int to_sm = kMost;
  const int rc = plan_rows(N, row, kThreads, again, tops, p, to_sm, [&](int c, int k) -> int64_t {
    int& n = known.count[dev][c == 1 ? 0 : c == 2 ? 1 : c == 4 ? 2 : 3][k - 1];
    if (n == 0) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3((unsigned)(c * 1024));
      cfg.blockDim = dim3((unsigned)kThreads);
      cfg.dynamicSmemBytes = with(k);
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = (unsigned)c;
      attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
      }
    }
    return n;
  });
  p.smem = with(to_sm);
  return rc;
}

template <typename T, bool kEntropy, bool kTop, int kThreads>
int run_logprobs(LogprobArgs g, cudaStream_t st) {
  static Resident known;
  constexpr size_t smem = kThreads != kShort ? (size_t)kSlotsOnce * kBatch * kThreads * 16 : 0;
  auto kernel = logprobs_kernel<T, kEntropy, kTop, kThreads>;
  const int64_t vectors = row_vectors(g.z, g.N, g.V, g.ld, sizeof(T));
  Plan p;
  const int rc = plan_launch<kThreads>(kernel, known, smem, g.N, vectors, false, kTop, p);
  if (rc != TLQ_OK) return rc;
  g.ctas = p.ctas;
  g.batches = (int)ceil_div(ceil_div(ceil_div(vectors, p.ctas), (int64_t)kBatch * kThreads), kRuns);
  return launch_next(kernel, dim3((unsigned)(p.rows * p.ctas)), kThreads, p.smem, (unsigned)p.ctas, st, g);
}

template <typename T, bool kGrad, int kThreads, bool kShift>
int run_distill(DistillArgs g, cudaStream_t st) {
  static Resident known;
  constexpr size_t smem = kThreads != kShort ? (size_t)(kThreads == 1024 ? kSlotsTwice : kSlotsOnce) * kBatch * kThreads * 16 : 0;
  auto kernel = distill_kernel<T, kGrad, kThreads, kShift>;
  Plan p;
  const int rc = plan_launch<kThreads>(kernel, known, smem, g.N, row_vectors(g.z, g.N, g.V, g.ld, sizeof(T)), kGrad, false, p);
  if (rc != TLQ_OK) return rc;
  g.ctas = p.ctas;
  return launch_next(kernel, dim3((unsigned)(p.rows * p.ctas)), kThreads, p.smem, (unsigned)p.ctas, st, g);
}

}  // namespace

int launch_token_logprobs(const void* logits, int f32, int64_t N, int64_t V, int64_t ld, float scale, const int32_t* ids, int K,
                          float* logp, float* entropy, float* lse, int32_t* top_ids, float* top_logp, cudaStream_t st) {
  LogprobArgs g{};
  g.z = logits; g.N = N; g.ld = ld; g.V = (int)V; g.K = K; g.f = factors_of(scale); g.scale = scale;
  g.ids = ids; g.logp = logp; g.entropy = entropy; g.lse = lse; g.top_ids = top_ids; g.top_logp = top_logp;
  auto of_type = [&](auto type, auto threads) {
    using T = decltype(type);
    constexpr int kThreads = decltype(threads)::value;
    if (entropy != nullptr) return K > 0 ? run_logprobs<T, true, true, kThreads>(g, st) : run_logprobs<T, true, false, kThreads>(g, st);
    return K > 0 ? run_logprobs<T, false, true, kThreads>(g, st) : run_logprobs<T, false, false, kThreads>(g, st);
  };
  const std::integral_constant<int, kShort> few;
  const std::integral_constant<int, kLong> many;
  const bool is_short = V * (f32 ? 4 : 2) <= (K > 0 ? kShortRow : short_row(f32));
  if (f32) return is_short ? of_type(0.f, few) : of_type(0.f, many);
  return is_short ? of_type((uint16_t)0, few) : of_type((uint16_t)0, many);
}

int launch_distill_loss(const void* logits, int f32, int64_t N, int64_t V, int64_t ld, float scale, const int32_t* top_ids,
                        const float* top_logits, int K, const float* weights, float* loss, void* grad, int64_t ldg, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  DistillArgs g{};
  g.z = logits; g.N = N; g.ld = ld; g.V = (int)V; g.K = K; g.f = factors_of(scale); g.scale = scale;
  g.ids = top_ids; g.top = top_logits; g.weights = weights; g.loss = loss; g.grad = grad; g.ldg = ldg;
  const bool is_short = V * (f32 ? 4 : 2) <= short_row(f32);
  auto with_grad = [&](auto type, auto off_grid) {
    using T = decltype(type);
    constexpr bool kShift = decltype(off_grid)::value;
    if (is_short) return run_distill<T, true, kShort, kShift>(g, st);
    // the smallest CTAs whose rows under way stay in the second-level cache
    const int64_t row = V * (int64_t)sizeof(T), most = kRowsUnderWay / row;
    return N <= most || 4 * sms <= most ? run_distill<T, true, 256, kShift>(g, st)
                                        : 2 * sms <= most ? run_distill<T, true, 512, kShift>(g, st) : run_distill<T, true, 1024, kShift>(g, st);
  };
  auto of_type = [&](auto type) {
    using T = decltype(type);
    if (grad == nullptr) return is_short ? run_distill<T, false, kShort, false>(g, st) : run_distill<T, false, kLong, false>(g, st);
    const bool alike = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(grad)) & 15u) == 0 &&
                       (N == 1 || (ld - ldg) * (int64_t)sizeof(T) % 16 == 0);
    return alike ? with_grad(type, std::false_type()) : with_grad(type, std::true_type());
  };
  return f32 ? of_type(0.f) : of_type((uint16_t)0);
}

}  // namespace tlq
