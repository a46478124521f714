// Attention of many query rows over the 8-bit cache (prompts and chunks of prompts) on the tensor-memory path.
//
// The formulas are those of kv_attention.cu: scores from (kc + 128) with the 128 sum(q) taken out by a constant of the row,
// p_j = 2^(t_j - m) with t_j = a (q . kc_j) + log2(vstep), output sums of p vc and sums of p / vstep.
//
// A CTA works on 256 rows of one (request, kv head), a row being one query head of one token: two tiles of 128 rows, so
// that the exponentials of one run while the tensor core works on the other.  Per tile and 128 cached tokens: S = q K^T
// (tcgen05, f16 x f16 -> f32, tensor memory), a thread per row takes the maximum and the exponentials of its row from
// tensor memory and writes P over S as f16, O += P V with P from tensor memory.  The output sum is rescaled only when the
// maximum of a row has grown by more than 4 (a factor of 16 in p): p is kept as 2^11 p, so that it fits 16 bits either way.
//   warps 0..3, 4..7  softmax of tile 0, 1: a thread is a row (and its accumulator lane), its 128 scores in registers
//   warps 8..11       bring the codes of keys and values from the cache into registers, turn them into f16 and lay them
//                     out for the tensor core (128-byte swizzle); two stages each
//   warp 12           issues the products
//   warp 13           finds the parts of items that this CTA works on and passes them on through a ring (14 and 15 idle:
//                     registers are shared out by groups of four warps)
// Nothing in the loops may spill: with 200 KB of shared memory in use the first-level cache is too small for local memory,
// and a few spilled words per step cost more than the step (versions that spilled ran at 850 to 990 us, see below).
// Work is cut as in the few-row kernel: items (row tiles of a kv head) lie on one line, weighted by their cached tokens,
// every CTA takes an equal part of it; an item that is cut leaves partial sums, and the CTA that completes it joins them.
//
// Bound: the tensor core (4 D flops per visible pair) and, next to it, the exponential unit: 256 x 128 exponentials at 16
// per cycle take as long as the products of the same tile.
#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

constexpr int kTile = 128, kItemRows = 256, kKeys = 128;
constexpr int kSoftWarps = 8, kLoadWarps = 4, kIssueWarp = kSoftWarps + kLoadWarps, kPlanWarp = kIssueWarp + 1;
constexpr int kThreads = 512;                              // four groups of four warps
// registers of a thread of each role: 2 x 192 + 80 + 48 = 4 x 128, what the block is launched with
constexpr int kSoftRegs = 192, kLoadRegs = 80, kIssueRegs = 48, kLaunchRegs = 128;
constexpr float kShift = 11.f, kGrow = 4.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kStepFloor = 7.8886090522101181e-31f;      // 2^-100, as in kv_attention.cu
constexpr float kUnit = 16777216.f;                        // 2^24
constexpr int kMinTiles = 6;                               // key tiles of a CTA's part, at least
constexpr int kItemCost = 2;                               // what an item costs beside its key tiles, in key tiles

struct PromptArgs {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* out;
  float* lse;
  float scale_log2;
  int causal, min_rows;         // requests with fewer rows than this belong to the few-row kernel
  KvSplit split;
};

template <int D>
constexpr uint32_t kPanels = D / 64;                       // 64 channels of f16 are one row of the swizzle
template <int D>
constexpr uint32_t kQBytes = kTile * D * 2;                // of one tile of queries
template <int D>
constexpr uint32_t kKBytes = kKeys * D * 2;                // of one stage of keys
template <int D>
constexpr uint32_t kVBytes = kKeys * D * 2;                // of one stage of values
template <int D>
constexpr size_t kSmem = 1024 + 2 * kQBytes<D> + 2 * kKBytes<D> + 2 * kVBytes<D>;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 ld_cache(const int8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// (code + 128) 2^-24 as f16, and exactly the code: see kv_attention.cu
__device__ __forceinline__ void keys_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t x = w ^ 0x80808080u;
  lo = __byte_perm(x, 0u, 0x4140);
  hi = __byte_perm(x, 0u, 0x4342);
}
__device__ __forceinline__ void values_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t x = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
  const __half2 off = __floats2half2_rn(1152.f, 1152.f);
  const __half2 ra = __hsub2(*reinterpret_cast<const __half2*>(&a), off);
  const __half2 rb = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&ra);
  hi = *reinterpret_cast<const uint32_t*>(&rb);
}

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  ptx::mma_bf16_ss(d, a, b, idesc, accumulate);            // kind::f16 covers both types; the descriptor names f16
}
// A from tensor memory
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// The wait for loads of tensor memory, naming 32 of the registers that they fill: no use of those can move before it.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ float as_f(uint32_t x) { return __uint_as_float(x); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// two 32-bit sums or products in one instruction
__device__ __forceinline__ void fma2(float& x, float& y, float a, float bx, float by, float c) {
  asm("{\n\t.reg .b64 p, q, r, s;\n\t"
      "mov.b64 p, {%2, %2};\n\tmov.b64 q, {%3, %4};\n\tmov.b64 r, {%5, %5};\n\t"
      "fma.rn.f32x2 s, q, p, r;\n\tmov.b64 {%0, %1}, s;\n\t}"
      : "=f"(x), "=f"(y) : "f"(a), "f"(bx), "f"(by), "f"(c));
}
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
  asm("{\n\t.reg .b64 p, q;\n\t"
      "mov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\t"
      "add.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
      : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------- the line of work
// Item `tile` of a request costs first + tile * more; the first n cost sum(n).
struct Costs {
  int tiles;
  long long first, more;
  __device__ __forceinline__ long long sum(long long n) const { return first * n + more * (n * (n - 1) / 2); }
};
__device__ __forceinline__ Costs costs_of(const KvArgs& a, const PromptArgs& g, const Request& r) {
  Costs c;
  const long long rows = (long long)r.q_len * a.group;
  c.tiles = rows >= g.min_rows ? (int)((rows + kItemRows - 1) / kItemRows) : 0;
  const int seen = g.causal ? min(max(r.kv - r.q_len, 0) + kItemRows / a.group, r.kv) : r.kv;
  c.first = 64LL * (kItemCost + 1) + 64LL * seen / kKeys;
  c.more = g.causal ? 64LL * kItemRows / kKeys / a.group : 0;
  return c;
}

// A part of an item: key tiles [k0, k1) of n; k0 < 0: there are no more.
struct __align__(16) Segment {
  int b, h, tile, k0;
  int k1, n, q0, q_len;
  long long at, len;            // the item on the line
  int kv, starts, pad[2];       // starts: the item starts in this CTA's part of the line
};
constexpr int kRing = 4;        // segments in the ring

// The key tiles [k0, k1) of an item (n of them, at `at` of the line) that the part [from, to) of the line holds.
__device__ __forceinline__ void cut(long long from, long long to, long long at, long long len, int n, int& k0, int& k1) {
  k0 = from <= at ? 0 : from >= at + len ? n : (int)((long long)n * (from - at) / len);
  k1 = to >= at + len ? n : to <= at ? 0 : (int)((long long)n * (to - at) / len);
}

// Walks the items that overlap [x0, x1) of the line.
struct Walk {
  long long x0, x1, base;       // base: where (request b, head h) starts on the line
  int b, h, tile;
  Request req;
  Costs costs;

  __device__ __forceinline__ int key_tiles(const KvArgs& a, const PromptArgs& g) const {
    const long long rows = (long long)req.q_len * a.group;
    const int row = (int)(min((long long)(tile + 1) * kItemRows, rows) - 1);
    const int last = g.causal ? min(req.kv - req.q_len + row / a.group, req.kv - 1) : req.kv - 1;
    return last < 0 ? 0 : last / kKeys + 1;
  }
  __device__ __forceinline__ void start(const KvArgs& a, const PromptArgs& g, int request, long long rest, long long from, long long to) {
    x0 = from; x1 = to;
    b = request;
    req = load_request(a, b);
    costs = costs_of(a, g, req);
    const long long one = costs.sum(costs.tiles);
    h = (int)(rest / one);
    const long long in = rest - h * one;
    base = from - in;
    int lo = 0, hi = costs.tiles - 1;                      // the last tile that starts at or before `in`
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (costs.sum(mid) <= in) lo = mid; else hi = mid - 1;
    }
    tile = lo;
  }
  // next part with something to do; false at the end
  __device__ __forceinline__ bool next(const KvArgs& a, const PromptArgs& g, Segment& s) {
    while (true) {
      while (tile >= costs.tiles) {
        base += costs.sum(costs.tiles);
        tile = 0;
        if (costs.tiles > 0 && ++h < a.n_kv) break;
        h = 0;
        if (++b >= a.B) return false;
        req = load_request(a, b);
        costs = costs_of(a, g, req);
      }
      s.at = base + costs.sum(tile);
      if (s.at >= x1) return false;
      s.len = costs.sum(tile + 1) - costs.sum(tile);
      s.n = key_tiles(a, g);
      cut(x0, x1, s.at, s.len, s.n, s.k0, s.k1);
      s.b = b; s.h = h; s.tile = tile; s.q0 = req.q0; s.q_len = req.q_len; s.kv = req.kv; s.starts = s.at >= x0 ? 1 : 0;
      const bool here = s.n == 0 ? s.at >= x0 : s.k0 < s.k1;   // an item without visible keys belongs to whoever has its start
      ++tile;
      if (here) return true;
    }
  }
};

struct Line {                   // the whole line, how many CTAs share it, this CTA's part
  long long total, workers, x0, x1;
};

struct Cut {                    // an item of which this CTA has only a part
  long long at, len;
  int b, h, tile, n;
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
kv_prompt_kernel(const KvArgs a, const PromptArgs g) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + 2 * kQBytes<D>, v_at = k_at + 2 * kKBytes<D>;
  __shared__ __align__(8) uint64_t bars[16 + 2 * kRing];
  __shared__ Segment s_ring[kRing];
  __shared__ __align__(16) float4 s_steps[4][2];           // of the two blocks of a key tile: kstep, log2 vstep, 1 / vstep, usable
  __shared__ long long sums[kThreads / 32];
  __shared__ Found found;
  __shared__ Cut s_cut[2];
  __shared__ Line s_line;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_join[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return ptx::smem_u32(&bars[i]); };
  // [0,2) q ready, [2,4) k ready, [4,6) k free, [6,8) v ready, [8,10) v free, [10,12) S ready, [12,14) P ready, [14,16) O ready,
  // then the ring of segments: ready, free
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(bar(i), 4);
      ptx::mbar_init(bar(2 + i), kLoadWarps);
      ptx::mbar_init(bar(4 + i), 1);
      ptx::mbar_init(bar(6 + i), kLoadWarps);
      ptx::mbar_init(bar(8 + i), 1);
      ptx::mbar_init(bar(10 + i), 1);
      ptx::mbar_init(bar(12 + i), 4);
      ptx::mbar_init(bar(14 + i), 1);
      s_cut[i].len = 0;
    }
    for (int i = 0; i < kRing; ++i) {
      ptx::mbar_init(bar(16 + i), 1);
      ptx::mbar_init(bar(16 + kRing + i), kSoftWarps + kLoadWarps + 1);
    }
    s_abort = 0;
    ptx::fence_barrier_init();
  }
  volatile int* abort_flag = &s_abort;

  // ---------------------------------------------------------------- this CTA's part of the line
  auto cost_of = [&](int b) {
    const Costs c = costs_of(a, g, load_request(a, b));
    return c.sum(c.tiles) * a.n_kv;
  };
  long long total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + (int)threadIdx.x;
    long long part;
    block_scan<kThreads>(b < a.B ? cost_of(b) : 0, sums, part);
    total += part;
  }
  if (total == 0) return;
  {
    // a part is worth joining from some key tiles on
    const long long workers = max(1LL, min((long long)gridDim.x, total / (64 * kMinTiles)));
    if (blockIdx.x >= workers) return;
    const long long x0 = total * blockIdx.x / workers, x1 = total * (blockIdx.x + 1) / workers;
    if (x0 >= x1) return;
    if (!locate_item<kThreads>(a.B, x0, cost_of, sums, &found)) return;
    if (threadIdx.x == 0) {                                // read back where they are needed: the loops have no registers to spare
      s_line.total = total; s_line.workers = workers; s_line.x0 = x0; s_line.x1 = x1;
    }
  }
  if (warp == kIssueWarp) ptx::tmem_alloc(ptx::smem_u32(&s_tmem), 512);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = s_tmem;                            // S of tile 0, 1 at columns 0, 128; O at 256, 384
  constexpr size_t kPitch = (size_t)kItemRows * (D + 2);   // floats of a partial: maxima, sums, output sums
  auto slot = [&](long long w, int i) { return g.split.partials + ((size_t)w * 2 + i) * kPitch; };
  // the next segment, by all lanes of a warp (or the one that issues)
  int seg = 0;
  uint32_t seg_phase = 0;
  auto next_segment = [&](bool& ok) {
    ok = ptx::mbar_wait(bar(16 + seg), seg_phase, abort_flag);
    return &s_ring[seg];
  };
  auto done_segment = [&]() {                              // its fields have been read
    ptx::mbar_arrive(bar(16 + kRing + seg));
    if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
  };

  if (warp < kSoftWarps) {
    more_registers<kSoftRegs>();
    // ------------------------------------------------------------------ softmax: a thread is a row
    const int t = warp >> 2, row_in_tile = (warp & 3) * 32 + lane;
    const uint32_t s_col = tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * kTile, o_col = s_col + 256;   // P over S
    uint32_t s_phase = 0, o_phase = 0;
    int step = 0;                                          // key tiles so far, of all segments
    bool ok = true;
    while (true) {
      const Segment* s = next_segment(ok);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok || s->k0 < 0) break;
      const int k0 = s->k0, k1 = s->k1;
      if (threadIdx.x == 0 && (k0 > 0 || k1 < s->n)) {
        Cut* c = &s_cut[s->starts];
        c->at = s->at; c->len = s->len; c->b = s->b; c->h = s->h; c->tile = s->tile; c->n = s->n;
      }
      int limit;
      float fac = 0.f, off = 0.f;
      {
        // the row of q: a power of two brings it into the range of f16
        const int row = s->tile * kItemRows + t * kTile + row_in_tile, token = row / a.group;
        const bool live = token < s->q_len;
        limit = !live ? -1 : g.causal ? min(s->kv - s->q_len + token, s->kv - 1) : s->kv - 1;
        if (k0 < k1) {
          const uint16_t* p = g.q;
          if (live) p += (int64_t)(s->q0 + token) * g.ldq + (int64_t)(s->h * a.group + row - token * a.group) * D;
          uint4 v[D / 8];
#pragma unroll
          for (int i = 0; i < D / 8; ++i) v[i] = live ? __ldg(reinterpret_cast<const uint4*>(p) + i) : make_uint4(0, 0, 0, 0);
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            float e[8];
            unpack8(v[i], e);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(e[j]));
          }
          const int ex = top > 0.f && top <= 3.4e38f ? ilogbf(top) : 0;
          const float d0 = ldexpf(1.0f, -(ex / 2)), d1 = ldexpf(1.0f, -(ex - ex / 2));
          const uint32_t q_row = q_at + t * kQBytes<D> + row_in_tile * 128;
          float qs = 0.f;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            float e[8];
            unpack8(v[i], e);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              w[j] = pack_f16(e[2 * j] * d0 * d1, e[2 * j + 1] * d0 * d1);
              const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
              qs += y.x + y.y;
            }
            sts128(q_row + (i >> 3) * (kTile * 128) + (((i & 7) ^ (row_in_tile & 7)) << 4), w[0], w[1], w[2], w[3]);
          }
          fac = ldexpf(g.scale_log2, ex + 24);
          off = qs * (128.f / kUnit);
          ptx::fence_proxy_async();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(t));
        }
      }

      float m = -INFINITY, l = 0.f;
      for (int k = k0; k < k1; ++k, ++step) {
        ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(10 + t), s_phase, abort_flag));
        if (!ok) break;
        s_phase ^= 1u;
        ptx::tc_fence_after();
        uint32_t v[4][32];                                 // the row of S
#pragma unroll
        for (int c = 0; c < 4; ++c) ptx::tmem_ld32(s_col + 32 * c, v[c]);
        const float4 w0 = s_steps[step & 3][0], w1 = s_steps[step & 3][1];
        float a0 = fac * w0.x, a1 = fac * w1.x;
        float b0 = fmaf(-off, a0, w0.y), b1 = fmaf(-off, a1, w1.y);
        const int see = limit - k * kKeys;                 // last key of the tile that the row sees
        const bool masked = __any_sync(0xFFFFFFFFu, see < kKeys - 1) || w0.w == 0.f || w1.w == 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_wait_for(v[c]);
        if (masked) {                                      // t itself, with nothing where there is nothing to see
          const int see0 = w0.w == 0.f ? -1 : see, see1 = w1.w == 0.f ? -1 : see;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const float x = fmaf(as_f(v[c][j]), c < 2 ? a0 : a1, c < 2 ? b0 : b1);
              v[c][j] = __float_as_uint(32 * c + j <= (c < 2 ? see0 : see1) ? x : -INFINITY);
            }
          a0 = a1 = 1.f;
          b0 = b1 = 0.f;
        }
        float top;
        {
          float r[2][4];
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              float& x = r[c >> 1][j & 3];
              x = (c & 1) == 0 && j < 4 ? as_f(v[c][j]) : fmaxf(x, as_f(v[c][j]));
            }
          top = fmaxf(fmaf(fmaxf(fmaxf(r[0][0], r[0][1]), fmaxf(r[0][2], r[0][3])), a0, b0),
                      fmaf(fmaxf(fmaxf(r[1][0], r[1][1]), fmaxf(r[1][2], r[1][3])), a1, b1));
        }
        // a maximum that has grown by more than kGrow: the output sum follows
        if (__any_sync(0xFFFFFFFFu, top > m + kGrow || (m == -INFINITY && top > -INFINITY))) {
          const float mn = fmaxf(m, top);
          const float corr = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
          m = mn;
          l *= corr;
          if (k > k0) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t x[16];
              ptx::tmem_ld16(o_col + 16 * c, x);
              tmem_ld_wait_for(x);
#pragma unroll
              for (int j = 0; j < 16; ++j) x[j] = __float_as_uint(as_f(x[j]) * corr);
              tmem_st16(o_col + 16 * c, x);
            }
          }
        }
        const float shift = kShift - (m == -INFINITY ? 0.f : m);
        b0 += shift;
        b1 += shift;
        float sum0[2] = {0.f, 0.f}, sum1[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float x, y;
            fma2(x, y, c < 2 ? a0 : a1, as_f(v[c][j]), as_f(v[c][j + 1]), c < 2 ? b0 : b1);
            x = exp2_fast(x);
            y = exp2_fast(y);
            if (c < 2) add2(sum0[0], sum0[1], x, y); else add2(sum1[0], sum1[1], x, y);
            p[j / 2] = pack_f16(x, y);
          }
          tmem_st16(s_col + 16 * c, p);                    // all of S has been read
        }
        const float l0 = sum0[0] + sum0[1], l1 = sum1[0] + sum1[1];
        l += (l0 > 0.f ? l0 * s_steps[step & 3][0].z : l0) + (l1 > 0.f ? l1 * s_steps[step & 3][1].z : l1);
        tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(12 + t));
      }
      if (!ok) break;

      // ---------------------------------------------------------------- leave the item
      if (k0 < k1) {
        ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(14 + t), o_phase, abort_flag));
        if (!ok) break;
        o_phase ^= 1u;
        ptx::tc_fence_after();
      }
      {
        const bool none = m == -INFINITY && l == 0.f;      // a row that sees nothing (a NaN row has a NaN sum)
        const bool whole = k0 == 0 && k1 == s->n;
        const float inv = none ? 0.f : 1.0f / l;
        const int r = t * kTile + row_in_tile, row = s->tile * kItemRows + r, token = row / a.group;
        const bool live = token < s->q_len;
        const int64_t at = (int64_t)(s->q0 + token) * a.n_heads + s->h * a.group + row - token * a.group;
        float* part = slot(blockIdx.x, s->starts);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          if (k0 < k1) {
            ptx::tmem_ld32(o_col + 32 * c, v);
            tmem_ld_wait_for(v);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0u;
          }
          if (live && whole) {
            uint4* to = reinterpret_cast<uint4*>(g.out + at * D + 32 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 z = __floats2bfloat162_rn(none ? 0.f : as_f(v[8 * i + 2 * j]) * inv,
                                                               none ? 0.f : as_f(v[8 * i + 2 * j + 1]) * inv);
                y[j] = *reinterpret_cast<const uint32_t*>(&z);
              }
              to[i] = make_uint4(y[0], y[1], y[2], y[3]);
            }
          } else if (live) {
            uint4* to = reinterpret_cast<uint4*>(part + 2 * kItemRows + (size_t)r * D + 32 * c);
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
          __syncwarp();
        }
        if (live && whole && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(l) + m - kShift);
        if (live && !whole) {
          part[r] = m;
          part[kItemRows + r] = l;
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) done_segment(); else if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
    }
    if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 230);
  } else if (warp < kSoftWarps + kLoadWarps) {
    fewer_registers<kLoadRegs>();
    // ------------------------------------------------------------------ codes of keys and values to f16 operands
    // A warp takes 8 rows x 64 bytes at a time.  Keys: row group (lw / panels) + i * 4 / panels of 16, the same panel for all
    // i; values: row group lw + 4 i of a block's D / 8.  Either way the first half of the i is the tile's first block.
    constexpr int kNum = D / 16, kGroups = 4 / kPanels<D>;   // pieces of a warp; key row groups that the warps take at a time
    const int lw = warp - kSoftWarps, lr = lane & 7, piece = lane >> 3;
    const int k_row = (lw / kPanels<D>) * 8 + lr, k_panel = lw % kPanels<D>;
    const int8_t* const k_from = a.k_codes + k_row * D + k_panel * 64 + piece * 16;
    const int8_t* const v_from = a.v_codes + (lw * 8 + lr) * kKvBlock + piece * 16;
    const uint32_t swizzled0 = ((2 * piece) ^ lr) << 4, swizzled1 = ((2 * piece + 1) ^ lr) << 4;
    const uint32_t k_to = k_at + k_panel * (kKeys * 128) + k_row * 128, v_to = v_at + (lw * 8 + lr) * 128;
    int step = 0, b = 0, h = 0, k = 0, k1 = 0, n_blocks = 0;
    bool ok = true;
    uint4 kr[kNum], vr[kNum];
    int phys[2];
    float ks = 0.f, vs = 0.f;                              // steps of the block `lane` (lanes 0 and 1 of the first warp)
    int64_t block[2];                                      // of the tile whose codes are under way, in bytes
    bool usable[2];
    auto advance = [&]() {                                 // to the next segment with key tiles
      while (true) {
        const Segment* from = next_segment(ok);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) return false;
        b = from->b; h = from->h; k = from->k0; k1 = from->k1;
        n_blocks = (from->kv + kKvBlock - 1) / kKvBlock;
        __syncwarp();
        if (lane == 0) done_segment(); else if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
        if (k < 0) return false;
        if (k < k1) return true;
      }
    };
    auto look_up = [&]() {                                 // the blocks of key tile k
#pragma unroll
      for (int i = 0; i < 2; ++i)
        phys[i] = 2 * k + i < n_blocks ? __ldg(a.block_table + (int64_t)b * a.max_blocks + 2 * k + i) : -1;
    };
    auto load_keys = [&]() {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        usable[i] = phys[i] >= 0 && phys[i] < a.n_blocks;
        if (!usable[i] && 2 * k + i < n_blocks) report_status(a.hdr, TLQ_ERR_SHAPE, 231);
        const int64_t at = (int64_t)(usable[i] ? phys[i] : 0) * a.n_kv + h;
        block[i] = at * (kKvBlock * D);
        if (lw == 0 && lane == i) {
          ks = __ldg(a.k_steps + at);
          vs = __ldg(a.v_steps + at);
        }
      }
#pragma unroll
      for (int i = 0; i < kNum; ++i) {
        // rows of the tile from k_row on, kGroups * 8 apart; a block is 64 of them
        const int row = i * kGroups * 8;
        kr[i] = ld_cache(k_from + block[row >> 6] + (row & 63) * D);
      }
    };
    auto load_values = [&]() {
#pragma unroll
      for (int i = 0; i < kNum; ++i) vr[i] = ld_cache(v_from + block[i / (kNum / 2)] + (i % (kNum / 2)) * 32 * kKvBlock);
    };
    bool more = advance();
    if (more) {
      look_up();
      load_keys();
      load_values();
    }
    while (more) {
      const float my_ks = ks, my_vs = vs;
      const float my_use = usable[0] && lane == 0 ? 1.f : usable[1] && lane == 1 ? 1.f : 0.f;
      // the tile after this one
      bool after = true;
      if (++k >= k1) after = advance();
      if (!ok) break;
      if (after) look_up();
      const int stage = step & 1;
      const uint32_t parity = ((uint32_t)(step >> 1) & 1u) ^ 1u;
      ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(4 + stage), parity, abort_flag));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < kNum; ++i) {
        const uint32_t to = k_to + stage * kKBytes<D> + i * kGroups * 8 * 128;
        uint32_t x[8];
        keys_to_f16(kr[i].x, x[0], x[1]); keys_to_f16(kr[i].y, x[2], x[3]);
        keys_to_f16(kr[i].z, x[4], x[5]); keys_to_f16(kr[i].w, x[6], x[7]);
        sts128(to + swizzled0, x[0], x[1], x[2], x[3]);
        sts128(to + swizzled1, x[4], x[5], x[6], x[7]);
      }
      if (lw == 0 && lane < 2) {
        const float v = my_vs < kStepFloor ? kStepFloor : my_vs;
        s_steps[step & 3][lane] = make_float4(my_ks, log2f(v), 1.0f / v, my_use);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(2 + stage));
      if (after) load_keys();
      ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(8 + stage), parity, abort_flag));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < kNum; ++i) {
        const uint32_t to = v_to + stage * kVBytes<D> + (i / (kNum / 2)) * (D * 128) + (i % (kNum / 2)) * 32 * 128;
        uint32_t x[8];
        values_to_f16(vr[i].x, x[0], x[1]); values_to_f16(vr[i].y, x[2], x[3]);
        values_to_f16(vr[i].z, x[4], x[5]); values_to_f16(vr[i].w, x[6], x[7]);
        sts128(to + swizzled0, x[0], x[1], x[2], x[3]);
        sts128(to + swizzled1, x[4], x[5], x[6], x[7]);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(6 + stage));
      if (after) load_values();
      ++step;
      more = after;
    }
    if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 232);
  } else {
    fewer_registers<kIssueRegs>();
    if (warp == kIssueWarp && lane == 0) {
    // ------------------------------------------------------------------ products
    constexpr uint32_t kIdescS = ptx::make_idesc(1, 0, kTile, kKeys, false);   // f16 x f16 -> f32
    constexpr uint32_t kIdescO = ptx::make_idesc(1, 0, kTile, D, false);
    int step = 0;
    uint32_t q_phase = 0, p_phase = 0;
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      ok = ok && ptx::mbar_wait(bar(i), parity, abort_flag);
      ptx::tc_fence_after();
    };
    auto scores = [&](int t, int st) {
#pragma unroll
      for (uint32_t c = 0; c < kPanels<D>; ++c) {
        const uint64_t x = ptx::smem_desc_sw128(q_at + t * kQBytes<D> + c * (kTile * 128));
        const uint64_t y = ptx::smem_desc_sw128(k_at + (st & 1) * kKBytes<D> + c * (kKeys * 128));
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_f16_ss(tmem + t * kTile, x + 2 * i, y + 2 * i, kIdescS, c > 0 || i > 0);
      }
      ptx::mma_commit(bar(10 + t));
    };
    while (true) {
      const Segment* from = next_segment(ok);
      if (!ok) break;
      struct { int k0, k1; } s = {from->k0, from->k1};
      done_segment();
      if (s.k0 < 0) break;
      if (s.k0 >= s.k1) continue;
      for (int t = 0; t < 2; ++t) wait(t, q_phase);
      q_phase ^= 1u;
      wait(2 + (step & 1), (uint32_t)(step >> 1) & 1u);
      if (!ok) break;
      scores(0, step);
      scores(1, step);
      ptx::mma_commit(bar(4 + (step & 1)));
      for (int k = s.k0; k < s.k1 && ok; ++k, ++step) {
        const int stage = step & 1;
        wait(6 + stage, (uint32_t)(step >> 1) & 1u);
        const bool next = k + 1 < s.k1;
        for (int t = 0; t < 2 && ok; ++t) {
          wait(12 + t, p_phase);
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint64_t y = ptx::smem_desc_sw128(v_at + stage * kVBytes<D> + c * (D * 128));
#pragma unroll
            for (int i = 0; i < 4; ++i)
              mma_f16_ts(tmem + 256 + t * kTile, tmem + t * kTile + 32 * c + 8 * i, y + 2 * i, kIdescO, k > s.k0 || c > 0 || i > 0);
          }
          if (next) {
            if (t == 0) wait(2 + ((step + 1) & 1), (uint32_t)((step + 1) >> 1) & 1u);
            if (!ok) break;
            scores(t, step + 1);
          } else {
            ptx::mma_commit(bar(14 + t));
          }
        }
        if (!ok) break;
        ptx::mma_commit(bar(8 + stage));
        if (next) ptx::mma_commit(bar(4 + ((step + 1) & 1)));
        p_phase ^= 1u;
      }
    }
    if (!ok) report_status(a.hdr, TLQ_ERR_TIMEOUT, 233);
    } else if (warp == kPlanWarp && lane == 0) {
      // ---------------------------------------------------------------- segments
      Walk walk;
      walk.start(a, g, found.request, found.rest, s_line.x0, s_line.x1);
      uint32_t phase = 1;
      while (true) {
        Segment s;
        const bool more = walk.next(a, g, s);
        if (!more) s.k0 = -1;
        if (!ptx::mbar_wait(bar(16 + kRing + seg), phase, abort_flag)) {
          report_status(a.hdr, TLQ_ERR_TIMEOUT, 234);
          break;
        }
        s_ring[seg] = s;
        ptx::mbar_arrive(bar(16 + seg));
        if (!more) break;
        if (++seg == kRing) { seg = 0; phase ^= 1u; }
      }
    }
  }
  __syncwarp();
  // the rest is run by all warps: back to what they were launched with
  if (warp < kSoftWarps) fewer_registers<kLaunchRegs>(); else more_registers<kLaunchRegs>();
  if (*abort_flag != 0)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);      // products under way end before their memory is given back
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  if (*abort_flag != 0) return;

  // ------------------------------------------------------------------ join the CTAs that share an item
  const long long total_cost = s_line.total, workers = s_line.workers;
  auto edge = [&](long long w) { return total_cost * w / workers; };
  auto worker_of = [&](long long x) { return ((x + 1) * workers - 1) / total_cost; };
  if (threadIdx.x < 2) {
    const Cut c = s_cut[threadIdx.x];
    s_join[threadIdx.x] = 0;
    if (c.len > 0) {
      int k0, k1;
      cut(s_line.x0, s_line.x1, c.at, c.len, c.n, k0, k1);
      int32_t* counter = g.split.counters + worker_of(c.at);
      __threadfence();                                     // the CTA's partials, which the barrier has ordered before this
      const int before = atomicAdd(counter, k1 - k0);      // key tiles of the item that are done
      if (before + (k1 - k0) == c.n) {
        *counter = 0;
        s_join[threadIdx.x] = 1;
      }
      __threadfence();
    }
  }
  __syncthreads();
  for (int i = 0; i < 2; ++i) {
    if (!s_join[i]) continue;
    const Cut c = s_cut[i];
    const Request req = load_request(a, c.b);
    const long long rows = (long long)req.q_len * a.group;
    const long long first = worker_of(c.at), final = worker_of(c.at + c.len - 1);
    for (int e = threadIdx.x; e < kItemRows * (D / 4); e += kThreads) {
      const int r = e / (D / 4), d = (e % (D / 4)) * 4;
      const int row = c.tile * kItemRows + r;
      if (row >= rows) break;
      float mm = -INFINITY, den = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (long long w = first; w <= final; ++w) {
        int k0, k1;
        cut(edge(w), edge(w + 1), c.at, c.len, c.n, k0, k1);
        if (k0 >= k1) continue;
        const float* p = slot(w, c.at >= edge(w) ? 1 : 0);
        const float m = __ldcg(p + r), l = __ldcg(p + kItemRows + r);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p + 2 * kItemRows) + e);
        const float mn = fmaxf(mm, m), mu = mn == -INFINITY ? 0.f : mn;
        const float f = exp2_fast(mm - mu), h = exp2_fast(m - mu);
        mm = mn;
        den = den * f + l * h;
        sum.x = sum.x * f + v.x * h; sum.y = sum.y * f + v.y * h;
        sum.z = sum.z * f + v.z * h; sum.w = sum.w * f + v.w * h;
      }
      const int64_t at = (int64_t)(req.q0 + row / a.group) * a.n_heads + c.h * a.group + row % a.group;
      const bool none = mm == -INFINITY && den == 0.f;
      const float inv = none ? 0.f : 1.0f / den;
      const __nv_bfloat162 y0 = __floats2bfloat162_rn(none ? 0.f : sum.x * inv, none ? 0.f : sum.y * inv);
      const __nv_bfloat162 y1 = __floats2bfloat162_rn(none ? 0.f : sum.z * inv, none ? 0.f : sum.w * inv);
      *reinterpret_cast<uint2*>(g.out + at * D + d) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
      if (d == 0 && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(den) + mm - kShift);
    }
  }
}

template <int D>
int launch(const KvArgs& a, const PromptArgs& g, cudaStream_t st) {
  static OncePerDevice once;
  const int rc = once_per_device(once, [] {
    return cudaFuncSetAttribute(kv_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem<D>);
  });
  if (rc != TLQ_OK) return rc;
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  kv_prompt_kernel<D><<<sms < kMaxWorkers ? sms : kMaxWorkers, kThreads, kSmem<D>, st>>>(a, g);
  return after_launch();
}

}  // namespace

int launch_kv_prompt(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal, int min_rows,
                     uint16_t* out, float* lse, const KvSplit& split, cudaStream_t st) {
  PromptArgs g{};
  g.q = q; g.ldq = ldq; g.out = out; g.lse = lse;
  g.scale_log2 = scale * kLog2e;
  g.causal = causal;
  g.min_rows = min_rows;
  g.split = split;
  return head_dim == 128 ? launch<128>(a, g, st) : launch<64>(a, g, st);
}

}  // namespace tlq
