// Attention of many query rows over the 8-bit cache (prompts and chunks of prompts) on the tensor-memory path.
//
// The formulas are those of kv_attention.cu: scores from (kc + 128) with the 128 sum(q) taken out by a constant of the row,
// p_j = 2^(t_j - m) with t_j = a (q . kc_j) + log2(vstep), output sums of p vc and sums of p / vstep.
//
// A CTA works on 256 rows of one (request, kv head), a row being one query head of one token: two tiles of 128 rows.  Per
// tile and cache block (64 keys): S = q K^T (tcgen05, f16 x f16 -> f32, tensor memory), a thread per row takes the maximum
// and the exponentials of its row from tensor memory and writes P over S as f16, O += P V with P from tensor memory.  S has
// two buffers per tile: while a row's exponentials of one block are taken, the tensor core finishes P V of the block before
// and S of the block after it.  The output sum is rescaled only when the maximum of a row has grown by more than 4.9 (a
// factor of 30 in p): p is kept as 2^11 p, and 2^(11 + 4.9) = 61100 still is a 16-bit float (65504 at most).
//   warps 0..3, 4..7  softmax of tile 0, 1: a thread is a row (and its accumulator lane)
//   warps 8..11       copy the codes of keys and values to shared memory two blocks ahead, turn them into f16 and lay them out
//                     for the tensor core (128-byte swizzle); four stages
//   warps 12, 15      issue the products of tile 0, 1 (one warp for both spends its time waiting: 2500 cycles a block)
//   warp 13           finds the parts of items that this CTA works on and passes them on through a ring
//   warp 14           looks up the cache blocks to come and their steps and passes them on through another ring
// Nothing in the loops may spill: with 225 KB of shared memory in use the first-level cache is too small for local memory, and
// one reload per step costs as much as a product.  A tile without rows is passed over.
// Work is cut as in the few-row kernel: items (row tiles of a kv head) lie on one line, weighted by their cached tokens, every
// CTA takes an equal part of it; an item that is cut leaves partial sums, which kv_join.cu joins.
//
// Bound: 4 D flops per visible pair on the tensor core.  Measured: 8192 tokens, 28 heads over 4 kv heads 558 to 562 us, 860 TFLOP/s
// (292 us at the 1646 TFLOP/s of a large bf16 product); the tensor pipe is active 42 % of the time, the exponential unit 43 %.  A
// block takes about 2200 cycles for 256 rows.  Neither unit bounds it: 554 us without exponentials, 548 without products, 543 without
// both, 519 without the codes' layout too.  What remains is the chain of a block, scores -> maximum -> p -> product, across the
// barriers between the roles, and 8 blocks' worth of time around every item.  Tried on earlier states of this kernel, and slower:
// taking the exponentials from the maximum of the blocks before while this block's is found, the next block's scores loaded before
// P is handed over, two pieces of O rescaled at once.
#include <type_traits>

#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

constexpr int kTile = 128, kItemRows = 256, kKeys = kKvBlock, kStages = 4;
constexpr int kSoftWarps = 8, kLoadWarps = 4, kIssueWarp = kSoftWarps + kLoadWarps, kPlanWarp = kIssueWarp + 1, kScoutWarp = kIssueWarp + 2;
constexpr int kThreads = 512;                              // four groups of four warps
// registers of a thread of each role: 2 x 176 + 72 + 88 = 4 x 128, what the block is launched with
constexpr int kSoftRegs = 176, kLoadRegs = 72, kIssueRegs = 88;
constexpr float kShift = kPromptShift, kGrow = 4.9f;
static_assert(kShift + kGrow < 15.99f, "the largest p has to fit a 16-bit float");
constexpr int kMinTiles = 6;                               // blocks of a CTA's part, at least (512 tokens x 512: 38 us, 40 with 12)
constexpr int kItemCost = 8;                               // what an item costs beside its blocks, in blocks (8192 tokens: 562, 572 with 12)

struct PromptArgs {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* out;
  float* lse;
  float scale_log2;
  int causal;
  KvSplit split;
};

constexpr int kRing = 4;                                   // segments in the planner's ring
constexpr int kTileRing = 16;                              // blocks in the scout's ring
// barriers
enum : int {
  kBarQ = 0,                       // [tile] q is laid out
  kBarS = 2,                       // [tile][buffer] S is complete
  kBarP = 6,                       // [tile][buffer] P is written
  kBarFull = 10,                   // [stage] keys and values of a block are laid out
  kBarFree = kBarFull + kStages,   // [stage] all products of a block have been made
  kBarSegFull = kBarFree + kStages, kBarSegFree = kBarSegFull + kRing,
  kBarTileFull = kBarSegFree + kRing, kBarTileFree = kBarTileFull + kTileRing,
  kBars = kBarTileFree + kTileRing
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
constexpr uint32_t kRawBytes = 2 * kKeys * D;              // codes of a block's keys and values
constexpr int kRaw = 2;                                    // blocks whose codes are under way
template <int D>
constexpr size_t kSmem = 1024 + 2 * kQBytes<D> + kStages * (kKBytes<D> + kVBytes<D>) + kRaw * kRawBytes<D>;

__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// 16 bytes straight to shared memory (`from` of them from global memory, zeros after that), and the wait for such copies
__device__ __forceinline__ void copy16(uint32_t to, const void* p, int from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(p), "r"(from) : "memory");
}
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void copy_mark() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// whether a phase of a barrier is complete, without waiting for it
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(is) : "r"(bar), "r"(parity) : "memory");
  return is != 0;
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
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }   // one instruction here
__device__ __forceinline__ float as_f(uint32_t x) { return __uint_as_float(x); }
// floor(log2 x) of a finite x > 0 (-126 for the smallest), else 0; and 2^n for n in [-126, 127]
__device__ __forceinline__ int exponent_of(float x) {
  const int e = (int)(__float_as_uint(x) >> 23);
  return x == 0.f || e == 255 ? 0 : max(e, 1) - 127;
}
__device__ __forceinline__ float power_of_two(int n) { return __uint_as_float((uint32_t)(n + 127) << 23); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
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

// Scores of keys first .. first + 31 to t, with nothing where there is nothing to see (keys after `see`).
__device__ __forceinline__ void hide(uint32_t (&v)[32], int first, int see, float a, float b) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(first + j <= see ? fmaf(as_f(v[j]), a, b) : -INFINITY);
}

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
  c.tiles = rows >= kPromptRows ? (int)((rows + kItemRows - 1) / kItemRows) : 0;
  const int seen = g.causal ? min(max(r.kv - r.q_len, 0) + kItemRows / a.group, r.kv) : r.kv;
  c.first = 64LL * (kItemCost + 1) + 64LL * seen / kKeys;
  c.more = g.causal ? 64LL * kItemRows / kKeys / a.group : 0;
  return c;
}

// A part of an item: blocks [k0, k1) of n; k0 < 0: there are no more.
struct __align__(16) Segment {
  int b, h, tile, k0;
  int k1, n, q0, q_len;
  long long at, len;            // the item on the line
  int kv, starts, pad[2];       // starts: the item starts in this CTA's part of the line
};

// The blocks [k0, k1) of an item (n of them, at `at` of the line) that the part [from, to) of the line holds.
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

  __device__ __forceinline__ int blocks_seen(const KvArgs& a, const PromptArgs& g) const {
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
      s.n = blocks_seen(a, g);
      cut(x0, x1, s.at, s.len, s.n, s.k0, s.k1);
      s.b = b; s.h = h; s.tile = tile; s.q0 = req.q0; s.q_len = req.q_len; s.kv = req.kv; s.starts = s.at >= x0 ? 1 : 0;
      const bool here = s.n == 0 ? s.at >= x0 : s.k0 < s.k1;   // an item without visible keys belongs to whoever has its start
      ++tile;
      if (here) return true;
    }
  }
};

template <int D>
constexpr size_t kPitch = (size_t)kItemRows * (D + 2);     // floats of a partial: maxima, sums, output sums
template <int D>
__device__ __forceinline__ float* partial_of(const KvSplit& split, int cta, int i) { return prompt_partials(split, D) + ((size_t)cta * 2 + i) * kPitch<D>; }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
kv_prompt_kernel(const KvArgs a, const PromptArgs g) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + 2 * kQBytes<D>, v_at = k_at + kStages * kKBytes<D>, raw_at = v_at + kStages * kVBytes<D>;
  __shared__ __align__(8) uint64_t bars[kBars];
  __shared__ Segment s_ring[kRing];
  __shared__ __align__(16) float4 s_steps[kTileRing];      // of a block: kstep, log2 vstep, 1 / vstep, usable
  __shared__ int s_block[kTileRing];                       // and where it is (block x kv heads + head)
  __shared__ long long sums[kThreads / 32];
  __shared__ Found found;
  __shared__ long long s_from, s_to;                       // this CTA's part of the line
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;   // warp: known to be uniform
  auto bar = [&](int i) { return ptx::smem_u32(&bars[i]); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) ptx::mbar_init(bar(kBarQ + i), 4);
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(bar(kBarS + i), 1);
      ptx::mbar_init(bar(kBarP + i), 4);
    }
    for (int i = 0; i < kStages; ++i) {
      ptx::mbar_init(bar(kBarFull + i), kLoadWarps);
      ptx::mbar_init(bar(kBarFree + i), 2);
    }
    for (int i = 0; i < kRing; ++i) {
      ptx::mbar_init(bar(kBarSegFull + i), 1);
      ptx::mbar_init(bar(kBarSegFree + i), kSoftWarps + 3);
    }
    for (int i = 0; i < kTileRing; ++i) {
      ptx::mbar_init(bar(kBarTileFull + i), 1);
      ptx::mbar_init(bar(kBarTileFree + i), 1);
    }
    s_abort = 0;
    ptx::fence_barrier_init();
  }
  volatile int* abort_flag = &s_abort;

  after_previous();
  auto no_parts = [&]() { prompt_notes(g.split, D)[2 * blockIdx.x].item = prompt_notes(g.split, D)[2 * blockIdx.x + 1].item = -1; };
  if (threadIdx.x == 0) no_parts();
  if (!is_prompt_work<kThreads>(a, g.causal, sums)) return;   // left to the few-row kernel
  // ---------------------------------------------------------------- this CTA's part of the line
  auto cost_of = [&](int b) {
    const Costs c = costs_of(a, g, load_request(a, b));
    return c.sum(c.tiles) * a.n_kv;
  };
  {
    // a part is worth joining from some blocks on
    auto workers_of = [&](long long all) { return max(1LL, min((long long)gridDim.x, all / (64 * kMinTiles))); };
    long long total = 0;
    if (!plan_items<kThreads>(a.B, cost_of,
                              [&](long long all) {
                                const long long n = workers_of(all);
                                return blockIdx.x < n && all * blockIdx.x / n < all * (blockIdx.x + 1) / n ? all * blockIdx.x / n : -1LL;
                              },
                              sums, &found, total))
      return;
    if (threadIdx.x == 0) {                                // read back where they are needed: the loops have no registers to spare
      const long long n = workers_of(total);
      s_from = total * blockIdx.x / n; s_to = total * (blockIdx.x + 1) / n;
    }
  }
  if (warp == kIssueWarp) ptx::tmem_alloc(ptx::smem_u32(&s_tmem), 512);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = s_tmem;                            // S of tile t, buffer i at column 128 t + 64 i; O at 256 + 128 t
  // the next segment, by all lanes of a warp (or the one that issues)
  int seg = 0;
  uint32_t seg_phase = 0;
  auto next_segment = [&](bool& ok) {
    ok = ptx::mbar_wait(bar(kBarSegFull + seg), seg_phase, abort_flag);
    return &s_ring[seg];
  };
  auto done_segment = [&]() {                              // its fields have been read
    ptx::mbar_arrive(bar(kBarSegFree + seg));
    if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
  };

  auto tile_live = [&](const Segment* s, int t) {          // whether it has rows at all
    return (long long)s->tile * kItemRows + t * kTile < (long long)s->q_len * a.group;
  };
  // waits until all products of a block are complete (block number st of this CTA, none before st - kStages open)
  auto products_of = [&](int st) {
    return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(kBarFree + st % kStages), (uint32_t)(st / kStages) & 1u, abort_flag)) != 0;
  };

  // ------------------------------------------------------------------ products of tile T, by a whole warp
  // All lanes keep step, so that addresses and descriptors stay in uniform registers; one of them issues.
  auto issue = [&](auto tile_of) {
    constexpr int T = decltype(tile_of)::value;
    constexpr uint32_t kIdescS = ptx::make_idesc(1, 0, kTile, kKeys, false);   // f16 x f16 -> f32
    constexpr uint32_t kIdescO = ptx::make_idesc(1, 0, kTile, D, false);
    const bool leader = elect_one();
    int step = 0, passed = 0;                              // blocks so far, of all segments; those without a row of this tile
    uint32_t q_phase = 0;
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) { ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(i), parity, abort_flag)) != 0; };
    auto scores = [&](int st) {                            // S of block number st into its buffer
      const int buf = (st - passed) & 1;
      if (leader) {
#pragma unroll
        for (uint32_t c = 0; c < kPanels<D>; ++c) {
          const uint64_t x = ptx::smem_desc_sw128(q_at + T * kQBytes<D> + c * (kTile * 128));
          const uint64_t y = ptx::smem_desc_sw128(k_at + (st % kStages) * kKBytes<D> + c * (kKeys * 128));
#pragma unroll
          for (int i = 0; i < 4; ++i) mma_f16_ss(tmem + T * kTile + buf * kKeys, x + 2 * i, y + 2 * i, kIdescS, c > 0 || i > 0);
        }
        ptx::mma_commit(bar(kBarS + 2 * T + buf));
      }
      __syncwarp();
    };
    while (true) {
      const Segment* from = next_segment(ok);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const int k0 = from->k0, k1 = from->k1;
      const bool live = tile_live(from, T);
      __syncwarp();
      if (lane == 0) done_segment(); else if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
      if (k0 < 0) break;
      if (k0 >= k1) continue;
      if (!live) {                                         // no rows: the blocks pass
        for (int k = k0; k < k1 && ok; ++k, ++step, ++passed) {
          wait(kBarFull + step % kStages, (uint32_t)(step / kStages) & 1u);
          if (ok && lane == 0) ptx::mbar_arrive(bar(kBarFree + step % kStages));
        }
        if (!ok) break;
        continue;
      }
      wait(kBarQ + T, q_phase);
      if (!ok) break;
      ptx::tc_fence_after();
      q_phase ^= 1u;
      for (int st = step; st < step + 2 && st < step + k1 - k0 && ok; ++st) {
        wait(kBarFull + st % kStages, (uint32_t)(st / kStages) & 1u);
        if (ok) scores(st);
      }
      for (int k = k0; k < k1 && ok; ++k, ++step) {
        const int stage = step % kStages, ahead = step + 2, turn = step - passed;
        if (k + 2 < k1) wait(kBarFull + ahead % kStages, (uint32_t)(ahead / kStages) & 1u);   // long ready, off the chain P -> S
        if (!ok) break;
        wait(kBarP + 2 * T + (turn & 1), (uint32_t)(turn >> 1) & 1u);
        if (!ok) break;
        ptx::tc_fence_after();
        if (leader) {
          const uint64_t y = ptx::smem_desc_sw128(v_at + stage * kVBytes<D>);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mma_f16_ts(tmem + 256 + T * kTile, tmem + T * kTile + (turn & 1) * kKeys + 8 * i, y + 2 * i, kIdescO, k > k0 || i > 0);
        }
        if (k + 2 < k1) scores(ahead);
        if (leader) ptx::mma_commit(bar(kBarFree + stage));
        __syncwarp();
      }
    }
    if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 233);
  };

  if (warp < kSoftWarps) {
    more_registers<kSoftRegs>();
    // ------------------------------------------------------------------ softmax: a thread is a row
    const int t = warp >> 2, row_in_tile = (warp & 3) * 32 + lane;
    const uint32_t s_col = tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * kTile, o_col = s_col + 256;   // P over S
    constexpr int kRowLanes = D / 8, kRowsAtOnce = 32 / kRowLanes;       // lanes that hold a row, 16 bytes each
    int step = 0, passed = 0;                              // blocks so far, of all segments; those without a row of this tile
    bool ok = true;
    while (true) {
      const Segment* s = next_segment(ok);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok || s->k0 < 0) break;
      const int k0 = s->k0, k1 = s->k1;
      if (threadIdx.x == 0 && (k0 > 0 || k1 < s->n)) {
        PartNote* note = prompt_notes(g.split, D) + 2 * blockIdx.x + s->starts;
        note->item = s->at;
        note->first = k0 == 0; note->last = k1 == s->n;
        note->h = s->h; note->tile = s->tile; note->q0 = s->q0; note->q_len = s->q_len;
      }
      if (!tile_live(s, t)) {
        step += k1 - k0;
        passed += k1 - k0;
        __syncwarp();
        if (lane == 0) done_segment(); else if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
        continue;
      }
      const int row = s->tile * kItemRows + t * kTile + row_in_tile, token = row / a.group;
      const bool live = token < s->q_len;
      const int limit = !live ? -1 : g.causal ? min(s->kv - s->q_len + token, s->kv - 1) : s->kv - 1;
      float fac = 0.f, off = 0.f;
      if (k0 < k1) {
        // The warp's 32 rows of q come in whole, kRowLanes lanes to a row, straight to their place in shared memory; then every
        // lane turns its own row into f16 there, after a power of two that brings it into range.  In rolled loops: this is run
        // once per item, and code that runs once is slower to fetch than to execute.
        const int64_t from = live ? (int64_t)(s->q0 + token) * g.ldq + (int64_t)(s->h * a.group + row - token * a.group) * D : -1;
        const uint32_t tile_at = q_at + t * kQBytes<D>;
#pragma unroll 1
        for (int i = 0; i < D / 8; ++i) {
          const int at = i * kRowsAtOnce + lane / kRowLanes, r = (warp & 3) * 32 + at, piece = lane % kRowLanes;
          const int64_t p = __shfl_sync(0xFFFFFFFFu, from, at);
          const uint32_t to = tile_at + (piece >> 3) * (kTile * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
          copy16(to, p >= 0 ? g.q + p + 8 * piece : g.q, p >= 0 ? 16 : 0);
        }
        copy_wait();
        __syncwarp();
        const uint32_t mine = tile_at + row_in_tile * 128;
        float top = 0.f;
#pragma unroll 2
        for (int i = 0; i < D / 8; ++i) {
          float e[8];
          unpack8(lds128(mine + (i >> 3) * (kTile * 128) + (((i & 7) ^ (row_in_tile & 7)) << 4)), e);
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(e[j]));
        }
        const int ex = exponent_of(top);
        const float d0 = power_of_two(-(ex / 2)), d1 = power_of_two(-(ex - ex / 2));
        float qs = 0.f;
#pragma unroll 2
        for (int i = 0; i < D / 8; ++i) {
          const uint32_t at = mine + (i >> 3) * (kTile * 128) + (((i & 7) ^ (row_in_tile & 7)) << 4);
          float e[8];
          unpack8(lds128(at), e);
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] = pack_f16(e[2 * j] * d0 * d1, e[2 * j + 1] * d0 * d1);
            const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
            qs += z.x + z.y;
          }
          sts128(at, w[0], w[1], w[2], w[3]);
        }
        off = qs * (128.f / kUnit);
        fac = ldexpf(g.scale_log2, ex + 24);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(kBarQ + t));
      }

      float m = -INFINITY, l = 0.f;
      for (int k = k0; k < k1; ++k, ++step) {
        const int turn = step - passed, buf = (turn & 1) * kKeys;
        ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(kBarS + 2 * t + (turn & 1)), (uint32_t)(turn >> 1) & 1u, abort_flag));
        if (!ok) break;
        ptx::tc_fence_after();
        uint32_t v[2][32];                                 // the row of S
        ptx::tmem_ld32(s_col + buf, v[0]);
        ptx::tmem_ld32(s_col + buf + 32, v[1]);
        const float4 w = s_steps[step % kTileRing];
        float fa = fac * w.x, fb = fmaf(-off, fa, w.y);
        const int see = w.w == 0.f ? -1 : limit - k * kKeys;   // last key of the block that the row sees
        const bool masked = __any_sync(0xFFFFFFFFu, see < kKeys - 1);
        tmem_ld_wait_for(v[0]);
        tmem_ld_wait_for(v[1]);
        if (masked) {
          hide(v[0], 0, see, fa, fb);
          hide(v[1], 32, see, fa, fb);
          fa = 1.f;                                        // the hidden rows are t already
          fb = 0.f;
        }
        float r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = max3(as_f(v[0][j]), as_f(v[0][4 + j]), as_f(v[0][8 + j]));
#pragma unroll
        for (int j = 12; j < 28; j += 8)
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = max3(r[i], as_f(v[0][j + i]), as_f(v[0][j + 4 + i]));
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = max3(r[i], as_f(v[0][28 + i]), as_f(v[1][i]));
#pragma unroll
        for (int j = 4; j < 28; j += 8)
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = max3(r[i], as_f(v[1][j + i]), as_f(v[1][j + 4 + i]));
        const float top = fmaf(fmaxf(max3(r[0], r[1], r[2]), max3(r[3], max3(as_f(v[1][28]), as_f(v[1][29]), as_f(v[1][30])), as_f(v[1][31]))), fa, fb);
        // a maximum that has grown by more than kGrow: the output sum follows
        if (__any_sync(0xFFFFFFFFu, top > m + kGrow || (m == -INFINITY && top > -INFINITY))) {
          const float mn = fmaxf(m, top);
          const float corr = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
          m = mn;
          l *= corr;
          if (k > k0) {
            ok = products_of(step - 1);                    // P V of the block before has to be in it
            if (!ok) break;
            ptx::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t x[32];
              ptx::tmem_ld32(o_col + 32 * c, x);
              tmem_ld_wait_for(x);
#pragma unroll
              for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(as_f(x[j]) * corr);
              tmem_st32(o_col + 32 * c, x);
            }
          }
        }
        fb += kShift - (m == -INFINITY ? 0.f : m);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float y, z;
            fma2(y, z, fa, as_f(v[c][j]), as_f(v[c][j + 1]), fb);
            y = exp2_fast(y);
            z = exp2_fast(z);
            add2(sum[0], sum[1], y, z);
            p[j / 2] = pack_f16(y, z);
          }
          tmem_st16(s_col + buf + 16 * c, p);              // all of S has been read
        }
        const float both = sum[0] + sum[1];
        l += both > 0.f ? both * w.z : both;
        tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(kBarP + 2 * t + (turn & 1)));
      }
      if (!ok) break;

      // ---------------------------------------------------------------- leave the item
      if (k0 < k1) {
        ok = products_of(step - 1);
        if (!ok) break;
        ptx::tc_fence_after();
      }
      {
        const bool none = m == -INFINITY && l == 0.f;      // a row that sees nothing (a NaN row has a NaN sum)
        const bool whole = k0 == 0 && k1 == s->n;
        const float inv = none ? 0.f : 1.0f / l;
        const int64_t at = live ? (int64_t)(s->q0 + token) * a.n_heads + s->h * a.group + row - token * a.group : -1;
        // through the shared memory of the warp's own rows of q, which nobody reads any more, so that whole rows are stored:
        // all channels as bf16, in the layout of q, or 32 channels at a time as they are (for a partial)
        const uint32_t mine = q_at + t * kQBytes<D> + (warp & 3) * (32 * 128);
        float* part = partial_of<D>(g.split, blockIdx.x, s->starts) + 2 * kItemRows + (size_t)(t * kTile + (warp & 3) * 32) * D;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          if (k0 < k1) {
            ptx::tmem_ld32(o_col + 32 * c, v);
            tmem_ld_wait_for(v);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0u;
          }
          if (whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 z = __floats2bfloat162_rn(none ? 0.f : as_f(v[8 * i + 2 * j]) * inv,
                                                               none ? 0.f : as_f(v[8 * i + 2 * j + 1]) * inv);
                y[j] = *reinterpret_cast<const uint32_t*>(&z);
              }
              sts128(mine + (c >> 1) * (kTile * 128) + lane * 128 + (((4 * (c & 1) + i) ^ (lane & 7)) << 4), y[0], y[1], y[2], y[3]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) sts128(mine + lane * 128 + ((i ^ (lane & 7)) << 4), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            __syncwarp();
#pragma unroll 2
            for (int i = 0; i < 8; ++i) {
              const int r = 4 * i + (lane >> 3), piece = lane & 7;
              reinterpret_cast<uint4*>(part + (size_t)r * D + 32 * c)[piece] = lds128(mine + r * 128 + ((piece ^ (r & 7)) << 4));
            }
          }
          __syncwarp();
        }
        if (whole) {
#pragma unroll 2
          for (int i = 0; i < D / 8; ++i) {
            const int r = i * kRowsAtOnce + lane / kRowLanes, piece = lane % kRowLanes;
            const int64_t to = __shfl_sync(0xFFFFFFFFu, at, r);
            const uint4 y = lds128(mine + (piece >> 3) * (kTile * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4));
            if (to >= 0) reinterpret_cast<uint4*>(g.out + to * D)[piece] = y;
          }
          if (live && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(l) + m - kShift);
        } else {
          float* stats = partial_of<D>(g.split, blockIdx.x, s->starts) + t * kTile + row_in_tile;
          stats[0] = m;
          stats[kItemRows] = l;
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
    // A warp takes 8 rows x 64 bytes at a time.  Keys: row group lw / panels + i * 4 / panels of 8, the same panel for all i;
    // values: row group lw + 4 i of D / 8.
    constexpr int kNum = D / 32, kGroups = 4 / kPanels<D>;   // pieces of a warp; key row groups that the warps take at a time
    const int lw = warp - kSoftWarps, lr = lane & 7, piece = lane >> 3;
    const int k_row = (lw / kPanels<D>) * 8 + lr, k_panel = lw % kPanels<D>;
    const int8_t* const k_from = a.k_codes + k_row * D + k_panel * 64 + piece * 16;
    const int8_t* const v_from = a.v_codes + (lw * 8 + lr) * kKvBlock + piece * 16;
    const uint32_t swizzled0 = ((2 * piece) ^ lr) << 4, swizzled1 = ((2 * piece + 1) ^ lr) << 4;
    const uint32_t k_to = k_at + k_panel * (kKeys * 128) + k_row * 128, v_to = v_at + (lw * 8 + lr) * 128;
    // Codes of the next kRaw blocks are under way to places in shared memory that belong to one thread each, so that no
    // barrier is needed between their arrival and their use, and no register while they travel.
    const uint32_t raw = raw_at + (threadIdx.x - kSoftWarps * 32) * 16;
    constexpr uint32_t kRawStep = kLoadWarps * 32 * 16;
    int step = 0, fetched = 0;                             // blocks laid out, blocks asked for
    bool ok = true, more = true;
    // Asks for the next block of the scout's ring; waits for the ring only when there is nothing to lay out meanwhile, since
    // the scout may be waiting for what that completes (items in which nobody sees a key have no blocks).
    auto fetch = [&]() {
      const int at = fetched % kTileRing;
      const uint32_t full = bar(kBarTileFull + at), parity = (uint32_t)(fetched / kTileRing) & 1u;
      if (fetched > step) {
        if (!__all_sync(0xFFFFFFFFu, mbar_test(full, parity))) return;
      } else {
        ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(full, parity, abort_flag));
        if (!ok) return;
      }
      const int64_t block = (int64_t)s_block[at] * (kKvBlock * D);
      more = block >= 0;
      if (!more) return;
      const uint32_t to = raw + fetched % kRaw * kRawBytes<D>;
#pragma unroll
      for (int i = 0; i < kNum; ++i) copy16(to + i * kRawStep, k_from + block + i * kGroups * 8 * D, 16);
#pragma unroll
      for (int i = 0; i < kNum; ++i) copy16(to + (kNum + i) * kRawStep, v_from + block + i * 32 * kKvBlock, 16);
      copy_mark();
      ++fetched;
    };
    while (true) {
      while (more && ok && fetched - step < kRaw) {
        const int before = fetched;
        fetch();
        if (fetched == before) break;
      }
      if (!ok || fetched == step) break;
      if (fetched - step == kRaw) copy_wait_but<kRaw - 1>(); else copy_wait();
      const int stage = step % kStages;
      const uint32_t in = raw + step % kRaw * kRawBytes<D>;
      if (step >= kStages) {                               // the stage is free, and so is what the scout noted of its block
        ok = products_of(step - kStages);
        if (!ok) break;
        if (lw == 0 && lane == 0) ptx::mbar_arrive(bar(kBarTileFree + (step - kStages) % kTileRing));
      }
#pragma unroll
      for (int i = 0; i < kNum; ++i) {
        const uint32_t to = k_to + stage * kKBytes<D> + i * kGroups * 8 * 128;
        const uint4 y = lds128(in + i * kRawStep);
        uint32_t x[8];
        keys_to_f16(y.x, x[0], x[1]); keys_to_f16(y.y, x[2], x[3]);
        keys_to_f16(y.z, x[4], x[5]); keys_to_f16(y.w, x[6], x[7]);
        sts128(to + swizzled0, x[0], x[1], x[2], x[3]);
        sts128(to + swizzled1, x[4], x[5], x[6], x[7]);
      }
#pragma unroll
      for (int i = 0; i < kNum; ++i) {
        const uint32_t to = v_to + stage * kVBytes<D> + i * 32 * 128;
        const uint4 y = lds128(in + (kNum + i) * kRawStep);
        uint32_t x[8];
        values_to_f16(y.x, x[0], x[1]); values_to_f16(y.y, x[2], x[3]);
        values_to_f16(y.z, x[4], x[5]); values_to_f16(y.w, x[6], x[7]);
        sts128(to + swizzled0, x[0], x[1], x[2], x[3]);
        sts128(to + swizzled1, x[4], x[5], x[6], x[7]);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(kBarFull + stage));
      ++step;
    }
    copy_wait();
    if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 232);
  } else {
    fewer_registers<kIssueRegs>();
    if (warp == kIssueWarp) {
      issue(std::integral_constant<int, 0>{});
    } else if (warp == kIssueWarp + 3) {
      issue(std::integral_constant<int, 1>{});
    } else if (warp == kPlanWarp && lane == 0) {
      // ---------------------------------------------------------------- segments
      Walk walk;
      walk.start(a, g, found.request, found.rest, s_from, s_to);
      uint32_t phase = 1;
      while (true) {
        Segment s;
        const bool more = walk.next(a, g, s);
        if (!more) s.k0 = -1;
        if (!ptx::mbar_wait(bar(kBarSegFree + seg), phase, abort_flag)) {
          report_status(a.hdr, TLQ_ERR_TIMEOUT, 234);
          break;
        }
        s_ring[seg] = s;
        ptx::mbar_arrive(bar(kBarSegFull + seg));
        if (!more) break;
        if (++seg == kRing) { seg = 0; phase ^= 1u; }
      }
    } else if (warp == kScoutWarp) {
      // ---------------------------------------------------------------- the cache blocks to come, and their steps
      int step = 0;
      bool ok = true;
      while (ok) {
        const Segment* from = next_segment(ok);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        const int k0 = from->k0, k1 = from->k1, h = from->h;
        const int32_t* table = a.block_table + (int64_t)from->b * a.max_blocks;
        __syncwarp();
        if (lane == 0) done_segment(); else if (++seg == kRing) { seg = 0; seg_phase ^= 1u; }
        const int last = k0 < 0 ? k0 + 1 : k1;             // the end is passed on as a block that is none
        for (int k = k0; k < last && ok; k += 32) {
          const bool in = k0 >= 0 && k + lane < last;      // a lane for each of 32 blocks
          const int phys = in ? load_near(table + k + lane) : -1;
          const bool usable = phys >= 0 && phys < a.n_blocks;
          if (in && !usable) report_status(a.hdr, TLQ_ERR_SHAPE, 231);
          const int64_t at = (int64_t)(usable ? phys : 0) * a.n_kv + h;
          const float ks = load_near(a.k_steps + at), vs = load_near(a.v_steps + at), v = vs < kStepFloor ? kStepFloor : vs;
          const float4 w = make_float4(ks, log2f(v), 1.0f / v, usable ? 1.f : 0.f);
          for (int j = 0; j < min(32, last - k); ++j, ++step) {
            const int to = step % kTileRing;
            ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar(kBarTileFree + to), ((uint32_t)(step / kTileRing) & 1u) ^ 1u, abort_flag));
            if (!ok) break;
            if (lane == j) {
              s_steps[to] = w;
              s_block[to] = k0 < 0 ? -1 : (int)at;
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(kBarTileFull + to));
          }
        }
        if (k0 < 0) break;
      }
      if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 235);
    }
  }
  __syncwarp();
  if (*abort_flag != 0)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);      // products under way end before their memory is given back
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  if (*abort_flag != 0 && threadIdx.x == 0) no_parts();
}

template <int D>
int launch(const KvArgs& a, const PromptArgs& g, int ctas, cudaStream_t st) {
  static OncePerDevice once;
  const int rc = once_per_device(once, [] {
    return cudaFuncSetAttribute(kv_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem<D>);
  });
  if (rc != TLQ_OK) return rc;
  return launch_next(kv_prompt_kernel<D>, dim3((unsigned)ctas), kThreads, kSmem<D>, 1, st, a, g);
}

}  // namespace

int launch_kv_prompt(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal, uint16_t* out,
                     float* lse, const KvSplit& split, int ctas, cudaStream_t st) {
  PromptArgs g{};
  g.q = q; g.ldq = ldq; g.out = out; g.lse = lse;
  g.scale_log2 = scale * kLog2e;
  g.causal = causal;
  g.split = split;
  return head_dim == 128 ? launch<128>(a, g, ctas, st) : launch<64>(a, g, ctas, st);
}

}  // namespace tlq
