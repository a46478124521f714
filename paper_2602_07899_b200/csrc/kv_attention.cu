// Attention of few query rows over the 8-bit cache (decoding, drafted tokens): one pass over the cache.
//
//   o = sum_j softmax_j(scale * q . k_j) v_j,   k_j = kc_j * kstep(block of j),  v_j = vc_j * vstep(block of j).
//
// The steps never touch an element of the cache: with a = scale * log2(e) * kstep and b = log2(vstep) the kernel works on
// t_j = a (q . kc_j) + b and p_j = 2^(t_j - m), so that o = sum p_j vc_j / sum p_j / vstep, where the running maximum m
// is taken over t.  8-bit codes are exact in 16-bit floats, so both products run on the matrix instruction m16n8k16 in
// f16 with 32-bit sums.  For the scores it is cheaper to multiply by kc + 128 (three byte operations make four operands):
// the 128 sum(q) that this adds is a constant of a column and becomes part of b.
// q enters as f16 after a power of two per row that brings its largest element to [1, 2) (exact
// for all but elements 2^-14 below it); p enters as f16 scaled by 2^15, which keeps 11 bits for every p_j >= 2^-29 of the
// largest.  Maximum, sums and the output sum are 32-bit.
//
// Layout.  All query heads of a kv head (and the tokens of a short draft) are the 8 or 16 columns of the products
// S^T = K q^T (m = 16 tokens) and O^T = V^T P^T (m = 16 channels): with the cache on the m side no lane is idle when there
// are only 8 rows.  Which token or channel a matrix index means is free as long as both operands agree, so every lane
// reads its operands as whole 16-byte pieces of a row.  The probabilities change from result layout to operand layout by
// movmatrix.
//
// Split.  A unit is one block of 64 tokens of one (request, kv head, row tile).  All units form one line that is cut into
// equal parts, one per warp, whatever the requests' lengths.  A warp walks its part alone, with a ring of asynchronous
// copies of its own that runs ahead over item boundaries; it writes the items that lie inside its part, and leaves
// partial sums of at most two that do not, which kv_join.cu joins.
//
// Bound: the cache's bytes, 16 KB per block and kv head at 128 channels.  The ring holds 24 KB per warp, 192 KB per SM: at
// 44 GB/s and about 2 us per SM some 90 KB have to be under way all the time.  Measured: 64 requests of up to 32761 tokens,
// 4 kv heads (370 MB) 80 us, 57 of them from the first to the last block (6.5 TB/s); one token over 131071 with 8 kv heads
// (268 MB) 60 us, 42 for the blocks; the rest is the launch, the plan (2 us), the end of the grid and the join.  One token
// over 100: 8.4 us.  Items of 16 rows (16 columns) cost twice the matrix work: 8 requests of one token over 8192 keys take 27 us,
// 8 of 5 tokens (35 rows, three items for each of 4 kv heads) 56.
#include "serve.cuh"
#include "umma.cuh"

namespace tlq {
namespace {

constexpr int kWarps = kSplitWarps;
constexpr int kThreads = kWarps * 32;
constexpr float kShift = kFewShift;       // p is kept as 2^kShift * p in 16 bits

struct AttnArgs {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* out;
  float* lse;
  float scale_log2;          // scale * log2(e)
  int causal, prompts;       // prompts: the prompt kernel has run before (and may have had something to do)
  int whole;                 // items of up to this many blocks are not cut
  KvSplit split;
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
// Copy of `bytes` (a multiple of 16) that counts on the barrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Units of a request: row tiles x kv heads x (blocks + kItemUnits); blocks is one for a request without cached tokens, whose
// rows are empty.  What an item costs beside its blocks (its queries, its result) takes as long as kItemUnits blocks.
constexpr int kItemUnits = 1;
// Small items are not cut: the warp that has the unit before their blocks takes them all, and nothing has to be joined (nor the
// join launched, where no request can have more blocks: that alone is 5 us).  A single request of 500 tokens (8 blocks) is
// answered in 12 us cut and in 17 whole; 64 of them, an item or more for every CTA, in 27 cut and in 25 whole, 64 of 300 tokens
// in 23 and 14, 64 of 100 in 21 and 10.
constexpr int kWhole = 4, kWholeBusy = 8;                  // blocks, at most; where there may be an item for every CTA
// The units go to as many CTAs as there are, then to warps that get about this many: every part has to be joined.  One token
// over 60000 with 2 kv heads 37, 31 and 29 us for 2, 3 and 4, over 16384 with 8 25, 22 and 23; 9 tokens over 4096 with 4 kv heads
// 20, 21 and 24, 16 requests of 700 tokens 16, 19 and 19, 64 of 500 tokens 25, 25 and 20.
constexpr int kMinUnits = 3;
struct Units {
  int row_tiles, blocks;
  long long total;
};
__device__ __forceinline__ Units units_of(const KvArgs& a, const Request& r, int row_tile, int max_rows) {
  Units u;
  const long long rows = (long long)r.q_len * a.group;
  u.row_tiles = rows < max_rows ? (int)((rows + row_tile - 1) / row_tile) : 0;
  u.blocks = r.kv > 0 ? (r.kv + kKvBlock - 1) / kKvBlock : 1;
  u.total = (long long)u.row_tiles * a.n_kv * (u.blocks + kItemUnits);
  return u;
}


// A place on the line of units: block `blk` of an item (request b, kv head h, row tile), or one of the units before it (blk < 0).
struct Walker {
  int b, h, tile, blk, max_rows;
  Request req;
  Units un;

  __device__ __forceinline__ void enter(const KvArgs& a, int request, int row_tile) {
    b = request;
    req = load_request(a, b);
    un = units_of(a, req, row_tile, max_rows);
  }
  // `rest` units into request `request`
  __device__ __forceinline__ void start(const KvArgs& a, int request, long long rest, int row_tile) {
    enter(a, request, row_tile);
    const long long item = rest / (un.blocks + kItemUnits);
    blk = (int)(rest - item * (un.blocks + kItemUnits)) - kItemUnits;
    h = (int)(item / un.row_tiles);
    tile = (int)(item - (long long)h * un.row_tiles);
  }
  // to the first unit of the next item
  __device__ __forceinline__ void next_item(const KvArgs& a, int row_tile) {
    blk = -kItemUnits;
    if (++tile < un.row_tiles) return;
    tile = 0;
    if (++h < a.n_kv) return;
    h = 0;
    do {
      if (b + 1 >= a.B) return;                            // past the end: nobody looks further
      enter(a, b + 1, row_tile);
    } while (un.total == 0);
  }
};

// Row of the output that column c of an item belongs to.
__device__ __forceinline__ int64_t out_row(const KvArgs& a, const Request& r, int h, int row) {
  return (int64_t)(r.q0 + row / a.group) * a.n_heads + h * a.group + row % a.group;
}

template <int D>
constexpr int kAhead = D == 128 ? 2 : 3;                   // blocks that the ring runs ahead
template <int D>
constexpr int kChunks = 2 * kAhead<D> - 1;                 // a chunk is the keys, or the values, of one block
template <int D>
constexpr size_t kRingBytes = (size_t)kWarps * kChunks<D> * kKvBlock * D;

// Rows of no request see nothing.  The last CTAs see to it, when they have done their own: 0.3 us less than all of them before they
// begin (one token over 100: 8.4 and 8.6); out of line, since code that is not run should not be fetched either.
constexpr unsigned kPadCtas = 16;
template <int D>
__device__ __noinline__ void empty_rows(const Padding pad, int64_t T, int n_heads, uint16_t* out, float* lse) {
  const int64_t t = (int64_t)(gridDim.x - 1 - blockIdx.x) * kThreads + threadIdx.x, n = (int64_t)min(kPadCtas, gridDim.x) * kThreads;
  zero_rows(out, 0, pad.before, (int64_t)n_heads * D / 8, t, n);
  zero_rows(out, pad.after, T, (int64_t)n_heads * D / 8, t, n);
  if (lse == nullptr) return;
  for (int64_t i = t; i < (int64_t)pad.before * n_heads; i += n) lse[i] = -INFINITY;
  for (int64_t i = (int64_t)pad.after * n_heads + t; i < T * n_heads; i += n) lse[i] = -INFINITY;
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 1)
kv_attention_kernel(const KvArgs a, const AttnArgs g) {
  constexpr int kRows = 8 * NT;
  constexpr int kRing = kChunks<D>, kDeep = kAhead<D>;
  constexpr uint32_t kBytes = kKvBlock * D;
  constexpr size_t kPitch = (size_t)kRows * (D + 2);       // floats of a partial
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t s_bars[kWarps * kRing];
  __shared__ long long sums[kWarps];
  __shared__ Found found;
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gr = lane >> 2, tq = lane & 3;

  // ---------------------------------------------------------------- this CTA's part of the line of units
  if (threadIdx.x == 0) s_abort = 0;
  if (lane == 0) {
    for (int i = 0; i < kRing; ++i) ptx::mbar_init(ptx::smem_u32(&s_bars[warp * kRing + i]), 1);
    ptx::fence_barrier_init();
  }
  after_previous();
  if (blockIdx.x == 0 && threadIdx.x == 0) *few_workers(g.split, D) = 0;
  const int max_rows = g.prompts && is_prompt_work<kThreads>(a, g.causal, sums) ? kPromptRows : 0x7FFFFFFF;
  auto count_units = [&](int b) { return units_of(a, load_request(a, b), kRows, max_rows).total; };
  auto workers_of = [&](long long all) { return min(all, (long long)gridDim.x); };
  long long total = 0;
  Padding pad{0, (int)a.T};
  if (blockIdx.x + kPadCtas >= gridDim.x) pad = load_padding(a.cu_q, a.B, a.T);
  auto padding = [&]() {
    if (pad.before > 0 || pad.after < a.T) empty_rows<D>(pad, a.T, a.n_heads, g.out, g.lse);
  };
  const bool some = plan_items<kThreads>(a.B, count_units,
                                         [&](long long all) { return (long long)blockIdx.x < workers_of(all) ? all * blockIdx.x / workers_of(all) : -1LL; },
                                         sums, &found, total);
  if (!some) {
    padding();
    return;
  }
  const long long workers = workers_of(total);
  const long long u_begin = total * blockIdx.x / workers, u_end = total * (blockIdx.x + 1) / workers;

  // ---------------------------------------------------------------- this warp's part of it
  const int active = (int)min((total + workers * kMinUnits - 1) / (workers * kMinUnits), (long long)kWarps);   // warps of every CTA
  auto bound_of = [&](int w) { return w >= active ? u_end : u_begin + (u_end - u_begin) * w / active; };
  const long long w_begin = bound_of(warp), w_end = bound_of(warp + 1);
  const uint32_t ring = ptx::smem_u32(smem) + warp * (kRing * kBytes);
  const uint32_t bars = ptx::smem_u32(&s_bars[warp * kRing]);
  // the warp's parts: of an item that began before it, of an item that goes on after it
  const size_t worker = (size_t)blockIdx.x * active + warp;
  PartNote* const notes = few_notes(g.split, D) + 2 * worker;
  if (warp < active && lane < 2) notes[lane].item = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) *few_workers(g.split, D) = (int)workers * active;
  __syncwarp();

  if (w_begin < w_end) {
    Walker con;                                            // what is computed now
    con.max_rows = max_rows;
    {
      int b = found.request;
      long long rest = found.rest + (w_begin - u_begin);
      con.enter(a, b, kRows);
      while (rest >= con.un.total) {                       // the part may begin some requests after the CTA's
        rest -= con.un.total;
        con.enter(a, ++b, kRows);
      }
      con.start(a, b, rest, kRows);
    }
    long long unit = w_begin;
    if (con.un.blocks <= g.whole && con.blk > -kItemUnits) {   // an item that the warp before this one takes
      unit += con.un.blocks - con.blk;
      con.next_item(a, kRows);
    }
    Walker pro = con;                                      // what is copied next
    long long pro_left = w_end - unit;
    // steps and first places of the blocks under way
    float q_k[kDeep], q_v[kDeep];
    int q_base[kDeep];
    int phys = 0;                                          // of the block at `pro`
    const int8_t* v_src = nullptr;                         // values of the block whose keys were copied last
    // leaves the units before an item's blocks (and items of requests without cached tokens) and looks the block up
    auto look_up = [&]() {
      while (pro_left > 0) {
        if (pro.blk < 0) {
          pro_left += pro.blk;
          pro.blk = 0;
          if (pro.un.blocks <= g.whole) pro_left = max(pro_left, (long long)pro.un.blocks);
        } else if (pro.req.kv > 0) {
          phys = load_near(a.block_table + (int64_t)pro.b * a.max_blocks + pro.blk);
          return;
        } else {                                           // one block that is none
          --pro_left;
          pro.next_item(a, kRows);
        }
      }
    };
    int put = 0;                                           // chunk that is copied next
    auto copy = [&](const int8_t* src) {
      __syncwarp();                                        // every lane has read what the chunk held
      if (lane == 0) {
        ptx::mbar_expect_tx(bars + 8 * put, kBytes);
        bulk_load(ring + put * kBytes, src, kBytes, bars + 8 * put);
      }
      put = put + 1 == kRing ? 0 : put + 1;
    };
    // copies the keys of the next block into the ring and notes its steps at place i of the queue
    auto copy_keys = [&](int i) {
      if (pro_left <= 0) { v_src = nullptr; return; }
      const bool bad = phys < 0 || phys >= a.n_blocks;
      if (bad) report_status(a.hdr, TLQ_ERR_SHAPE, 210);
      const int64_t at = (int64_t)(bad ? 0 : phys) * a.n_kv + pro.h;
      q_base[i] = bad ? 0x7FFFFFFF - kKvBlock : pro.blk * kKvBlock;
      q_k[i] = load_near(a.k_steps + at);
      q_v[i] = load_near(a.v_steps + at);
      copy(a.k_codes + at * kBytes);
      v_src = a.v_codes + at * kBytes;
      --pro_left;
      if (++pro.blk >= pro.un.blocks) pro.next_item(a, kRows);
      look_up();
    };
    auto copy_values = [&]() {
      if (v_src != nullptr) copy(v_src);
    };
    look_up();
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      copy_keys(i);
      if (i + 1 < kDeep) copy_values();                    // the last block's values follow when a chunk is free
    }
    int take = 0;                                          // chunk that is read next
    uint32_t phase = 0;
    bool ok = true;
    auto arrive = [&]() {
      ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bars + 8 * take, phase, &s_abort));
      return ring + take * kBytes;
    };
    auto taken = [&]() {
      if (++take == kRing) { take = 0; phase ^= 1u; }
    };

    while (unit < w_end && ok) {
      const bool small = con.un.blocks <= g.whole;
      if (con.blk < 0) {
        unit -= con.blk;
        con.blk = 0;
        if (unit >= w_end && !small) break;
      }
      const int blk0 = con.blk;
      const long long left = w_end - unit;
      const int blk1 = small || con.un.blocks - blk0 <= left ? con.un.blocks : blk0 + (int)left;
      const Request req = con.req;
      const int n_rows = min(kRows, req.q_len * a.group - con.tile * kRows);
      const int past = req.kv - req.q_len, row0 = con.tile * kRows;

      // ------------------------------------------------------------ query rows, as the n side of the products
      uint32_t qf[NT][D / 16][2];
      float fac[NT][2];                                    // of columns 2 tq, 2 tq + 1: scale * log2(e) * 2^(24 + exponent)
      float off[NT][2];                                    // and 128 2^-24 sum(q)
      int last[NT][2];                                     // last place that the column sees
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = n * 8 + gr;
        float x[D / 4];
        float top = 0.f;
        if (r < n_rows) {
          const int row = row0 + r;
          const uint16_t* p = g.q + (int64_t)(req.q0 + row / a.group) * g.ldq + (int64_t)(con.h * a.group + row % a.group) * D;
#pragma unroll
          for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float e[8];
              unpack8(load_near(reinterpret_cast<const uint4*>(p + 64 * c + 16 * tq + 8 * i)), e);
#pragma unroll
              for (int j = 0; j < 8; ++j) x[c * 16 + i * 8 + j] = e[j];
            }
        } else {
#pragma unroll
          for (int j = 0; j < D / 4; ++j) x[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < D / 4; ++j) top = fmaxf(top, fabsf(x[j]));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const int ex = top > 0.f && top <= 3.4e38f ? ilogbf(top) : 0;
        const float f = ldexpf(g.scale_log2, ex + 24);
        float qs = 0.f;
        // 2^-ex in two factors, either of which is a normal number
        const float d0 = ldexpf(1.0f, -(ex / 2)), d1 = ldexpf(1.0f, -(ex - ex / 2));
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          qf[n][s][0] = pack_f16(x[4 * s] * d0 * d1, x[4 * s + 1] * d0 * d1);
          qf[n][s][1] = pack_f16(x[4 * s + 2] * d0 * d1, x[4 * s + 3] * d0 * d1);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&qf[n][s][i]));
            qs += y.x + y.y;
          }
        }
        qs += __shfl_xor_sync(0xFFFFFFFFu, qs, 1);
        qs += __shfl_xor_sync(0xFFFFFFFFu, qs, 2);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          fac[n][j] = __shfl_sync(0xFFFFFFFFu, f, (2 * tq + j) * 4);
          off[n][j] = __shfl_sync(0xFFFFFFFFu, qs, (2 * tq + j) * 4) * (128.f / kUnit);
          const int c = n * 8 + 2 * tq + j;
          last[n][j] = c >= n_rows ? -1 : g.causal ? min(past + (row0 + c) / a.group, req.kv - 1) : req.kv - 1;
        }
      }
      // a block that ends at or before this place needs no mask
      const int sure = g.causal ? min(past + row0 / a.group, req.kv - 1) : req.kv - 1;

      float o[NT][D / 16][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[n][i][j] = 0.f;
      }

      const int n_blk = req.kv > 0 ? blk1 - blk0 : 0;
      for (int it = 0; it < n_blk; ++it) {
        // ---------------------------------------------------------- S^T = K q^T
        float sc[NT][4][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[n][i][j] = 0.f;
        const uint32_t ka = arrive() + (16 * (gr >> 1) + (gr & 1)) * D + 16 * tq;
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 k0 = lds128(ka + 4 * i * D + 64 * c), k1 = lds128(ka + (4 * i + 2) * D + 64 * c);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t a0, a1, a2, a3;
              keys_to_f16(word(k0, w), a0, a2);
              keys_to_f16(word(k1, w), a1, a3);
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16(sc[n][i], a0, a1, a2, a3, qf[n][4 * c + w][0], qf[n][4 * c + w][1]);
            }
          }
        taken();
        copy_values();
        const float kstep = q_k[0], vstep = q_v[0] < kStepFloor ? kStepFloor : q_v[0], vinv = 1.0f / vstep, vlog = log2f(vstep);
        const int base = q_base[0];

        // ---------------------------------------------------------- running softmax of each column
        const bool masked = base + kKvBlock - 1 > sure;
        uint32_t pf[NT][4][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float f = fac[n][j] * kstep, add = fmaf(-off[n][j], f, vlog);
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float x = fmaf(sc[n][i][2 * e + j], f, add);
                if (masked && base + 16 * (gr >> 1) + (gr & 1) + 4 * i + 2 * e > last[n][j]) x = -INFINITY;
                sc[n][i][2 * e + j] = x;
                top = fmaxf(top, x);
              }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            const float mn = fmaxf(m[n][j], top);
            const float mu = mn == -INFINITY ? 0.f : mn;
            const float corr = exp2_fast(m[n][j] - mu);
            m[n][j] = mn;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float p = exp2_fast(sc[n][i][2 * e + j] - mu + kShift);
                sc[n][i][2 * e + j] = p;
                sum += p;
              }
            l[n][j] = fmaf(l[n][j], corr, sum > 0.f ? sum * vinv : sum);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              o[n][i][j] *= corr;
              o[n][i][2 + j] *= corr;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pf[n][i][0] = transpose8(pack_f16(sc[n][i][0], sc[n][i][1]));
            pf[n][i][1] = transpose8(pack_f16(sc[n][i][2], sc[n][i][3]));
          }
        }
        // ---------------------------------------------------------- O^T += V^T P^T
        const uint32_t va = arrive() + gr * kKvBlock + 16 * tq;
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const uint4 v0 = lds128(va + 16 * i * kKvBlock), v1 = lds128(va + (16 * i + 8) * kKvBlock);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a0, a1, a2, a3;
            values_to_f16(word(v0, w), a0, a2);
            values_to_f16(word(v1, w), a1, a3);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(o[n][i], a0, a1, a2, a3, pf[n][w][0], pf[n][w][1]);
          }
        }
        taken();
#pragma unroll
        for (int i = 0; i + 1 < kDeep; ++i) {
          q_k[i] = q_k[i + 1];
          q_v[i] = q_v[i + 1];
          q_base[i] = q_base[i + 1];
        }
        copy_keys(kDeep - 1);
      }
      if (!ok) break;
      // -------------------------------------------------------------- leave the item
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xFFFFFFFFu, l[n][j], d);
      const bool whole = blk0 == 0 && blk1 == con.un.blocks;
      if (whole) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int c = n * 8 + 2 * tq + j;
            if (c >= n_rows) continue;
            const int64_t at = out_row(a, req, con.h, row0 + c);
            const bool none = m[n][j] == -INFINITY && l[n][j] == 0.f;    // a row that sees nothing (a NaN row has a NaN sum)
            const float inv = none ? 0.f : 1.0f / l[n][j];
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const __nv_bfloat16 y = __float2bfloat16_rn(none ? 0.f : o[n][i][2 * e + j] * inv);
                g.out[at * D + 16 * i + 8 * e + gr] = *reinterpret_cast<const uint16_t*>(&y);
              }
            if (gr == 0 && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(l[n][j]) + m[n][j] - kShift);
          }
      } else {
        float* to = few_partials(g.split) + (2 * worker + (blk0 == 0 ? 1 : 0)) * kPitch;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int c = n * 8 + 2 * tq + j;
            if (gr == 0) {
              to[c] = m[n][j];
              to[kRows + c] = l[n][j];
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              to[2 * kRows + c * D + 16 * i + gr] = o[n][i][j];
              to[2 * kRows + c * D + 16 * i + 8 + gr] = o[n][i][2 + j];
            }
          }
        if (lane == 0) {
          PartNote* d = notes + (blk0 == 0 ? 1 : 0);
          d->item = unit - blk0;
          d->first = blk0 == 0; d->last = blk1 == con.un.blocks;
          d->h = con.h; d->tile = con.tile; d->q0 = req.q0; d->q_len = req.q_len;
        }
      }
      unit += blk1 - blk0;
      con.blk = blk1;
      if (unit < w_end) con.next_item(a, kRows);
    }
    if (!ok && lane == 0) report_status(a.hdr, TLQ_ERR_TIMEOUT, 211);
  }
  padding();
  __syncthreads();
  if (*(volatile int*)&s_abort != 0) {                     // a copy that never came: give those under way time to land
    if (warp < active && lane < 2) notes[lane].item = -1;
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
}

template <int D, int NT>
int launch(const KvArgs& a, const AttnArgs& g, int ctas, cudaStream_t st) {
  static OncePerDevice once;
  const int rc = once_per_device(once, [] {
    return cudaFuncSetAttribute(kv_attention_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes<D>);
  });
  if (rc != TLQ_OK) return rc;
  return launch_next(kv_attention_kernel<D, NT>, dim3((unsigned)ctas), kThreads, kRingBytes<D>, 1, st, a, g);
}

}  // namespace

int launch_kv_attention(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal,
                        uint16_t* out, float* lse, const KvSplit& split, cudaStream_t st) {
  AttnArgs g{};
  g.q = q; g.ldq = ldq; g.out = out; g.lse = lse;
  g.scale_log2 = scale * kLog2e;
  g.causal = causal;
  g.split = split;
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  const int ctas = sms < kMaxWorkers ? sms : kMaxWorkers;
  const int64_t rows = (int64_t)a.group * (a.T < a.max_q_len ? a.T : a.max_q_len);     // of one request, at most
  const double most = (double)a.T * a.n_heads * ((double)a.max_blocks * kKvBlock + kRowKeys);
  g.prompts = rows >= kPromptRows && most >= (double)kPromptPairs * (rows < kFullRows ? 3 : 1);
  const int64_t tiles = a.T * a.group / kMaxRowTile;       // row tiles of all requests, about
  g.whole = (tiles > a.B ? tiles : a.B) * a.n_kv >= ctas ? kWholeBusy : kWhole;
  int rc = TLQ_OK;
  if (g.prompts) rc = launch_kv_prompt(q, ldq, head_dim, a, scale, causal, out, lse, split, ctas, st);
  if (rc != TLQ_OK) return rc;
  const bool narrow = rows <= 8;
  if (head_dim == 128) rc = narrow ? launch<128, 1>(a, g, ctas, st) : launch<128, 2>(a, g, ctas, st);
  else rc = narrow ? launch<64, 1>(a, g, ctas, st) : launch<64, 2>(a, g, ctas, st);
  if (rc != TLQ_OK) return rc;
  if (!g.prompts && a.max_blocks <= g.whole) return TLQ_OK;  // nothing was cut
  return launch_kv_join(head_dim, a, ctas, narrow ? 8 : 16, g.prompts != 0, out, lse, split, st);
}

}  // namespace tlq
