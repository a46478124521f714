// Joins the parts of attention items that several workers share (kv_attention.cu: warps, kv_prompt.cu: CTAs).
//
// A worker walks its part of a line of items and leaves, of an item that is not all its own, the maximum m, the sum l and the
// output sums o of every row, and a note that says of which item they are; an item's parts are those of consecutive workers.
// With M = max m_i the row is sum o_i 2^(m_i - M) / sum l_i 2^(m_i - M), in the order of the workers whatever finished first.
//
// A kernel of its own.  When the last arriver of an item joined it inside the kernels above, 15 to 20 us went by between the
// last block and the end: two levels (warps, CTAs) of dependent reads, in code that runs once and costs its fetch, while other
// SMs keep the memory's queues full, and one SM reading all parts of an item.  Bound: latency, three dependent reads for up to
// 32 parts (1 us each), one more for every 32.  Measured: 32 requests x 2048 keys 31 -> 28 us in all, 9 tokens x 4096 keys
// 26 -> 20, prompts of 64 tokens over 16384 180 -> 62.
//
// Grid: x names the workers whose notes a CTA looks at, y the rows of their items (one row, or 32 of a prompt), so that a single
// item cut into many parts is still read by many SMs.
#include "serve.cuh"

namespace tlq {
namespace {

constexpr int kThreads = 256;

struct JoinArgs {
  uint16_t* out;
  float* lse;
  KvSplit split;
};

__device__ __forceinline__ PartNote load_note(const PartNote* p) {
  union { int4 v[2]; PartNote n; } u;
  u.v[0] = load_far(reinterpret_cast<const int4*>(p));
  u.v[1] = load_far(reinterpret_cast<const int4*>(p) + 1);
  return u.n;
}
// which item a part is of, and whether it is the last of it
struct PartOf {
  long long item;
  int first, last;
};
__device__ __forceinline__ PartOf load_part_of(const PartNote* p) {
  union { int4 v; PartOf n; } u;
  u.v = load_far(reinterpret_cast<const int4*>(p));
  return u.n;
}

struct RowShared {                        // of a row of a few-row item, from every warp
  PartNote notes[2 * kSplitWarps];
  float4 sums[kThreads];
  float m[kThreads / 16], l[kThreads / 16];
};
struct TileShared {                       // of kPromptJoinRows rows of a prompt's item
  float f[kMaxWorkers * kPromptJoinRows]; // [part][row]: maximum, then the factor of its sums
  float inv[kPromptJoinRows];
  int parts[kMaxWorkers];                 // numbers of the partials
  float over_warps[2][kThreads / 32][kPromptJoinRows];
  int counts[kThreads / 32];
};

// Rows row0 .. row1 - 1, one after another, of the items whose first blocks workers 8 blockIdx.x .. 8 blockIdx.x + 7 had.  Every
// group of D / 4 threads takes every kGroups-th part; notes, maxima, sums and outputs of kAtOnce parts of a group are asked for
// together, whether or not they will turn out to be the item's: one trip to memory for an item of up to kGroups * kAtOnce parts.
template <int D, int kItem>
__device__ __forceinline__ void join_rows(const KvArgs& a, const JoinArgs& g, const float* partials, const PartNote* notes, int row0,
                                          int row1, int workers, float shift, RowShared& s) {
  constexpr size_t kPitch = (size_t)kItem * (D + 2);
  constexpr int kWide = D / 4, kGroups = kThreads / kWide, kAtOnce = 4;
  const int t = threadIdx.x, group = t / kWide, piece = t % kWide;
  PartNote mine;
  mine.item = -1;
  if (t < 2 * kSplitWarps) {
    if ((int)blockIdx.x * kSplitWarps + t / 2 < workers) mine = load_note(notes + (size_t)blockIdx.x * 2 * kSplitWarps + t);
    s.notes[t] = mine;
  }
  if (!__syncthreads_or(mine.item >= 0 && mine.first)) return;
  for (int i = 0; i < 2 * kSplitWarps * (row1 - row0); ++i) {
    const int at = i % (2 * kSplitWarps), r = row0 + i / (2 * kSplitWarps);
    const PartNote it = s.notes[at];
    if (it.item < 0 || !it.first || (long long)it.q_len * a.group - (long long)it.tile * kItem <= r) continue;
    const int w = (int)blockIdx.x * kSplitWarps + at / 2;
    float m = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j0 = 0;; j0 += kGroups * kAtOnce) {
      PartOf p[kAtOnce];
      float pm[kAtOnce], pl[kAtOnce];
      float4 v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int j = j0 + i * kGroups + group, k = j == 0 ? 2 * w + (at & 1) : 2 * min(w + j, workers - 1);
        const float* from = partials + (size_t)k * kPitch;
        p[i] = load_part_of(notes + k);
        pm[i] = load_far(from + r);
        pl[i] = load_far(from + kItem + r);
        v[i] = load_far(reinterpret_cast<const float4*>(from + 2 * kItem + r * D) + piece);
        if (w + j >= workers) p[i].item = -1;
      }
      bool end = w + j0 + kGroups * kAtOnce >= workers;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const bool same = p[i].item == it.item;
        end |= p[i].item >= 0 && (!same || p[i].last);
        if (!same) continue;
        const float mn = fmaxf(m, pm[i]), mu = mn == -INFINITY ? 0.f : mn;
        const float old = exp2_fast(m - mu), f = exp2_fast(pm[i] - mu);
        m = mn;
        l = l * old + pl[i] * f;
        sum.x = sum.x * old + v[i].x * f; sum.y = sum.y * old + v[i].y * f;
        sum.z = sum.z * old + v[i].z * f; sum.w = sum.w * old + v[i].w * f;
      }
      if (__syncthreads_or(end)) break;                    // (and the places below are free)
    }
    s.sums[t] = sum;
    if (piece == 0) {
      s.m[group] = m;
      s.l[group] = l;
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int i = 1; i < kGroups; ++i) m = fmaxf(m, s.m[i]);
      const float mu = m == -INFINITY ? 0.f : m;
      l = 0.f;
      sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const float f = exp2_fast(s.m[i] - mu);
        const float4 x = s.sums[i * kWide + piece];
        l = fmaf(s.l[i], f, l);
        sum.x = fmaf(x.x, f, sum.x); sum.y = fmaf(x.y, f, sum.y); sum.z = fmaf(x.z, f, sum.z); sum.w = fmaf(x.w, f, sum.w);
      }
      const bool none = m == -INFINITY && l == 0.f;        // a row that sees nothing (a NaN row has a NaN sum)
      const float inv = none ? 0.f : 1.0f / l;
      const int row = it.tile * kItem + r;
      const int64_t to = (int64_t)(it.q0 + row / a.group) * a.n_heads + it.h * a.group + row % a.group;
      const __nv_bfloat162 y0 = __floats2bfloat162_rn(sum.x * inv, sum.y * inv), y1 = __floats2bfloat162_rn(sum.z * inv, sum.w * inv);
      reinterpret_cast<uint2*>(g.out + to * D)[piece] =
          make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
      if (piece == 0 && g.lse != nullptr) g.lse[to] = none ? -INFINITY : kLn2 * (log2f(l) + m - shift);
    }
    // (the next item's loads end in a barrier before the shared memory is written again)
  }
}

// kPromptJoinRows rows of the items whose first blocks CTA blockIdx.x of the prompt kernel had.
template <int D>
__device__ __forceinline__ void join_tile(const KvArgs& a, const JoinArgs& g, const float* partials, const PartNote* notes, int row0,
                                          float shift, TileShared& s) {
  constexpr int kItem = kPromptItemRows, kRows = kPromptJoinRows;
  static_assert(kRows == 32, "a lane for each row");
  constexpr size_t kPitch = (size_t)kItem * (D + 2);
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, workers = (int)gridDim.x;
  // over the rows' parts, all threads alike: `r` is a thread's row where it handles (part, row) pairs
  const int r = t % kRows;
  auto over_rows = [&](float v, bool is_max, int which) {
    s.over_warps[which][warp][lane] = v;                   // a lane for each row
    __syncthreads();
    v = s.over_warps[which][0][r];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) v = is_max ? fmaxf(v, s.over_warps[which][i][r]) : v + s.over_warps[which][i][r];
    return v;
  };
  for (int at = 0; at < 2; ++at) {
    const PartNote it = load_note(notes + 2 * blockIdx.x + at);
    if (it.item < 0 || !it.first) continue;
    const int live = (int)min((long long)kRows, (long long)it.q_len * a.group - (long long)it.tile * kItem - row0);
    if (live <= 0) continue;
    // the other parts, in order
    int n = 1;
    if (t == 0) s.parts[0] = 2 * (int)blockIdx.x + at;
    for (int w0 = (int)blockIdx.x + 1; w0 < workers; w0 += kThreads) {
      PartOf p{-1, 0, 0};
      if (w0 + t < workers) p = load_part_of(notes + 2 * (size_t)(w0 + t));
      const bool same = p.item == it.item;
      const uint32_t some = __ballot_sync(0xFFFFFFFFu, same);
      if (lane == 0) s.counts[warp] = __popc(some);
      const bool end = __syncthreads_or(p.item >= 0 && (!same || p.last));
      int before = n + __popc(some & ((1u << lane) - 1u));
#pragma unroll
      for (int i = 0; i < kThreads / 32; ++i) {
        if (i < warp) before += s.counts[i];
        n += s.counts[i];
      }
      if (same) s.parts[before] = 2 * (w0 + t);
      __syncthreads();
      if (end) break;
    }
    // factors of the parts
    float m = -INFINITY;
    for (int j = t / kRows; j < n; j += kThreads / kRows) {
      const float x = load_far(partials + (size_t)s.parts[j] * kPitch + row0 + r);
      s.f[j * kRows + r] = x;
      m = fmaxf(m, x);
    }
    m = over_rows(m, true, 0);
    const float mu = m == -INFINITY ? 0.f : m;
    float den = 0.f;
    for (int j = t / kRows; j < n; j += kThreads / kRows) {
      const float f = exp2_fast(s.f[j * kRows + r] - mu);
      s.f[j * kRows + r] = f;
      den = fmaf(f, load_far(partials + (size_t)s.parts[j] * kPitch + kItem + row0 + r), den);
    }
    den = over_rows(den, false, 1);                        // (and all factors are written)
    const bool none = m == -INFINITY && den == 0.f;        // a row that sees nothing (a NaN row has a NaN sum)
    if (t < live) {
      const int row = it.tile * kItem + row0 + t;
      if (g.lse != nullptr)
        g.lse[(int64_t)(it.q0 + row / a.group) * a.n_heads + it.h * a.group + row % a.group] =
            none ? -INFINITY : kLn2 * (log2f(den) + m - shift);
      s.inv[t] = none ? 0.f : 1.0f / den;
    }
    // sums of the outputs, in pieces of four channels
    constexpr int kEach = kRows * (D / 4) / kThreads;
    static_assert(kEach >= 1, "");
    float4 sum[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) sum[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int j = 0; j < n; ++j) {
      const float4* from = reinterpret_cast<const float4*>(partials + (size_t)s.parts[j] * kPitch + 2 * kItem + (size_t)row0 * D) + t;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float4 v = load_far(from + e * kThreads);
        const float f = s.f[j * kRows + (e * kThreads + t) / (D / 4)];
        sum[e].x = fmaf(v.x, f, sum[e].x); sum[e].y = fmaf(v.y, f, sum[e].y);
        sum[e].z = fmaf(v.z, f, sum[e].z); sum[e].w = fmaf(v.w, f, sum[e].w);
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = e * kThreads + t, c = i / (D / 4), d = (i % (D / 4)) * 4;
      if (c >= live) continue;
      const int row = it.tile * kItem + row0 + c;
      const int64_t to = (int64_t)(it.q0 + row / a.group) * a.n_heads + it.h * a.group + row % a.group;
      const float inv = s.inv[c];
      const __nv_bfloat162 y0 = __floats2bfloat162_rn(inv == 0.f ? 0.f : sum[e].x * inv, inv == 0.f ? 0.f : sum[e].y * inv);
      const __nv_bfloat162 y1 = __floats2bfloat162_rn(inv == 0.f ? 0.f : sum[e].z * inv, inv == 0.f ? 0.f : sum[e].w * inv);
      *reinterpret_cast<uint2*>(g.out + to * D + d) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
    }
    __syncthreads();                                       // before the next item takes the places of this one
  }
}

// y: groups of rows of the prompt kernel's items, then the rows of the few-row kernel's, kRowsEach to a CTA: where the prompt
// kernel has run too there are enough CTAs without one for each row, and little for them to do.
template <int D, int kFewRows, bool kPrompts>
__global__ void __launch_bounds__(kThreads)
kv_join_kernel(const KvArgs a, const JoinArgs g) {
  __shared__ union Places { RowShared row; TileShared tile; __device__ Places() {} } s;
  after_previous();
  constexpr int kRowsEach = kPrompts ? 4 : 1;
  const int y = (int)blockIdx.y - (kPrompts ? kPromptItemRows / kPromptJoinRows : 0);
  if (y >= 0)
    join_rows<D, kFewRows>(a, g, few_partials(g.split), few_notes(g.split, D), y * kRowsEach, (y + 1) * kRowsEach,
                           load_far(few_workers(g.split, D)), kFewShift, s.row);
  else if constexpr (kPrompts)
    join_tile<D>(a, g, prompt_partials(g.split, D), prompt_notes(g.split, D), (int)blockIdx.y * kPromptJoinRows, kPromptShift, s.tile);
}

template <int D>
int launch(const KvArgs& a, const JoinArgs& g, int ctas, int few_rows, bool prompts, cudaStream_t st) {
  const dim3 grid((unsigned)ctas, (unsigned)(prompts ? kPromptItemRows / kPromptJoinRows + few_rows / 4 : few_rows));
  if (few_rows == 8) return launch_next(kv_join_kernel<D, 8, false>, grid, kThreads, 0, 1, st, a, g);
  return prompts ? launch_next(kv_join_kernel<D, 16, true>, grid, kThreads, 0, 1, st, a, g)
                 : launch_next(kv_join_kernel<D, 16, false>, grid, kThreads, 0, 1, st, a, g);
}

}  // namespace

int launch_kv_join(int head_dim, const KvArgs& a, int ctas, int few_rows, bool prompts, uint16_t* out, float* lse,
                   const KvSplit& split, cudaStream_t st) {
  JoinArgs g{};
  g.out = out; g.lse = lse;
  g.split = split;
  return head_dim == 128 ? launch<128>(a, g, ctas, few_rows, prompts, st) : launch<64>(a, g, ctas, few_rows, prompts, st);
}

}  // namespace tlq
