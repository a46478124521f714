// Attention of few query rows over the 8-bit cache (decoding, drafted tokens): one pass over the cache.
//
//   o = sum_j softmax_j(scale * q . k_j) v_j,   k_j = kc_j * kstep(block of j),  v_j = vc_j * vstep(block of j).
//
// The steps never touch an element of the cache: with a = scale * log2(e) * kstep and b = log2(vstep) the kernel works on
// t_j = a (q . kc_j) + b and p_j = 2^(t_j - m), so that o = sum p_j vc_j / sum p_j / vstep, where the running maximum m
// is taken over t.  8-bit codes are exact in 16-bit floats, so both products run on the matrix instruction m16n8k16 in
// f16 with 32-bit sums.  q enters as f16 after a power of two per row that brings its largest element to [1, 2) (exact
// for all but elements 2^-14 below it); p enters as f16 scaled by 2^15, which keeps 11 bits for every p_j >= 2^-29 of the
// largest.  Maximum, sums and the output sum are 32-bit.
//
// Layout.  All query heads of a kv head (and the tokens of a short draft) are the 8 or 16 columns of the products
// S^T = K q^T (m = 16 tokens) and O^T = V^T P^T (m = 16 channels): with the cache on the m side no lane is idle when there
// are only 8 rows.  Which token or channel a matrix index means is free as long as both operands agree, so every lane
// reads its operands from global memory as whole 16-byte pieces, straight into registers: no shared memory, no barrier.
// The probabilities change from result layout to operand layout by movmatrix.
//
// Split.  A unit is one block of 64 tokens of one (request, kv head, row tile).  All units form one line that is cut into
// equal parts, one per CTA, whatever the requests' lengths; a CTA's eight warps take its blocks in turn, each with its own
// running softmax, joined through shared memory at the end of an item.  An item that several CTAs share is joined by the
// one that finishes last (partials in the workspace; its counter goes back to zero), in a fixed order.
//
// Bound: the cache's bytes.  16 KB per block and kv head at 128 channels.
#include "serve.cuh"

namespace tlq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr float kShift = 15.f;            // p is kept as 2^kShift * p in 16 bits
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnArgs {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* out;
  float* lse;
  float scale_log2;          // scale * log2(e)
  int causal;
  KvSplit split;
};

__device__ __forceinline__ uint4 ld_cache(const int8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Four 8-bit codes to two pairs of f16: 1024 + (code + 128) by byte placement, minus 1152.
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t x = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
  const __half2 off = __floats2half2_rn(1152.f, 1152.f);
  const __half2 ra = __hsub2(*reinterpret_cast<const __half2*>(&a), off);
  const __half2 rb = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&ra);
  hi = *reinterpret_cast<const uint32_t*>(&rb);
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
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Steps below this have a smaller logarithm than the running maximum can carry; values that small count as zero.
constexpr float kStepFloor = 7.8886090522101181e-31f;      // 2^-100

template <int D, int NT>
struct Block {                 // one block of one kv head, in this lane's registers
  uint4 k[4][D / 64][2];       // [16 tokens][64 channels][row g or g + 8]
  uint4 v[D / 16][2];          // [16 channels][row g or g + 8]
  float kstep, vstep;
  int base;                    // place of its first token, or a place beyond every mask
};

template <int D, int NT>
__device__ __forceinline__ void load_k(Block<D, NT>& s, const KvArgs& a, int phys, int h, int blk, int g, int t) {
  const bool bad = phys < 0 || phys >= a.n_blocks;
  if (bad) {
    report_status(a.hdr, TLQ_ERR_SHAPE, 210);
    phys = 0;
  }
  const int64_t at = (int64_t)phys * a.n_kv + h;
  s.base = bad ? 0x7FFFFFFF - kKvBlock : blk * kKvBlock;
  s.kstep = __ldg(a.k_steps + at);
  s.vstep = __ldg(a.v_steps + at);
  const int8_t* p = a.k_codes + at * (kKvBlock * D) + (16 * (g >> 1) + (g & 1)) * D + 16 * t;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      s.k[i][c][0] = ld_cache(p + 4 * i * D + 64 * c);
      s.k[i][c][1] = ld_cache(p + (4 * i + 2) * D + 64 * c);
    }
}
template <int D, int NT>
__device__ __forceinline__ void load_v(Block<D, NT>& s, const KvArgs& a, int phys, int h, int g, int t) {
  if (phys < 0 || phys >= a.n_blocks) phys = 0;
  const int8_t* p = a.v_codes + ((int64_t)phys * a.n_kv + h) * (kKvBlock * D) + g * kKvBlock + 16 * t;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    s.v[i][0] = ld_cache(p + 16 * i * kKvBlock);
    s.v[i][1] = ld_cache(p + (16 * i + 8) * kKvBlock);
  }
}

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Units of a request: row tiles x kv heads x blocks (one for a request without cached tokens, whose rows are empty).
struct Units {
  int row_tiles, blocks;
  long long total;
};
__device__ __forceinline__ Units units_of(const KvArgs& a, const Request& r, int row_tile) {
  Units u;
  u.row_tiles = (int)(((long long)r.q_len * a.group + row_tile - 1) / row_tile);
  u.blocks = r.kv > 0 ? (r.kv + kKvBlock - 1) / kKvBlock : 1;
  u.total = (long long)u.row_tiles * a.n_kv * u.blocks;
  return u;
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 1)
kv_attention_kernel(const KvArgs a, const AttnArgs g) {
  constexpr int kRows = 8 * NT;
  extern __shared__ float smem[];
  float* s_o = smem;                               // [kWarps][kRows][D + 1]
  float* s_m = s_o + kWarps * kRows * (D + 1);     // [kWarps][kRows]
  float* s_l = s_m + kWarps * kRows;
  __shared__ long long sums[kWarps];
  __shared__ Found found;
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gr = lane >> 2, tq = lane & 3;

  // ---------------------------------------------------------------- this CTA's part of the line of units
  long long total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + (int)threadIdx.x;
    const long long n = b < a.B ? units_of(a, load_request(a, b), kRows).total : 0;
    long long part;
    block_scan<kThreads>(n, sums, part);
    total += part;
  }
  if (total == 0) return;
  // no more CTAs than give each warp of a CTA a block
  long long workers = (total + kWarps - 1) / kWarps;
  if (workers > (long long)gridDim.x) workers = gridDim.x;
  if ((long long)blockIdx.x >= workers) return;
  const long long u_begin = total * blockIdx.x / workers, u_end = total * (blockIdx.x + 1) / workers;
  auto worker_of = [&](long long unit) { return ((unit + 1) * workers - 1) / total; };
  if (!locate_item<kThreads>(a.B, u_begin, [&](int b) { return units_of(a, load_request(a, b), kRows).total; }, sums,
                             &found))
    return;
  int b = found.request;
  Request req = load_request(a, b);
  Units un = units_of(a, req, kRows);
  long long unit = u_begin;
  long long rest = found.rest;                     // units of request b before `unit`

  while (unit < u_end) {
    if (rest >= un.total) {                        // next request with any work
      rest -= un.total;
      do {
        if (++b >= a.B) return;
        req = load_request(a, b);
        un = units_of(a, req, kRows);
      } while (un.total == 0);
      continue;
    }
    const int item = (int)(rest / un.blocks), blk0 = (int)(rest % un.blocks);
    const int h = item / un.row_tiles, tile = item % un.row_tiles;
    const long long item_begin = unit - blk0, item_end = item_begin + un.blocks;
    const int blk1 = item_end <= u_end ? un.blocks : blk0 + (int)(u_end - unit);
    const int n_rows = min(kRows, req.q_len * a.group - tile * kRows);
    const int past = req.kv - req.q_len;

    // -------------------------------------------------------------- query rows, as the n side of the products
    uint32_t qf[NT][D / 16][2];
    float fac[NT][2];                              // of columns 2 tq, 2 tq + 1: scale * log2(e) * 2^exponent
    int last[NT][2];                               // last place that the column sees
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = n * 8 + gr;
      float f = 0.f;
      float x[D / 4];
      float top = 0.f;
      const bool live = r < n_rows;
      const int row = tile * kRows + r;
      if (live) {
        const uint16_t* p = g.q + (int64_t)(req.q0 + row / a.group) * g.ldq + (int64_t)(h * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float e[8];
            unpack8(*reinterpret_cast<const uint4*>(p + 64 * c + 16 * tq + 8 * i), e);
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
      f = ldexpf(g.scale_log2, ex);
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        qf[n][s][0] = pack_f16(ldexpf(x[4 * s], -ex), ldexpf(x[4 * s + 1], -ex));
        qf[n][s][1] = pack_f16(ldexpf(x[4 * s + 2], -ex), ldexpf(x[4 * s + 3], -ex));
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        fac[n][j] = __shfl_sync(0xFFFFFFFFu, f, (2 * tq + j) * 4);
        const int c = n * 8 + 2 * tq + j;
        last[n][j] = c >= n_rows ? -1 : g.causal ? min(past + (tile * kRows + c) / a.group, req.kv - 1) : req.kv - 1;
      }
    }
    // a block that ends at or before this place needs no mask
    const int row0 = tile * kRows;
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

    const int32_t* table = a.block_table + (int64_t)b * a.max_blocks;
    const int stop = req.kv > 0 ? blk1 : 0;
    int blk = blk0 + warp;
    if (blk < stop) {
      Block<D, NT> s;
      int phys = __ldg(table + blk);
      load_k(s, a, phys, h, blk, gr, tq);
      load_v(s, a, phys, h, gr, tq);
      int phys_next = blk + kWarps < stop ? __ldg(table + blk + kWarps) : 0;
      while (true) {
        // ---------------------------------------------------------- S^T = K q^T
        float sc[NT][4][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[n][i][j] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              codes_to_f16(word(s.k[i][c][0], w), a0, a2);
              codes_to_f16(word(s.k[i][c][1], w), a1, a3);
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16(sc[n][i], a0, a1, a2, a3, qf[n][4 * c + w][0], qf[n][4 * c + w][1]);
            }
        const float kstep = s.kstep, vstep = s.vstep < kStepFloor ? kStepFloor : s.vstep, vinv = 1.0f / vstep, vlog = log2f(vstep);
        const int base = s.base, next = blk + kWarps;
        const bool more = next < stop;
        if (more) load_k(s, a, phys_next, h, next, gr, tq);

        // ---------------------------------------------------------- running softmax of each column
        const bool masked = base + kKvBlock - 1 > sure;
        uint32_t pf[NT][4][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float f = fac[n][j] * kstep;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float x = fmaf(sc[n][i][2 * e + j], f, vlog);
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
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a0, a1, a2, a3;
            codes_to_f16(word(s.v[i][0], w), a0, a2);
            codes_to_f16(word(s.v[i][1], w), a1, a3);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(o[n][i], a0, a1, a2, a3, pf[n][w][0], pf[n][w][1]);
          }
        if (!more) break;
        load_v(s, a, phys_next, h, gr, tq);
        blk = next;
        phys_next = blk + kWarps < stop ? __ldg(table + blk + kWarps) : 0;
      }
    }
    // ---------------------------------------------------------------- join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xFFFFFFFFu, l[n][j], d);
    __syncthreads();                               // the previous item's readers are done
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = n * 8 + 2 * tq + j;
        if (gr == 0) {
          s_m[warp * kRows + c] = m[n][j];
          s_l[warp * kRows + c] = l[n][j];
        }
        float* to = s_o + (warp * kRows + c) * (D + 1);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          to[16 * i + gr] = o[n][i][j];
          to[16 * i + 8 + gr] = o[n][i][2 + j];
        }
      }
    __syncthreads();
    const bool whole = item_begin >= u_begin && item_end <= u_end;
    const int slot = blockIdx.x * 2 + (item_begin >= u_begin ? 1 : 0);
    float* part = g.split.partials + (size_t)slot * kRows * (D + 2);
    for (int e = threadIdx.x; e < kRows * D; e += kThreads) {
      const int c = e / D, d = e % D;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, s_m[w * kRows + c]);
      const float mu = mm == -INFINITY ? 0.f : mm;
      float sum = 0.f, den = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(s_m[w * kRows + c] - mu);
        sum = fmaf(s_o[(w * kRows + c) * (D + 1) + d], f, sum);
        den = fmaf(s_l[w * kRows + c], f, den);
      }
      if (whole) {
        if (c < n_rows) {
          const int row = tile * kRows + c;
          const int64_t at = (int64_t)(req.q0 + row / a.group) * a.n_heads + h * a.group + row % a.group;
          const bool none = mm == -INFINITY && den == 0.f;       // a row that sees nothing (a NaN row has den = NaN)
          const __nv_bfloat16 y = __float2bfloat16_rn(none ? 0.f : sum / den);
          g.out[at * D + d] = *reinterpret_cast<const uint16_t*>(&y);
          if (d == 0 && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(den) + mm - kShift);
        }
      } else {
        part[2 * kRows + e] = sum;
        if (d == 0) {
          part[c] = mm;
          part[kRows + c] = den;
        }
      }
    }
    if (!whole) {
      // ---------------------------------------------------------------- join the CTAs that share the item
      const long long first = worker_of(item_begin), final = worker_of(item_end - 1);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) s_last = atomicAdd(g.split.counters + first, 1) == (int)(final - first);
      __syncthreads();
      if (s_last) {
        __threadfence();
        if (threadIdx.x == 0) g.split.counters[first] = 0;
        const float* base = g.split.partials;
        const size_t pitch = (size_t)kRows * (D + 2);
        for (int e = threadIdx.x; e < kRows * D; e += kThreads) {
          const int c = e / D, d = e % D;
          if (c >= n_rows) break;
          float mm = -INFINITY, sum = 0.f, den = 0.f;
          for (long long w = first; w <= final; ++w) {
            const float* p = base + (size_t)(2 * w + (w == first ? 1 : 0)) * pitch;
            mm = fmaxf(mm, __ldcg(p + c));
          }
          const float mu = mm == -INFINITY ? 0.f : mm;
#pragma unroll 4
          for (long long w = first; w <= final; ++w) {
            const float* p = base + (size_t)(2 * w + (w == first ? 1 : 0)) * pitch;
            const float f = exp2_fast(__ldcg(p + c) - mu);
            sum = fmaf(__ldcg(p + 2 * kRows + e), f, sum);
            den = fmaf(__ldcg(p + kRows + c), f, den);
          }
          const int row = tile * kRows + c;
          const int64_t at = (int64_t)(req.q0 + row / a.group) * a.n_heads + h * a.group + row % a.group;
          const bool none = mm == -INFINITY && den == 0.f;
          const __nv_bfloat16 y = __float2bfloat16_rn(none ? 0.f : sum / den);
          g.out[at * D + d] = *reinterpret_cast<const uint16_t*>(&y);
          if (d == 0 && g.lse != nullptr) g.lse[at] = none ? -INFINITY : kLn2 * (log2f(den) + mm - kShift);
        }
      }
    }
    unit += blk1 - blk0;
    rest += blk1 - blk0;
  }
}

template <int D, int NT>
int launch(const KvArgs& a, const AttnArgs& g, cudaStream_t st) {
  constexpr size_t smem = (size_t)kWarps * 8 * NT * (D + 3) * sizeof(float);
  static OncePerDevice once;
  const int rc = once_per_device(once, [] {
    return cudaFuncSetAttribute(kv_attention_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  });
  if (rc != TLQ_OK) return rc;
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  const int grid = sms < kMaxWorkers ? sms : kMaxWorkers;
  kv_attention_kernel<D, NT><<<grid, kThreads, smem, st>>>(a, g);
  return after_launch();
}

}  // namespace

int launch_kv_attention(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal,
                        uint16_t* out, float* lse, const KvSplit& split, cudaStream_t st) {
  AttnArgs g{};
  g.q = q; g.ldq = ldq; g.out = out; g.lse = lse;
  g.scale_log2 = scale * kLog2e;
  g.causal = causal;
  g.split = split;
  const bool narrow = (int64_t)a.group * a.max_q_len <= 8;
  if (head_dim == 128) return narrow ? launch<128, 1>(a, g, st) : launch<128, 2>(a, g, st);
  return narrow ? launch<64, 1>(a, g, st) : launch<64, 2>(a, g, st);
}

}  // namespace tlq
