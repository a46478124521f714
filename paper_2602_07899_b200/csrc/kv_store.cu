// Norms of queries and keys, position rotation and the write of keys and values into the 8-bit cache, in one pass over
// the rows of the fused projection.
//
// Per head h of a token with place p:  y = x * rsqrt(mean_c x_c^2 + eps) * w  (queries and keys, when w is given),
// (y_i, y_{i+D/2}) <- (y_i cos - y_{i+D/2} sin, y_{i+D/2} cos + y_i sin) with the angle of pair i, queries rounded to
// bf16 once.  Keys and values are quantized as the layer's activations are (paper Sec. 2.2, symmetric, n = 8), with one
// step for the 64 tokens of a cache block and one head: step = max|.| / 127.  A block that already holds tokens of its
// request keeps the larger of its old step and the new tokens' one; when it grows, the older codes follow it,
// c <- rint(c * old / new).
//
// All statistics and products are in 32 bits; codes are those of the IEEE division (by a reciprocal, and by the
// division itself where the quotient comes near a tie), so that codes of values, which see no norm, are the definition's.
//
// Bound: bytes.  The rows are read once and everything is kept in registers between the maximum and the codes.  One CTA
// owns a cache block of one head (its tokens lie in one request), because its step needs all of them; the remaining CTAs
// stream query rows, two per thread group at once.  Values lie channel by token in the cache (what a matrix instruction over
// tokens reads), so a CTA turns its 64 x D bytes in shared memory and writes rows of 64 bytes.  Measured: 16384 tokens, 64 + 8 + 8
// heads of 128 channels with norms (713 MB) 151 us, 4.7 TB/s, the schedulers busy 60 % of the time with conversions and rotations;
// 6 ragged prompts (29 MB) 12.4 us; 32 requests of one token 5.4 us, latency.
#include "serve.cuh"

namespace tlq {
namespace {

constexpr int kStoreThreads = 256;

struct StoreArgs {
  const uint16_t* qkv;
  int64_t ld;
  RopeArgs rope;
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  float eps;
  uint16_t* q_out;
  uint16_t* k_values;
  uint16_t* v_values;
  unsigned kv_ctas, period;   // CTA number i * period, i < kv_ctas, is one of the cache part; the others stream query rows
  unsigned q_ctas;            // how many do
};

// Channels of one lane: [4 l, 4 l + 4) and the same of the upper half, so that both members of its four rotation pairs
// are its own.  A row takes D / 8 lanes.
template <int D>
struct Row {
  float lo[4], hi[4];
};

// The same channels as they lie in memory.
struct Raw {
  uint2 lo, hi;
};
template <int D>
__device__ __forceinline__ Raw load_raw(const uint16_t* p, int l) {
  Raw r;
  r.lo = load_near(reinterpret_cast<const uint2*>(p + 4 * l));
  r.hi = load_near(reinterpret_cast<const uint2*>(p + D / 2 + 4 * l));
  return r;
}
template <int D>
__device__ __forceinline__ Row<D> floats(const Raw& w) {
  Row<D> r;
  r.lo[0] = __uint_as_float(w.lo.x << 16); r.lo[1] = __uint_as_float(w.lo.x & 0xFFFF0000u);
  r.lo[2] = __uint_as_float(w.lo.y << 16); r.lo[3] = __uint_as_float(w.lo.y & 0xFFFF0000u);
  r.hi[0] = __uint_as_float(w.hi.x << 16); r.hi[1] = __uint_as_float(w.hi.x & 0xFFFF0000u);
  r.hi[2] = __uint_as_float(w.hi.y << 16); r.hi[3] = __uint_as_float(w.hi.y & 0xFFFF0000u);
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int D>
__device__ __forceinline__ void store_row(uint16_t* p, const float (&lo)[4], const float (&hi)[4], int l) {
  *reinterpret_cast<uint2*>(p + 4 * l) = make_uint2(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]));
  *reinterpret_cast<uint2*>(p + D / 2 + 4 * l) = make_uint2(pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
}

template <int D>
__device__ __forceinline__ void norm_row(Row<D>& r, const Row<D>& w, float eps) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) s = fmaf(r.lo[j], r.lo[j], fmaf(r.hi[j], r.hi[j], s));
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  const float k = rsqrtf(s * (1.0f / D) + eps);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    r.lo[j] = r.lo[j] * k * w.lo[j];
    r.hi[j] = r.hi[j] * k * w.hi[j];
  }
}

// Row of the angle table for a token and each position axis.  A position outside of the table is noted in `bad` (the caller
// reports it) and row 0 read in its place; without a branch, so that the loads of several tokens can be under way at once.
struct Places {
  int at[3];
};
__device__ __forceinline__ Places load_places(const RopeArgs& rope, int64_t T, int64_t token, bool& bad) {
  Places p;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int pos = i < rope.n_axes ? load_near(rope.positions + i * T + token) : 0;
    const bool in = pos >= 0 && (int64_t)pos < rope.n_positions;
    bad = bad || !in;
    p.at[i] = in ? pos : 0;
  }
  return p;
}
// Cosines and sines of the four pairs from 4 l on.
struct Angles {
  float c[4], s[4];
};
template <int D>
__device__ __forceinline__ Angles load_angles(const RopeArgs& rope, const Places& p, int l) {
  Angles g;
  const int first = 4 * l;
  const int axis = (first >= rope.pairs_end[0] ? 1 : 0) + (first >= rope.pairs_end[1] ? 1 : 0);
  const int last = (first + 3 >= rope.pairs_end[0] ? 1 : 0) + (first + 3 >= rope.pairs_end[1] ? 1 : 0);
  if (rope.n_axes == 1 || axis == last) {              // one axis for all four
    const int at = rope.n_axes == 1 || axis == 0 ? p.at[0] : axis == 1 ? p.at[1] : p.at[2];
    const float* row = rope.cos_sin + (int64_t)at * D + first;
    const float4 c = load_near(reinterpret_cast<const float4*>(row)), s = load_near(reinterpret_cast<const float4*>(row + D / 2));
    g.c[0] = c.x; g.c[1] = c.y; g.c[2] = c.z; g.c[3] = c.w;
    g.s[0] = s.x; g.s[1] = s.y; g.s[2] = s.z; g.s[3] = s.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = (first + j >= rope.pairs_end[0] ? 1 : 0) + (first + j >= rope.pairs_end[1] ? 1 : 0);
      const float* row = rope.cos_sin + (int64_t)(i == 0 ? p.at[0] : i == 1 ? p.at[1] : p.at[2]) * D + first + j;
      g.c[j] = load_near(row);
      g.s[j] = load_near(row + D / 2);
    }
  }
  return g;
}
template <int D>
__device__ __forceinline__ void rotate_row(Row<D>& r, const Angles& g) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = r.lo[j], b = r.hi[j];
    r.lo[j] = a * g.c[j] - b * g.s[j];
    r.hi[j] = b * g.c[j] + a * g.s[j];
  }
}

__device__ __forceinline__ float finite_size(float x) {
  const float m = fabsf(x);
  return m <= 3.402823466e38f ? m : 0.f;
}

// rint(x / step) in [-127, 127], of the IEEE quotient; a NaN becomes 0.  inv is the rounded 1 / step: x * inv is within
// 127 * 2^-22 of the quotient, so only a product that close to a tie needs the division itself.
__device__ __forceinline__ int to_code(float x, float step, float inv) {
  float q = x * inv, r = rintf(q);
  if (fabsf(q - r) > 0.5f - 6e-5f) r = rintf(__fdiv_rn(x, step));
  return (int)fminf(fmaxf(r, -127.f), 127.f) * (q == q ? 1 : 0);
}

constexpr int kQueryWaves = 24;                      // CTAs per SM of those that stream queries
// Values of tokens that have no codes.  Not inlined, and with arguments by value: the loops of the kernel have no registers to spare.
// Those of one head, tokens [from, from + count):
template <int D>
__device__ __noinline__ void no_values(uint16_t* k, uint16_t* v, int n_kv, int h, int64_t from, int count) {
  for (int i = threadIdx.x; i < count * (D / 8); i += kStoreThreads) {
    const int64_t at = ((from + i / (D / 8)) * n_kv + h) * (D / 8) + i % (D / 8);
    if (k != nullptr) reinterpret_cast<uint4*>(k)[at] = make_uint4(0, 0, 0, 0);
    if (v != nullptr) reinterpret_cast<uint4*>(v)[at] = make_uint4(0, 0, 0, 0);
  }
}
// Those of the rows of no request, by CTAs of their own where values are asked for.  (A look at the padding by those that stream queries,
// ahead of their rows or behind them, costs the 16384-token prompt 2 to 5 us of 150.)
constexpr unsigned kPadCtas = 4;
template <int D>
__device__ __noinline__ void no_rows(const int32_t* cu_q, int B, int64_t T, uint16_t* k, uint16_t* v, int n_kv) {
  const Padding pad = load_padding(cu_q, B, T);
  const int64_t t = (int64_t)(gridDim.x - 1 - blockIdx.x) * kStoreThreads + threadIdx.x, n = (int64_t)kPadCtas * kStoreThreads;
  for (uint16_t* p : {k, v})
    if (p != nullptr) {
      zero_rows(p, 0, pad.before, (int64_t)n_kv * D / 8, t, n);
      zero_rows(p, pad.after, T, (int64_t)n_kv * D / 8, t, n);
    }
}

constexpr int kSweepsQ = 2;                          // sweeps of a CTA over query rows whose loads are under way at once
constexpr int kPitch = kKvBlock + 4;                 // bytes of a channel in `turned`: neighbouring channels in other banks

template <int D>
__global__ void __launch_bounds__(kStoreThreads, 3)
kv_store_kernel(const KvArgs a, const StoreArgs g) {
  constexpr int kLanes = D / 8;                      // lanes of a row
  constexpr int kRows = kStoreThreads / kLanes;      // rows of one sweep
  constexpr int kSweeps = kKvBlock / kRows;
  const int l = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
  const bool turn = g.rope.positions != nullptr;
  after_previous();
  if (blockIdx.x >= g.kv_ctas + g.q_ctas) {          // padding
    no_rows<D>(a.cu_q, a.B, a.T, g.k_values, g.v_values, a.n_kv);
    return;
  }

  // The two kinds are mixed: those of the cache part spend their time in a chain of dependent steps, those of the queries
  // wait for memory.
  const unsigned turn_of = blockIdx.x / g.period;
  if (turn_of >= g.kv_ctas || blockIdx.x - turn_of * g.period != 0) {
    // ------------------------------------------------------------------ queries: kSweepsQ sweeps over rows of (token, head)
    // A lane has 16 bytes of either half of a row, twice what it has in the cache part, so that D / 16 lanes make a row.
    constexpr int kLanesQ = D / 16, kRowsQ = kStoreThreads / kLanesQ;
    const int lq = threadIdx.x % kLanesQ;
    const unsigned rows = (unsigned)(a.T * a.n_heads);
    uint4 w[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (g.q_norm != nullptr) {
      w[0] = load_near(reinterpret_cast<const uint4*>(g.q_norm + 8 * lq));
      w[1] = load_near(reinterpret_cast<const uint4*>(g.q_norm + D / 2 + 8 * lq));
    }
    bool bad = false;
    constexpr unsigned kChunk = kSweepsQ * kRowsQ;
    for (unsigned chunk = blockIdx.x - min(turn_of + 1, g.kv_ctas); (uint64_t)chunk * kChunk < rows; chunk += g.q_ctas) {
      const unsigned first = chunk * kChunk + threadIdx.x / kLanesQ;
      uint4 x[kSweepsQ][2];
      unsigned token[kSweepsQ];
#pragma unroll
      for (int i = 0; i < kSweepsQ; ++i) {
        const unsigned r = first + (unsigned)(i * kRowsQ);
        token[i] = r / (unsigned)a.n_heads;
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        if (r < rows) {
          const uint16_t* p = g.qkv + (int64_t)token[i] * g.ld + (int64_t)(r - token[i] * (unsigned)a.n_heads) * D + 8 * lq;
          x[i][0] = load_once(p);
          x[i][1] = load_once(p + D / 2);
        }
      }
      Angles turns[2]{};
      if (turn && first < rows) {                        // under way together with the rows
        const Places at = load_places(g.rope, a.T, token[0], bad);
        turns[0] = load_angles<D>(g.rope, at, 2 * lq);
        turns[1] = load_angles<D>(g.rope, at, 2 * lq + 1);
      }
#pragma unroll
      for (int i = 0; i < kSweepsQ; ++i) {
        const unsigned r = first + (unsigned)(i * kRowsQ);
        float lo[8], hi[8];
        unpack8(x[i][0], lo);
        unpack8(x[i][1], hi);
        if (g.q_norm != nullptr) {
          float s = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) s = fmaf(lo[j], lo[j], fmaf(hi[j], hi[j], s));
#pragma unroll
          for (int o = kLanesQ / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
          const float k = rsqrtf(s * (1.0f / D) + g.eps);
          float wl[8], wh[8];
          unpack8(w[0], wl);
          unpack8(w[1], wh);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            lo[j] = lo[j] * k * wl[j];
            hi[j] = hi[j] * k * wh[j];
          }
        }
        if (r >= rows) continue;
        if (turn) {
          if (i > 0 && token[i] != token[i - 1]) {       // heads of a token share its angles
            const Places at = load_places(g.rope, a.T, token[i], bad);
            turns[0] = load_angles<D>(g.rope, at, 2 * lq);
            turns[1] = load_angles<D>(g.rope, at, 2 * lq + 1);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float c = turns[j >> 2].c[j & 3], s = turns[j >> 2].s[j & 3], u = lo[j], v = hi[j];
            lo[j] = u * c - v * s;
            hi[j] = v * c + u * s;
          }
        }
        uint16_t* to = g.q_out + (int64_t)r * D + 8 * lq;
        *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(lo[4], lo[5]), pack_bf16(lo[6], lo[7]));
        *reinterpret_cast<uint4*>(to + D / 2) = make_uint4(pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]), pack_bf16(hi[4], hi[5]), pack_bf16(hi[6], hi[7]));
      }
    }
    if (bad) report_status(a.hdr, TLQ_ERR_SHAPE, 201);
    return;
  }

  // -------------------------------------------------------------------- one cache block of one head
  __shared__ long long sums[kStoreThreads / 32];
  __shared__ Found found;
  __shared__ float tops[2][kStoreThreads / 32];
  __shared__ __align__(16) int8_t turned[D * kPitch];
  const int h = (int)(turn_of % (unsigned)a.n_kv);
  auto blocks_of = [&](int b) -> long long {
    const Request r = load_request(a, b);
    return r.q_len > 0 ? (r.kv - 1) / kKvBlock - max(r.kv - r.q_len, 0) / kKvBlock + 1 : 0;
  };
  if (!locate_item<kStoreThreads>(a.B, turn_of / (unsigned)a.n_kv, blocks_of, sums, &found)) return;
  const Request req = load_request(a, found.request);
  const int begin = req.kv - req.q_len;              // place of the request's first new token
  if (begin < 0 && found.rest == 0) {                // fewer cached tokens than new ones, or a request that is left out
    if (threadIdx.x == 0) report_status(a.hdr, TLQ_ERR_SHAPE, 202);
    no_values<D>(g.k_values, g.v_values, a.n_kv, h, req.q0, min(-begin, req.q_len));
  }
  if (req.kv < 1) return;
  const int blk = max(begin, 0) / kKvBlock + (int)found.rest;
  const int p0 = max(max(begin, 0), blk * kKvBlock); // places [p0, p1) of the new tokens in this block
  const int p1 = min(req.kv, (blk + 1) * kKvBlock);
  const int n_new = p1 - p0;
  const int64_t tok0 = (int64_t)req.q0 + (p0 - begin);
  const int phys = a.block_table[(int64_t)found.request * a.max_blocks + blk];
  if (phys < 0 || phys >= a.n_blocks) {
    if (threadIdx.x == 0) report_status(a.hdr, TLQ_ERR_SHAPE, 203);
    no_values<D>(g.k_values, g.v_values, a.n_kv, h, tok0, n_new);
    return;
  }
  const int off0 = p0 - blk * kKvBlock;

  Raw kraw[kSweeps], vraw[kSweeps];
#pragma unroll
  for (int i = 0; i < kSweeps; ++i) {
    const int n = i * kRows + row;
    kraw[i] = vraw[i] = Raw{};
    if (n < n_new) {
      const uint16_t* p = g.qkv + (tok0 + n) * g.ld + (int64_t)(a.n_heads + h) * D;
      kraw[i] = load_raw<D>(p, l);
      vraw[i] = load_raw<D>(p + (int64_t)a.n_kv * D, l);
    }
  }
  Row<D> w{};
  if (g.k_norm != nullptr) w = floats<D>(load_raw<D>(g.k_norm, l));
  Angles turns[kSweeps];
  bool bad = false;
  if (turn) {
    Places at[kSweeps];
#pragma unroll
    for (int i = 0; i < kSweeps; ++i) at[i] = load_places(g.rope, a.T, tok0 + min(i * kRows + row, n_new - 1), bad);
#pragma unroll
    for (int i = 0; i < kSweeps; ++i) turns[i] = load_angles<D>(g.rope, at[i], l);
  }
  if (bad) report_status(a.hdr, TLQ_ERR_SHAPE, 201);
  Row<D> kx[kSweeps];
  float ktop = 0.f, vtop = 0.f, zeros = 0.f;         // zeros: NaN as soon as anything is not finite
#pragma unroll
  for (int i = 0; i < kSweeps; ++i) {
    const int n = i * kRows + row;
    kx[i] = floats<D>(kraw[i]);
    if (g.k_norm != nullptr) norm_row(kx[i], w, g.eps);
    if (n < n_new) {
      if (turn) rotate_row(kx[i], turns[i]);
      const Row<D> v = floats<D>(vraw[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ktop = fmaxf(ktop, fmaxf(fabsf(kx[i].lo[j]), fabsf(kx[i].hi[j])));
        vtop = fmaxf(vtop, fmaxf(fabsf(v.lo[j]), fabsf(v.hi[j])));
        zeros = fmaf(kx[i].lo[j], 0.f, fmaf(kx[i].hi[j], 0.f, fmaf(v.lo[j], 0.f, fmaf(v.hi[j], 0.f, zeros))));
      }
    }
  }
  const bool odd = zeros != 0.f;
  if (odd) {                                         // the largest of what is finite
    ktop = vtop = 0.f;
#pragma unroll
    for (int i = 0; i < kSweeps; ++i) {
      if (i * kRows + row >= n_new) break;
      const Row<D> v = floats<D>(vraw[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ktop = fmaxf(ktop, fmaxf(finite_size(kx[i].lo[j]), finite_size(kx[i].hi[j])));
        vtop = fmaxf(vtop, fmaxf(finite_size(v.lo[j]), finite_size(v.hi[j])));
      }
    }
  }
  if (odd) report_status(a.hdr, TLQ_ERR_NONFINITE, 204);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ktop = fmaxf(ktop, __shfl_xor_sync(0xFFFFFFFFu, ktop, o));
    vtop = fmaxf(vtop, __shfl_xor_sync(0xFFFFFFFFu, vtop, o));
  }
  if ((threadIdx.x & 31) == 0) {
    tops[0][threadIdx.x >> 5] = ktop;
    tops[1][threadIdx.x >> 5] = vtop;
  }
  const int64_t at = (int64_t)phys * a.n_kv + h;
  const float kold = off0 > 0 ? load_near(a.k_steps + at) : 0.f, vold = off0 > 0 ? load_near(a.v_steps + at) : 0.f;
  __syncthreads();                                   // also: every thread has read the old steps
#pragma unroll
  for (int i = 0; i < kStoreThreads / 32; ++i) {
    ktop = fmaxf(ktop, tops[0][i]);
    vtop = fmaxf(vtop, tops[1][i]);
  }
  const float kstep = fmaxf(kold, __fdiv_rn(fmaxf(ktop, TLQ_RANGE_FLOOR), 127.f));
  const float vstep = fmaxf(vold, __fdiv_rn(fmaxf(vtop, TLQ_RANGE_FLOOR), 127.f));
  const float kinv = __fdiv_rn(1.f, kstep), vinv = __fdiv_rn(1.f, vstep);
  if (threadIdx.x == 0) {
    a.k_steps[at] = kstep;
    a.v_steps[at] = vstep;
  }
  int8_t* kc = a.k_codes + at * kKvBlock * D;
  int8_t* vc = a.v_codes + at * kKvBlock * D;
  // older codes follow a step that grew
  if (kold > 0.f && kstep > kold) {
    const float f = __fdiv_rn(kold, kstep);
    for (int i = threadIdx.x; i < off0 * D / 4; i += kStoreThreads) {
      char4 c = reinterpret_cast<char4*>(kc)[i];
      c.x = (signed char)(int)rintf((float)c.x * f); c.y = (signed char)(int)rintf((float)c.y * f);
      c.z = (signed char)(int)rintf((float)c.z * f); c.w = (signed char)(int)rintf((float)c.w * f);
      reinterpret_cast<char4*>(kc)[i] = c;
    }
  }
  if (vold > 0.f && vstep > vold) {
    const float f = __fdiv_rn(vold, vstep);
    for (int i = threadIdx.x; i < D * kKvBlock; i += kStoreThreads)
      if (i % kKvBlock < off0) vc[i] = (int8_t)(int)rintf((float)vc[i] * f);
  }
#pragma unroll
  for (int i = 0; i < kSweeps; ++i) {
    const int n = i * kRows + row;
    if (n >= n_new) break;
    const Row<D> v = floats<D>(vraw[i]);
    uint32_t lo = 0, hi = 0;
    float klo[4], khi[4], vlo[4], vhi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int a0 = to_code(kx[i].lo[j], kstep, kinv), a1 = to_code(kx[i].hi[j], kstep, kinv);
      const int b0 = to_code(v.lo[j], vstep, vinv), b1 = to_code(v.hi[j], vstep, vinv);
      lo |= (uint32_t)(a0 & 255) << (8 * j);
      hi |= (uint32_t)(a1 & 255) << (8 * j);
      turned[(4 * l + j) * kPitch + n] = (int8_t)b0;
      turned[(D / 2 + 4 * l + j) * kPitch + n] = (int8_t)b1;
      klo[j] = (float)a0 * kstep; khi[j] = (float)a1 * kstep;
      vlo[j] = (float)b0 * vstep; vhi[j] = (float)b1 * vstep;
    }
    *reinterpret_cast<uint32_t*>(kc + (off0 + n) * D + 4 * l) = lo;
    *reinterpret_cast<uint32_t*>(kc + (off0 + n) * D + D / 2 + 4 * l) = hi;
    const int64_t to = ((tok0 + n) * a.n_kv + h) * D;
    if (g.k_values != nullptr) store_row<D>(g.k_values + to, klo, khi, l);
    if (g.v_values != nullptr) store_row<D>(g.v_values + to, vlo, vhi, l);
  }
  __syncthreads();
  if (n_new == kKvBlock) {
    for (int i = threadIdx.x; i < D * kKvBlock / 4; i += kStoreThreads)
      reinterpret_cast<uint32_t*>(vc)[i] =
          *reinterpret_cast<const uint32_t*>(turned + (i / (kKvBlock / 4)) * kPitch + (i % (kKvBlock / 4)) * 4);
  } else {
    for (int i = threadIdx.x; i < D * n_new; i += kStoreThreads) {
      const int c = i / n_new, n = i % n_new;
      vc[c * kKvBlock + off0 + n] = turned[c * kPitch + n];
    }
  }
}

}  // namespace

int launch_kv_store(const uint16_t* qkv, int64_t ld, int head_dim, const KvArgs& a, const RopeArgs& rope,
                    const uint16_t* q_norm, const uint16_t* k_norm, float eps, uint16_t* q_out, uint16_t* k_values,
                    uint16_t* v_values, cudaStream_t st) {
  StoreArgs g{};
  g.qkv = qkv; g.ld = ld; g.rope = rope; g.q_norm = q_norm; g.k_norm = k_norm; g.eps = eps;
  g.q_out = q_out; g.k_values = k_values; g.v_values = v_values;
  // n tokens of one request touch at most (n - 1) / 64 + 2 blocks and at most n
  int64_t blocks = a.T / kKvBlock + 2 * (int64_t)a.B;
  if (blocks > a.T) blocks = a.T;
  // enough CTAs of the streaming kind to fill the GPU several times over, each going round: a launch of one CTA for every
  // chunk spends its time on bringing CTAs up
  const int sms = device_sm_count();
  if (sms <= 0) return TLQ_ERR_CUDA;
  int64_t q_ctas = ceil_div(a.T * a.n_heads, (int64_t)kSweepsQ * kStoreThreads / (head_dim / 16));
  if (q_ctas > (int64_t)sms * kQueryWaves) q_ctas = (int64_t)sms * kQueryWaves;
  if (blocks * a.n_kv + q_ctas + kPadCtas > 0x7FFFFFFFLL) return TLQ_ERR_SHAPE;
  g.kv_ctas = (unsigned)(blocks * a.n_kv);
  g.q_ctas = (unsigned)q_ctas;
  const unsigned grid = g.kv_ctas + (unsigned)q_ctas;
  // Mixed when the cache part alone is more than the GPU holds at once (16384-token prompt, 64 / 8 heads: 152 us mixed, 171
  // with the cache part first); otherwise its chain is the longest and goes first (six ragged prompts: 12.5 us against 14.1).
  g.period = (int64_t)g.kv_ctas > 3 * (int64_t)sms ? grid / g.kv_ctas : 1;
  const dim3 all(grid + (k_values != nullptr || v_values != nullptr ? kPadCtas : 0u));
  return head_dim == 128 ? launch_next(kv_store_kernel<128>, all, kStoreThreads, 0, 1, st, a, g)
                         : launch_next(kv_store_kernel<64>, all, kStoreThreads, 0, 1, st, a, g);
}

}  // namespace tlq
