// Shared declarations of the serving operators: the 8-bit product, the key-value store and attention over the cache.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace tlq {

constexpr int kKvBlock = TLQ_KV_BLOCK;   // tokens of one cache block

// What the kernels need of a batch and of the cache (device pointers).
struct KvArgs {
  int8_t* k_codes;            // [n_blocks][Hkv][64][D]
  int8_t* v_codes;            // [n_blocks][Hkv][D][64]
  float* k_steps;             // [n_blocks][Hkv]
  float* v_steps;
  const int32_t* cu_q;        // [B + 1]
  const int32_t* kv_len;      // [B]
  const int32_t* block_table; // [B][max_blocks]
  int64_t T;                  // rows of q / qkv
  int n_blocks, max_blocks, B, max_q_len;
  int n_heads, n_kv, group;   // group = n_heads / n_kv
  WorkspaceHeader* hdr;
};

__device__ __forceinline__ void report_status(WorkspaceHeader* hdr, int status, int where) {
  hdr->where = where;
  hdr->status = status;
}

// Lengths of one request, forced into what the call's buffers hold, so that no metadata can move an access out of bounds; anything
// else is reported.  A request whose cached tokens go beyond its table, or that has more new tokens than the batch allows, is left
// out whole (as if it had no cached token): with lengths cut to what fits its new tokens would take the places of older ones.
struct Request {
  int q0, q_len, kv;          // first row of q, new tokens, cached tokens with the new ones
};
__device__ __forceinline__ Request load_request(const KvArgs& a, int b) {
  const int c0 = a.cu_q[b], c1 = a.cu_q[b + 1], kv = a.kv_len[b];
  Request r;
  r.q0 = max(0, min(c0, (int)a.T));
  const int end = max(r.q0, min(c1, (int)a.T));
  r.q_len = end - r.q0;
  const bool fits = kv >= 0 && kv <= (long long)a.max_blocks * kKvBlock && r.q_len <= a.max_q_len;
  r.kv = fits ? kv : 0;
  if (r.q0 != c0 || end != c1 || !fits) report_status(a.hdr, TLQ_ERR_SHAPE, 200);
  return r;
}

// Rows of the token tensors that belong to no request: those before the first one's and after the last one's (padding).
struct Padding {
  int before, after;          // rows [0, before) and [after, T)
};
__device__ __forceinline__ Padding load_padding(const int32_t* cu_q, int B, int64_t T) {
  Padding p;
  p.before = max(0, min(cu_q[0], (int)T));
  p.after = max(p.before, min(cu_q[B], (int)T));
  return p;
}
// Rows [from, to) of `pieces` 16-byte pieces each become zeros; thread number t of n does its share.
__device__ __forceinline__ void zero_rows(void* p, int64_t from, int64_t to, int64_t pieces, int64_t t, int64_t n) {
  for (int64_t i = from * pieces + t; i < to * pieces; i += n) reinterpret_cast<uint4*>(p)[i] = make_uint4(0, 0, 0, 0);
}

// Inclusive scan of one value per thread of a block of kThreads; `sums` is kThreads / 32 words of shared memory.
template <int kThreads>
__device__ __forceinline__ long long block_scan(long long v, long long* sums, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long n = __shfl_up_sync(0xFFFFFFFFu, v, o);
    if (lane >= o) v += n;
  }
  __syncthreads();               // earlier readers of `sums` are done
  if (lane == 31) sums[warp] = v;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const long long s = sums[w];
    if (w < warp) before += s;
    total += s;
  }
  return v + before;
}

// The request that holds item number `target` when request b owns count(b) items, and the item's number in it.
// All threads of the block call it; `found` (shared) receives {request, number in it}.  False when there is none.
struct Found {
  long long rest;
  int request;
};
template <int kThreads, typename F>
__device__ __forceinline__ bool locate_item(int B, long long target, F count, long long* sums, Found* found) {
  long long base = 0;
  if (threadIdx.x == 0) found->request = -1;
  for (int b0 = 0; b0 < B; b0 += kThreads) {
    const int b = b0 + (int)threadIdx.x;
    const long long n = b < B ? count(b) : 0;
    long long total;
    const long long upto = block_scan<kThreads>(n, sums, total);
    if (n > 0 && target - base >= upto - n && target - base < upto) {
      found->request = b;
      found->rest = target - base - (upto - n);
    }
    base += total;
    if (target < base) break;
  }
  __syncthreads();
  return found->request >= 0;
}

// Both in one: the number of all items, and the item that target_of(total) names (none where that is negative).
template <int kThreads, typename F, typename G>
__device__ __forceinline__ bool plan_items(int B, F count, G target_of, long long* sums, Found* found, long long& total) {
  const int b = (int)threadIdx.x;
  const long long n = b < B ? count(b) : 0;
  if (threadIdx.x == 0) found->request = -1;
  const long long upto = block_scan<kThreads>(n, sums, total);
  for (int b0 = kThreads; b0 < B; b0 += kThreads) {
    long long part;
    block_scan<kThreads>(b0 + b < B ? count(b0 + b) : 0, sums, part);
    total += part;
  }
  if (total == 0) return false;
  const long long target = target_of(total);
  if (target < 0) return false;
  if (B > kThreads) return locate_item<kThreads>(B, target, count, sums, found);
  if (n > 0 && target >= upto - n && target < upto) {
    found->request = b;
    found->rest = target - (upto - n);
  }
  __syncthreads();
  return found->request >= 0;
}

constexpr int kPromptRows = 32;           // requests with at least this many query rows per kv head go to it ...
// ... if such requests have this many pairs of a row and a key, every row counted with 256 keys on top (the few-row kernel
// works on 16 rows at a time and pays for each such item once), requests of fewer than 64 rows by a third (the prompt kernel
// works on 128 rows at least).  The prompt kernel and its join take 25 us however little there is to do, the few-row kernel 8 to
// 12, and 6 more behind a prompt kernel that finds it has nothing to do, but that one gets no more than 0.25 M pairs done in a us.
// Measured, few-row kernel alone against prompt kernel:
// 126 rows x 4096 keys x 4 kv heads (2.2 M) 24 : 33 us, 336 x 2000 x 4 (3.0 M) 28 : 38, prompts of 512 tokens with 512 rows x 8
// (2.1 M) 24 : 27, 3072 x 2 (3.1 M) 24 : 36 and 3584 x 4 (7.3 M) 32 : 38, 800 rows x 1000 x 8 (7.7 M) 51 : 40, 840 x 4096 x 4
// (15 M) 61 : 47, 576 rows in 8 requests x 8000 x 8 (38 M) 131 : 92; requests of 32 to 40 rows: 35 x 30000 x 4 (4.2 M) 38 : 57,
// 128 x 8192 x 8 (8.7 M) 44 : 63, 280 x 8192 x 4 (9.5 M) 56 : 64, 320 x 8192 x 8 (22 M) 89 : 94.  (The limits come from when the
// few-row kernel took 5 to 10 us longer for its joins: the prompts of 512 tokens and the requests of 35 rows are the ones that would
// gain from a higher one, 800 rows x 1000 x 8 from a lower one.)
constexpr long long kPromptPairs = 3100000;
constexpr int kFullRows = 64;
constexpr int kRowKeys = 256;

// Whether the requests of at least kPromptRows rows are the prompt kernel's: their pairs of a row and a key (about half of the
// new ones where the mask is causal), all counted by both kernels alike.  All threads of the block call it.
template <int kThreads>
__device__ __forceinline__ bool is_prompt_work(const KvArgs& a, int causal, long long* sums) {
  long long all = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + (int)threadIdx.x;
    long long n = 0, total;
    if (b < a.B) {
      const Request r = load_request(a, b);
      const long long rows = (long long)r.q_len * a.group;
      if (rows >= kPromptRows) n = rows * ((causal ? max(r.kv - r.q_len / 2, r.kv / 2) : r.kv) + kRowKeys) * a.n_kv / (rows < kFullRows ? 3 : 1);
    }
    block_scan<kThreads>(n, sums, total);
    all += total;
  }
  return all >= kPromptPairs;
}

// ---------------------------------------------------------------------------------------------- numbers of the attention kernels
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Four 8-bit codes to two pairs of f16.  Keys: code + 128 in the lowest byte of a 16-bit float is the (subnormal, exact)
// number (code + 128) 2^-24.  Values: exactly the code, as 1024 + (code + 128) by byte placement, minus 1152; a sum of
// p (code + 128) less 128 sum(p) would leave a rounding of 2^-23 x 128 in channels whose own values are small.
constexpr float kUnit = 16777216.f;       // 2^24
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

// ---------------------------------------------------------------------------------------------- launches
// Kernels of these operators follow one another in every layer, most of them a few microseconds long.  They are launched
// so that a kernel's blocks may come up while the one before it on the stream still runs (programmatic dependent
// launch); after_previous() is the first thing that reads or writes memory: it waits until everything earlier on the
// stream is complete and visible, and then lets the next kernel come up in turn.
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// Nothing that a call is given is therefore constant for its kernel's whole life, which begins while the kernel before may still
// write it: the read-only path (ld.global.nc, which __ldg and const __restrict__ ask for) is not for these kernels.  The loads
// below are ordinary ones, for which the wait makes everything that was written before visible, and volatile, so that none can
// move before it.
template <typename T>
__device__ __forceinline__ T load_near(const T* p) {       // may stay in the SM's first-level cache
  static_assert(sizeof(T) == 4 || sizeof(T) == 8 || sizeof(T) == 16, "");
  union { T t; uint32_t w[sizeof(T) / 4]; } u;
  if constexpr (sizeof(T) == 4)
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(u.w[0]) : "l"(p) : "memory");
  else if constexpr (sizeof(T) == 8)
    asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(u.w[0]), "=r"(u.w[1]) : "l"(p) : "memory");
  else
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]) : "l"(p) : "memory");
  return u.t;
}
// From the second-level cache: partial sums, each read once.  (The steps of the cache are better kept near, since a warp's next
// blocks have theirs in the same lines: 64 requests of one token 79.7 us, 82.7 with these.)
template <typename T>
__device__ __forceinline__ T load_far(const T* p) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 16, "");
  union { T t; uint32_t w[sizeof(T) / 4]; } u;
  if constexpr (sizeof(T) == 4)
    asm volatile("ld.global.cg.b32 %0, [%1];" : "=r"(u.w[0]) : "l"(p) : "memory");
  else
    asm volatile("ld.global.cg.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]) : "l"(p) : "memory");
  return u.t;
}
__device__ __forceinline__ uint4 load_once(const void* p) { // 16 bytes that no other warp of the SM will read
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
template <typename... Params, typename... Args>
inline int launch_next(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, unsigned cluster, cudaStream_t st,
                       Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return TLQ_ERR_CUDA;
  }
  return after_launch();
}

// ---------------------------------------------------------------------------------------------- launchers
// kv_store.cu
struct RopeArgs {
  const int32_t* positions;   // [axes][T] or null (no rotation)
  const float* cos_sin;       // [n_positions][D]: cosines of the D/2 pairs, then sines
  int64_t n_positions;
  int n_axes;
  int pairs_end[3];           // pairs [pairs_end[a-1], pairs_end[a]) turn by position axis a
};
int launch_kv_store(const uint16_t* qkv, int64_t ld, int head_dim, const KvArgs& a, const RopeArgs& rope,
                    const uint16_t* q_norm, const uint16_t* k_norm, float eps, uint16_t* q_out, uint16_t* k_values,
                    uint16_t* v_values, cudaStream_t st);

// kv_attention.cu, kv_prompt.cu, kv_join.cu: the split over the cache
constexpr int kMaxWorkers = 160;          // CTAs that share one call's work (one per SM)
constexpr int kSplitWarps = 8;            // warps of one of them in the few-row kernel, each with a part of its own
constexpr int kMaxRowTile = 16;           // query rows of one of its items (8 or 16)
constexpr int kPromptItemRows = 256;      // query rows of one item of the prompt kernel
constexpr int kPromptJoinRows = 32;       // rows of such an item that a CTA joins
constexpr float kFewShift = 15.f, kPromptShift = 11.f;     // the sums hold 2^shift p
// Value steps below this count as this: blocks that nothing was written to have a step of zero (the store's own are 7.9e-8 at least).
// The sum of p / step over the 2^30 tokens that a table can name stays below 2^(16 + 80 + 30), inside the 32-bit range.
constexpr float kStepFloor = 8.2718061255302767e-25f;      // 2^-80
static_assert((long long)(1 << 24) * kKvBlock <= 1ll << 30, "max_blocks is at most 2^24");
struct __align__(16) PartNote {           // a part of an item's blocks
  long long item;             // where the item is on the line of its kernel; negative: there is no part
  int first, last;            // the part has the item's first, its last blocks
  int h, tile, q0, q_len;     // kv head, row tile, first row of q and new tokens of the request
};
// The workspace after its header: two partials of every worker (a maximum, a sum and D output sums of each row), their notes; of
// the few-row kernel, then of the prompt kernel.  All of it is written in every call before it is read.
__host__ __device__ constexpr size_t few_floats(int d) { return (size_t)kMaxWorkers * kSplitWarps * 2 * kMaxRowTile * ((size_t)d + 2); }
__host__ __device__ constexpr size_t prompt_floats(int d) { return (size_t)kMaxWorkers * 2 * kPromptItemRows * ((size_t)d + 2); }
constexpr size_t kNoteFloats = sizeof(PartNote) / sizeof(float);
constexpr size_t kFewNoteFloats = (kMaxWorkers * kSplitWarps * 2 + 1) * kNoteFloats;   // and the number of workers behind them
inline size_t kv_split_floats(int head_dim, int64_t rows) {
  const size_t few = few_floats(head_dim) + kFewNoteFloats;
  return rows < kPromptRows ? few : few + prompt_floats(head_dim) + kMaxWorkers * 2 * kNoteFloats;
}
struct KvSplit {
  float* base;                // kv_split_floats()
};
__device__ __forceinline__ float* few_partials(const KvSplit& s) { return s.base; }
__device__ __forceinline__ PartNote* few_notes(const KvSplit& s, int d) { return reinterpret_cast<PartNote*>(s.base + few_floats(d)); }
__device__ __forceinline__ int* few_workers(const KvSplit& s, int d) {
  return reinterpret_cast<int*>(few_notes(s, d) + kMaxWorkers * kSplitWarps * 2);
}
__device__ __forceinline__ float* prompt_partials(const KvSplit& s, int d) { return s.base + few_floats(d) + kFewNoteFloats; }
__device__ __forceinline__ PartNote* prompt_notes(const KvSplit& s, int d) {
  return reinterpret_cast<PartNote*>(prompt_partials(s, d) + prompt_floats(d));
}
int launch_kv_prompt(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal, uint16_t* out,
                     float* lse, const KvSplit& split, int ctas, cudaStream_t st);
int launch_kv_join(int head_dim, const KvArgs& a, int ctas, int few_rows, bool prompts, uint16_t* out, float* lse,
                   const KvSplit& split, cudaStream_t st);
int launch_kv_attention(const uint16_t* q, int64_t ldq, int head_dim, const KvArgs& a, float scale, int causal,
                        uint16_t* out, float* lse, const KvSplit& split, cudaStream_t st);

// linear_i8.cu
int launch_linear_i8(const int8_t* Xq, const float* t, const int8_t* Wq, const float* u, const uint16_t* bias, int64_t N,
                     int64_t C1, int64_t C2, uint16_t* Y, WorkspaceHeader* hdr, cudaStream_t st);

}  // namespace tlq
