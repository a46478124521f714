// C ABI of the serving operators: argument validation and workspace layout.
#include <math.h>

#include "serve.cuh"

namespace tlq {
namespace {

constexpr size_t kHeaderBytes = sizeof(WorkspaceHeader);

int check_cache(const tlq_kv_cache* c) {
  if (c == nullptr || c->struct_size != sizeof(tlq_kv_cache)) return TLQ_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return TLQ_ERR_UNSUPPORTED;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_blocks < 1 || (int64_t)c->n_blocks * c->n_kv_heads > 0x7FFFFFFFLL)
    return TLQ_ERR_SHAPE;
  if (c->k_codes == nullptr || c->v_codes == nullptr || c->k_steps == nullptr || c->v_steps == nullptr)
    return TLQ_ERR_INVALID_ARG;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return TLQ_ERR_ALIGN;
  return TLQ_OK;
}

int check_batch(const tlq_kv_batch* b) {
  if (b == nullptr || b->struct_size != sizeof(tlq_kv_batch)) return TLQ_ERR_INVALID_ARG;
  if (b->n_requests < 1 || b->n_requests > 65535 || b->max_q_len < 0 || b->max_blocks < 1 || b->max_blocks > (1 << 24))
    return TLQ_ERR_SHAPE;
  if (b->cu_q == nullptr || b->kv_len == nullptr || b->block_table == nullptr) return TLQ_ERR_INVALID_ARG;
  return TLQ_OK;
}

int check_heads(int32_t n_heads, const tlq_kv_cache* c) {
  return n_heads >= 1 && n_heads <= 65536 && n_heads % c->n_kv_heads == 0 ? TLQ_OK : TLQ_ERR_SHAPE;
}

// Query rows of one request and kv head, at most.
int64_t query_rows(const tlq_kv_cache* c, const tlq_kv_batch* b, int32_t n_heads, int64_t T) {
  const int64_t n = T < b->max_q_len ? T : b->max_q_len;
  return n * (n_heads / c->n_kv_heads);
}

KvArgs make_args(const tlq_kv_cache* c, const tlq_kv_batch* b, int32_t n_heads, int64_t T, void* workspace) {
  KvArgs a{};
  a.k_codes = c->k_codes; a.v_codes = c->v_codes; a.k_steps = c->k_steps; a.v_steps = c->v_steps;
  a.cu_q = b->cu_q; a.kv_len = b->kv_len; a.block_table = b->block_table;
  a.T = T;
  a.n_blocks = c->n_blocks; a.max_blocks = b->max_blocks; a.B = b->n_requests; a.max_q_len = b->max_q_len;
  a.n_heads = n_heads; a.n_kv = c->n_kv_heads; a.group = n_heads / c->n_kv_heads;
  a.hdr = reinterpret_cast<WorkspaceHeader*>(workspace);
  return a;
}

}  // namespace
}  // namespace tlq

using namespace tlq;

extern "C" {

size_t tlq_linear_i8_workspace_bytes(int64_t N, int64_t C1, int64_t C2) {
  if (N < 0 || N > 0x7FFFFF00LL || C1 < 16 || (C1 % 16) != 0 || C1 > 131056 || C2 < 1 || C2 > 0x7FFFFF00LL) return 0;
  return kHeaderBytes;
}

int tlq_linear_i8(const int8_t* Xq, const float* t, int64_t N, int64_t C1, const int8_t* Wq, const float* u, int64_t C2,
                  const void* bias, void* workspace, size_t workspace_bytes, void* Y, void* stream) {
  const size_t need = tlq_linear_i8_workspace_bytes(N, C1, C2);
  if (need == 0) return TLQ_ERR_SHAPE;
  if (Wq == nullptr || u == nullptr || workspace == nullptr) return TLQ_ERR_INVALID_ARG;
  if (N > 0 && (Xq == nullptr || t == nullptr || Y == nullptr)) return TLQ_ERR_INVALID_ARG;
  if (!aligned16(Xq) || !aligned16(Wq) || !aligned16(workspace) || !aligned16(Y)) return TLQ_ERR_ALIGN;
  if (workspace_bytes < need) return TLQ_ERR_WORKSPACE;
  int rc = have_device();
  if (rc != TLQ_OK || N == 0) return rc;
  return launch_linear_i8(Xq, t, Wq, u, reinterpret_cast<const uint16_t*>(bias), N, C1, C2, reinterpret_cast<uint16_t*>(Y),
                          reinterpret_cast<WorkspaceHeader*>(workspace), reinterpret_cast<cudaStream_t>(stream));
}

size_t tlq_kv_workspace_bytes(const tlq_kv_cache* cache, const tlq_kv_batch* batch, int32_t n_heads, int64_t T) {
  if (check_cache(cache) != TLQ_OK || check_batch(batch) != TLQ_OK || check_heads(n_heads, cache) != TLQ_OK || T < 0) return 0;
  return align_up(kHeaderBytes + kv_split_floats(cache->head_dim, query_rows(cache, batch, n_heads, T)) * sizeof(float), 256);
}

int tlq_kv_store(const void* qkv, int64_t T, int64_t ld, int32_t n_heads, const tlq_kv_cache* cache,
                 const tlq_kv_batch* batch, const int32_t* positions, int32_t n_axes, const int32_t* sections,
                 const float* cos_sin, int64_t n_positions, const void* q_norm, const void* k_norm, float eps, void* q_out,
                 void* k_values, void* v_values, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc == TLQ_OK) rc = check_batch(batch);
  if (rc == TLQ_OK) rc = check_heads(n_heads, cache);
  if (rc != TLQ_OK) return rc;
  if (T < 0 || T > 0x7FFFFF00LL || T * n_heads > 0x7FFFFF00LL) return TLQ_ERR_SHAPE;
  if (workspace == nullptr) return TLQ_ERR_INVALID_ARG;
  if (T > 0 && (qkv == nullptr || q_out == nullptr)) return TLQ_ERR_INVALID_ARG;
  const int d = cache->head_dim;
  if (ld < (int64_t)(n_heads + 2 * cache->n_kv_heads) * d || (ld % 8) != 0) return TLQ_ERR_SHAPE;
  if (!(eps >= 0.0f) || isinf(eps)) return TLQ_ERR_INVALID_ARG;
  RopeArgs rope{};
  if (positions != nullptr) {
    if (cos_sin == nullptr) return TLQ_ERR_INVALID_ARG;
    if (n_axes != 1 && n_axes != 3) return TLQ_ERR_UNSUPPORTED;
    if (n_positions < 1) return TLQ_ERR_SHAPE;
    if (sections == nullptr && n_axes != 1) return TLQ_ERR_INVALID_ARG;
    int64_t end = 0;
    for (int i = 0; i < n_axes; ++i) {
      const int64_t n = sections == nullptr ? d / 2 : sections[i];
      if (n < 0) return TLQ_ERR_SHAPE;
      end += n;
      if (end > d / 2) return TLQ_ERR_SHAPE;
      rope.pairs_end[i] = (int)end;
    }
    if (end != d / 2) return TLQ_ERR_SHAPE;
    rope.positions = positions;
    rope.cos_sin = cos_sin;
    rope.n_positions = n_positions;
    rope.n_axes = n_axes;
  }
  if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(k_values) || !aligned16(v_values) || !aligned16(workspace) ||
      !aligned16(cos_sin) || !aligned16(q_norm) || !aligned16(k_norm))
    return TLQ_ERR_ALIGN;
  if (workspace_bytes < tlq_kv_workspace_bytes(cache, batch, n_heads, T)) return TLQ_ERR_WORKSPACE;
  rc = have_device();
  if (rc != TLQ_OK || T == 0) return rc;
  return launch_kv_store(reinterpret_cast<const uint16_t*>(qkv), ld, d, make_args(cache, batch, n_heads, T, workspace), rope,
                         reinterpret_cast<const uint16_t*>(q_norm), reinterpret_cast<const uint16_t*>(k_norm), eps,
                         reinterpret_cast<uint16_t*>(q_out), reinterpret_cast<uint16_t*>(k_values),
                         reinterpret_cast<uint16_t*>(v_values), reinterpret_cast<cudaStream_t>(stream));
}

int tlq_kv_attention(const void* q, int64_t T, int64_t ldq, int32_t n_heads, const tlq_kv_cache* cache,
                     const tlq_kv_batch* batch, float scale, int32_t causal, void* workspace, size_t workspace_bytes,
                     void* out, float* lse, void* stream) {
  int rc = check_cache(cache);
  if (rc == TLQ_OK) rc = check_batch(batch);
  if (rc == TLQ_OK) rc = check_heads(n_heads, cache);
  if (rc != TLQ_OK) return rc;
  if (T < 0 || T > 0x7FFFFF00LL || T * (n_heads / cache->n_kv_heads) > 0x7FFFFF00LL) return TLQ_ERR_SHAPE;
  if (workspace == nullptr) return TLQ_ERR_INVALID_ARG;
  if (T > 0 && (q == nullptr || out == nullptr)) return TLQ_ERR_INVALID_ARG;
  if (ldq < (int64_t)n_heads * cache->head_dim || (ldq % 8) != 0) return TLQ_ERR_SHAPE;
  if (!(scale > 0.0f) || isinf(scale)) return TLQ_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return TLQ_ERR_ALIGN;
  if (workspace_bytes < tlq_kv_workspace_bytes(cache, batch, n_heads, T)) return TLQ_ERR_WORKSPACE;
  rc = have_device();
  if (rc != TLQ_OK || T == 0) return rc;
  uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
  KvSplit split;
  split.base = reinterpret_cast<float*>(ws + kHeaderBytes);
  return launch_kv_attention(reinterpret_cast<const uint16_t*>(q), ldq, cache->head_dim,
                             make_args(cache, batch, n_heads, T, workspace), scale, causal,
                             reinterpret_cast<uint16_t*>(out), lse, split, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
