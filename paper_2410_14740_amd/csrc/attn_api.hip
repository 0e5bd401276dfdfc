// Host side of the attention calls of the C ABI: argument checks and launches.
#include "kv_device.h"

namespace m2c {
int64_t prompt_workspace(const m2c_attn_desc* D, bool self, int n_seqs, int64_t total_q, int64_t total_k);
hipError_t launch_prompt_attention(const m2c_attn_desc* D, const void* q, const void* k,
                                   const void* v, const int32_t* cu_q, const int32_t* cu_k,
                                   int n_seqs, int64_t total_q, int64_t total_k, void* out,
                                   float* lse, hipStream_t stream);
}

namespace {

using m2c::api_fail;
using m2c::KvView;

struct CurrentDevice {
  int prev = -1;
  bool ok = false;
  explicit CurrentDevice(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    ok = prev == dev || hipSetDevice(dev) == hipSuccess;
    if (prev == dev) prev = -1;
  }
  ~CurrentDevice() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

m2c_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return M2C_OK;
  (void)hipGetLastError();
  return api_fail(M2C_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

constexpr int64_t kMaxRows = 1 << 30;  // rows of a call: their indices and those past the last fit 32 bits

constexpr int64_t kMaxTokenStride = 1 << 24;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Rows may share heads (a head stride of 0), but tokens lie apart; a tile of
// them spans less than 4 GB.
m2c_status check_rows(const char* what, const void* p, const int64_t* stride, int head_dim) {
  if (!p || !stride) return api_fail(M2C_ERR_INVALID_ARG, "%s: NULL argument", what);
  if (misaligned(p)) return api_fail(M2C_ERR_INVALID_ARG, "%s: not 16-byte aligned", what);
  for (int i = 0; i < 2; ++i)
    if (stride[i] < 0 || stride[i] % 8 || stride[i] > ((int64_t)1 << 40))
      return api_fail(M2C_ERR_INVALID_ARG, "%s: stride %lld: need a multiple of 8 elements, >= 0",
                      what, (long long)stride[i]);
  if (stride[0] < head_dim || stride[0] > kMaxTokenStride)
    return api_fail(M2C_ERR_INVALID_ARG, "%s: token stride %lld: need [head_dim, 2^24] elements", what,
                    (long long)stride[0]);
  return M2C_OK;
}

// Rows that are written: no two of them may overlap.
m2c_status check_written(const char* what, const void* p, const int64_t* stride, int64_t tokens, int heads,
                         int head_dim) {
  const m2c_status rc = check_rows(what, p, stride, head_dim);
  if (rc != M2C_OK) return rc;
  if (stride[0] < (heads - 1) * stride[1] + head_dim && stride[1] < (tokens - 1) * stride[0] + head_dim)
    return api_fail(M2C_ERR_INVALID_ARG, "%s: rows overlap with strides %lld, %lld", what,
                    (long long)stride[0], (long long)stride[1]);
  if (heads > 1 && stride[1] < head_dim)
    return api_fail(M2C_ERR_INVALID_ARG, "%s: head stride %lld: need >= head_dim", what, (long long)stride[1]);
  return M2C_OK;
}

m2c_status check_heads(int dtype, int n_heads, int n_kv_heads, int head_dim, float scale, int device) {
  if (dtype != M2C_DTYPE_FP16 && dtype != M2C_DTYPE_BF16)
    return api_fail(M2C_ERR_INVALID_ARG, "dtype %d: need M2C_DTYPE_FP16 or M2C_DTYPE_BF16", dtype);
  if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads > 1024 || n_heads % n_kv_heads)
    return api_fail(M2C_ERR_INVALID_ARG, "n_heads %d over n_kv_heads %d: need a multiple, at most 1024",
                    n_heads, n_kv_heads);
  if (head_dim != 64 && head_dim != 128)
    return api_fail(M2C_ERR_INVALID_ARG, "head_dim %d: need 64 or 128", head_dim);
  if (!(scale >= 0.0f) || scale > 1e30f)
    return api_fail(M2C_ERR_INVALID_ARG, "scale %g: need >= 0 and finite", (double)scale);
  if (device < 0) return api_fail(M2C_ERR_INVALID_ARG, "device %d", device);
  return M2C_OK;
}

m2c_status view_of(const m2c_kv_cache* c, KvView* v) {
  if (!c) return api_fail(M2C_ERR_INVALID_ARG, "cache is NULL");
  const m2c_status rc = check_heads(c->dtype, c->n_kv_heads, c->n_kv_heads, c->head_dim, 0.0f, c->device);
  if (rc != M2C_OK) return rc;
  if (c->n_seqs < 1 || c->n_seqs > 65535)
    return api_fail(M2C_ERR_INVALID_ARG, "n_seqs %d: need [1, 65535]", c->n_seqs);
  if (c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128)
    return api_fail(M2C_ERR_INVALID_ARG, "block_tokens %d: need 32, 64 or 128", c->block_tokens);
  if (c->max_blocks < 1 || c->max_blocks > 16384)
    return api_fail(M2C_ERR_INVALID_ARG, "max_blocks %d: need [1, 16384]", c->max_blocks);
  if (c->n_pages < 1 || c->n_pages > INT32_MAX)
    return api_fail(M2C_ERR_INVALID_ARG, "n_pages %lld: need [1, 2^31 - 1]", (long long)c->n_pages);
  if (c->reserved) return api_fail(M2C_ERR_INVALID_ARG, "reserved %d: need 0", c->reserved);
  const void* need[] = {c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->tail_k, c->tail_v,
                        c->table, c->len, c->weight, c->arrive, c->status};
  for (const void* p : need)
    if (!p) return api_fail(M2C_ERR_INVALID_ARG, "cache: NULL array");
  if (misaligned(c->k_codes) || misaligned(c->v_codes) || misaligned(c->tail_k) || misaligned(c->tail_v))
    return api_fail(M2C_ERR_INVALID_ARG, "cache: codes and tails need 16-byte alignment");
  v->k_codes = c->k_codes, v->v_codes = c->v_codes;
  v->k_scale = c->k_scale, v->v_scale = c->v_scale;
  v->tail_k = (uint8_t*)c->tail_k, v->tail_v = (uint8_t*)c->tail_v;
  v->table = c->table, v->len = c->len, v->weight = c->weight;
  v->arrive = c->arrive, v->status = c->status;
  v->n_pages = c->n_pages;
  v->n_seqs = c->n_seqs, v->n_kv_heads = c->n_kv_heads, v->head_dim = c->head_dim;
  v->block_tokens = c->block_tokens, v->max_blocks = c->max_blocks;
  v->bf = c->dtype == M2C_DTYPE_BF16;
  return M2C_OK;
}

m2c_status check_n(const KvView& C, int n) {
  if (n < 1 || n > C.n_seqs)
    return api_fail(M2C_ERR_INVALID_ARG, "n %d: need [1, n_seqs=%d]", n, C.n_seqs);
  return M2C_OK;
}

m2c_status check_prompt(const m2c_attn_desc* D, int n_seqs, int64_t total_q, int64_t total_k) {
  if (!D) return api_fail(M2C_ERR_INVALID_ARG, "prompt attention: NULL argument");
  const m2c_status rc = check_heads(D->dtype, D->n_heads, D->n_kv_heads, D->head_dim, D->scale, D->device);
  if (rc != M2C_OK) return rc;
  if (D->causal != 0 && D->causal != 1)
    return api_fail(M2C_ERR_INVALID_ARG, "causal %d: need 0 or 1", D->causal);
  if (D->max_q < 0) return api_fail(M2C_ERR_INVALID_ARG, "max_q %d: need >= 0", D->max_q);
  if (n_seqs < 1 || n_seqs > 65535)
    return api_fail(M2C_ERR_INVALID_ARG, "n_seqs %d: need [1, 65535]", n_seqs);
  if (total_q < 0 || total_q > kMaxRows || total_k < 0 || total_k > kMaxRows)
    return api_fail(M2C_ERR_INVALID_ARG, "total_q %lld, total_k %lld: need [0, 2^30]",
                    (long long)total_q, (long long)total_k);
  return M2C_OK;
}

#define CHECKED(call)                    \
  do {                                   \
    const m2c_status rc_ = (call);       \
    if (rc_ != M2C_OK) return rc_;       \
  } while (0)

}  // namespace

extern "C" {

int64_t m2c_prompt_attention_workspace(const m2c_attn_desc* D, const int32_t* cu_q, const int32_t* cu_k,
                                       int32_t n_seqs, int64_t total_q, int64_t total_k) {
  if (check_prompt(D, n_seqs, total_q, total_k) != M2C_OK) return -1;
  return total_q ? m2c::prompt_workspace(D, cu_q == cu_k, n_seqs, total_q, total_k) : 0;
}

m2c_status m2c_prompt_attention(const m2c_attn_desc* D, const void* q, const void* k, const void* v,
                                const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                                int64_t total_q, int64_t total_k, void* out, float* lse,
                                void* stream) {
  CHECKED(check_prompt(D, n_seqs, total_q, total_k));
  if (!cu_q || !cu_k) return api_fail(M2C_ERR_INVALID_ARG, "prompt attention: NULL argument");
  if (total_q == 0) return M2C_OK;
  if (D->workspace) {
    const int64_t need = m2c::prompt_workspace(D, cu_q == cu_k, n_seqs, total_q, total_k);
    if ((uintptr_t)D->workspace & 255)
      return api_fail(M2C_ERR_INVALID_ARG, "workspace: not 256-byte aligned");
    if (D->workspace_bytes < need)
      return api_fail(M2C_ERR_CAPACITY, "workspace of %lld bytes: need %lld", (long long)D->workspace_bytes,
                      (long long)need);
  }
  CHECKED(check_rows("q", q, D->q_stride, D->head_dim));
  CHECKED(check_written("out", out, D->out_stride, total_q, D->n_heads, D->head_dim));
  if (total_k > 0) {
    CHECKED(check_rows("k", k, D->k_stride, D->head_dim));
    CHECKED(check_rows("v", v, D->v_stride, D->head_dim));
  }
  CurrentDevice g(D->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", D->device);
  return launched(m2c::launch_prompt_attention(D, q, k, v, cu_q, cu_k, n_seqs, total_q, total_k, out,
                                               lse, (hipStream_t)stream),
                  "prompt attention");
}

m2c_status m2c_kv_reset(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CHECKED(check_n(C, n));
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  return launched(m2c::launch_kv_reset(C, seqs, n, (hipStream_t)stream), "reset");
}

m2c_status m2c_kv_append(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n,
                         const int32_t* cu, int64_t total, const int32_t* pos, const void* k,
                         const void* v, const int64_t k_stride[2], const int64_t v_stride[2],
                         void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CHECKED(check_n(C, n));
  if (total < 0 || total > kMaxRows || (!cu && total != n))
    return api_fail(M2C_ERR_INVALID_ARG, "total %lld: need [0, 2^30], and n without cu", (long long)total);
  if (total == 0) return M2C_OK;
  CHECKED(check_rows("k", k, k_stride, C.head_dim));
  CHECKED(check_rows("v", v, v_stride, C.head_dim));
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  return launched(m2c::launch_kv_append(C, seqs, n, cu, total, pos, k, v, k_stride, v_stride,
                                        (hipStream_t)stream), "append");
}

m2c_status m2c_kv_read(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, const int32_t* cu,
                       int64_t total, void* k, void* v, const int64_t k_stride[2],
                       const int64_t v_stride[2], void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CHECKED(check_n(C, n));
  if (!cu) return api_fail(M2C_ERR_INVALID_ARG, "cu is NULL");
  if (total < 0 || total > kMaxRows)
    return api_fail(M2C_ERR_INVALID_ARG, "total %lld: need [0, 2^30]", (long long)total);
  if (total == 0) return M2C_OK;
  CHECKED(check_written("k", k, k_stride, total, C.n_kv_heads, C.head_dim));
  CHECKED(check_written("v", v, v_stride, total, C.n_kv_heads, C.head_dim));
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  return launched(m2c::launch_kv_read(C, seqs, n, cu, total, k, v, k_stride, v_stride,
                                      (hipStream_t)stream), "read");
}

int64_t m2c_kv_attend_workspace(const m2c_kv_cache* cache, int32_t n, int32_t n_heads, int32_t track,
                                int32_t max_len) {
  KvView C;
  if (view_of(cache, &C) != M2C_OK || check_n(C, n) != M2C_OK ||
      check_heads(cache->dtype, n_heads, C.n_kv_heads, C.head_dim, 0.0f, cache->device) != M2C_OK)
    return -1;
  if (max_len < 0) {
    api_fail(M2C_ERR_INVALID_ARG, "max_len %d: need >= 0", max_len);
    return -1;
  }
  return m2c::kv_attend_workspace(C, n, n_heads, track != 0, max_len);
}

m2c_status m2c_kv_attend(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, int32_t n_heads,
                         float scale, const void* q, const int64_t q_stride[2], void* out,
                         const int64_t out_stride[2], float* lse, int32_t track, int32_t max_len,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CHECKED(check_n(C, n));
  CHECKED(check_heads(cache->dtype, n_heads, C.n_kv_heads, C.head_dim, scale, cache->device));
  if (track != 0 && track != 1) return api_fail(M2C_ERR_INVALID_ARG, "track %d: need 0 or 1", track);
  if (max_len < 0) return api_fail(M2C_ERR_INVALID_ARG, "max_len %d: need >= 0", max_len);
  CHECKED(check_rows("q", q, q_stride, C.head_dim));
  CHECKED(check_written("out", out, out_stride, n, n_heads, C.head_dim));
  const int64_t need = m2c::kv_attend_workspace(C, n, n_heads, track, max_len);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 255)))
    return api_fail(M2C_ERR_INVALID_ARG, "workspace: need %lld bytes, 256-byte aligned", (long long)need);
  if (workspace_bytes < need)
    return api_fail(M2C_ERR_CAPACITY, "workspace of %lld bytes: need %lld", (long long)workspace_bytes,
                    (long long)need);
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  return launched(m2c::launch_kv_attend(C, seqs, n, n_heads, scale, q, q_stride, out, out_stride, lse,
                                        track, max_len, workspace, (hipStream_t)stream), "attend");
}

m2c_status m2c_kv_evict(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, int32_t keep,
                        int32_t first, int32_t recent, int32_t* table_out, float* weight_out,
                        int32_t* len_out, void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CHECKED(check_n(C, n));
  if (first < 0 || recent < 0 || keep < 0 || (int64_t)first + recent > keep)
    return api_fail(M2C_ERR_INVALID_ARG, "keep %d, first %d, recent %d: need first + recent <= keep",
                    keep, first, recent);
  const int outs = (table_out != nullptr) + (weight_out != nullptr) + (len_out != nullptr);
  if (outs != 0 && outs != 3)
    return api_fail(M2C_ERR_INVALID_ARG, "table_out, weight_out, len_out: all three or none");
  if (outs && (table_out == C.table || weight_out == C.weight || len_out == C.len))
    return api_fail(M2C_ERR_INVALID_ARG, "outputs that are the cache's own arrays: pass none");
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  return launched(m2c::launch_kv_evict(C, seqs, n, keep, first, recent, table_out, weight_out, len_out,
                                       (hipStream_t)stream), "evict");
}

m2c_status m2c_kv_status(const m2c_kv_cache* cache, void* stream) {
  KvView C;
  CHECKED(view_of(cache, &C));
  CurrentDevice g(cache->device);
  if (!g.ok) return api_fail(M2C_ERR_INVALID_ARG, "device %d is not usable", cache->device);
  int32_t bits = 0;
  hipError_t e = hipMemcpyAsync(&bits, C.status, 4, hipMemcpyDeviceToHost, (hipStream_t)stream);
  if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
  if (e == hipSuccess && bits) {
    e = hipMemsetAsync(C.status, 0, 4, (hipStream_t)stream);
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
  }
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return api_fail(M2C_ERR_HIP, "cache status: %s", hipGetErrorString(e));
  }
  if (bits & m2c::kKvBadIndex)
    return api_fail(M2C_ERR_INVALID_ARG, "a call used a sequence or page id out of range, or row starts that "
                    "do not ascend (status 0x%x)", bits);
  if (bits & m2c::kKvCapacity)
    return api_fail(M2C_ERR_CAPACITY, "an append would have passed max_blocks * block_tokens tokens; "
                    "the sequence was left as it was (status 0x%x)", bits);
  if (bits & m2c::kKvState)
    return api_fail(M2C_ERR_STATE, "an append's pos was neither the start of a block nor in the last "
                    "block; the sequence was left as it was (status 0x%x)", bits);
  return M2C_OK;
}

}  // extern "C"
