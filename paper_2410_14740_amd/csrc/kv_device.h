// The key/value cache as its kernels see it.
#pragma once

#include <type_traits>

#include "rotary_device.h"

namespace m2c {

// Bits of the cache's status word, reported (and cleared) by m2c_kv_status.
constexpr int kKvBadIndex = 1;  // a sequence id or a live page id out of range, row starts that do not ascend
constexpr int kKvCapacity = 2;  // an append past max_blocks
constexpr int kKvState = 4;     // an append at a place that is no place of the sequence

struct KvView {
  int8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  uint8_t *tail_k, *tail_v;
  int32_t *table, *len;
  float* weight;
  int32_t *arrive, *status;
  int64_t n_pages;
  int32_t n_seqs, n_kv_heads, head_dim, block_tokens, max_blocks, bf;
};

hipError_t launch_kv_append(const KvView& C, const int32_t* seqs, int n, const int32_t* cu,
                            int64_t total, const int32_t* pos, const void* k, const void* v,
                            const int64_t* ks, const int64_t* vs, hipStream_t stream);
hipError_t launch_kv_append_rotated(const KvView& C, const TurnView& T, bool interleaved, const int32_t* seqs,
                                    int n, const int32_t* cu, int64_t total, const int32_t* pos, const void* k,
                                    const void* v, const int64_t* ks, const int64_t* vs, void* k_out,
                                    const int64_t* kos, const TurnRows& Q, hipStream_t stream);
hipError_t launch_kv_read(const KvView& C, const int32_t* seqs, int n, const int32_t* cu,
                          int64_t total, void* k, void* v, const int64_t* ks, const int64_t* vs,
                          hipStream_t stream);
hipError_t launch_kv_reset(const KvView& C, const int32_t* seqs, int n, hipStream_t stream);
int64_t kv_attend_workspace(const KvView& C, int n, int n_heads, int track, int max_len);
hipError_t launch_kv_attend(const KvView& C, const int32_t* seqs, int n, int n_heads, float scale,
                            const void* q, const int64_t* qs, void* out, const int64_t* os,
                            float* lse, int track, int max_len, void* workspace, hipStream_t stream);
int64_t kv_chunk_workspace(const KvView& C, int n, int n_heads, int64_t total, int max_q, int max_len);
hipError_t launch_kv_chunk(const KvView& C, const int32_t* seqs, int n, const int32_t* cu, int64_t total,
                           int n_heads, float scale, const void* q, const int64_t* qs, const void* k,
                           const int64_t* ks, const void* v, const int64_t* vs, void* out, const int64_t* os,
                           float* lse, int max_q, int max_len, void* workspace, hipStream_t stream);
hipError_t launch_kv_evict(const KvView& C, const int32_t* seqs, int n, int keep, int first,
                           int recent, int32_t* table_out, float* weight_out, int32_t* len_out,
                           hipStream_t stream);

}  // namespace m2c
