// Eviction of the cache's blocks by accumulated attention weight: per sequence
// and key/value head a selection of the heaviest blocks (ties to the lowest
// index) and one ordered move of the head's table and weight rows. 16 bytes per
// table entry and no page data: latency-bound, one workgroup per row with the
// row in registers. Measured: 256 rows of 34 entries 4.0 us, of 2049 entries
// 8.2 us (8.4 MB), a third of it four passes of a histogram with three barriers
// each. (The first pass's adds made one per digit and wave by ballots: 9.3 us.)
#include "kv_device.h"
#include "wave_ops.h"

namespace m2c {

namespace {

// Prefix of v over the workgroup's NT threads in thread order, *total the sum.
// tmp: NT / 64 words that nothing else uses until the next barrier after this.
template <int NT>
__device__ __forceinline__ uint32_t excl_scan(uint32_t v, uint32_t* tmp, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t incl = wave_incl_scan(v);
  if (lane == 63) tmp[wave] = incl;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w == wave) before = sum;
    sum += tmp[w];
  }
  *total = sum;
  return before + incl - v;
}

// Entry e of the row is held by thread e % NT as its e / NT-th.
template <int NT, int J>
__global__ void __launch_bounds__(NT) evict_kernel(const KvView C, const int32_t* seqs, int keep,
                                                   int first, int recent, int32_t* table_out,
                                                   float* weight_out, int32_t* len_out) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t tmp[3][NT / 64];
  const int b = blockIdx.x / C.n_kv_heads, head = blockIdx.x - b * C.n_kv_heads, tid = threadIdx.x;
  const int s = seqs ? seqs[b] : b;
  if (s < 0 || s >= C.n_seqs) {
    if (tid == 0) atomicOr(C.status, kKvBadIndex);
    return;
  }
  const int MB = C.max_blocks, BT = C.block_tokens;
  const int len = (int)clamp64(C.len[s], 0, (int64_t)MB * BT);
  const int m = len > 0 ? (len - 1) / BT : 0;  // blocks before the last one
  const int gone = m > keep ? m - keep : 0;
  const bool inplace = table_out == nullptr;
  if (gone == 0 && inplace) return;
  const int64_t row = ((int64_t)s * C.n_kv_heads + head) * MB;
  int32_t page[J];
  float w[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int e = j * NT + tid;
    page[j] = e < MB ? C.table[row + e] : 0;
    w[j] = e < MB ? C.weight[row + e] : 0.0f;
  }
  int32_t* to = (inplace ? C.table : table_out) + row;
  float* wo = (inplace ? C.weight : weight_out) + row;
  if (gone == 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = j * NT + tid;
      if (e < MB) to[e] = page[j], wo[e] = w[j];
    }
    if (head == 0 && tid == 0) len_out[s] = C.len[s];
    return;
  }

  // The key of the last block to be chosen by weight, and how many of the
  // blocks with that key are (the lowest indices): four digits of 8 bits.
  const int lo = first, hi = m - recent;  // the blocks that compete
  uint32_t key = 0;
  int need = keep - first - recent;
  bool all_ties = false;  // every block with that key is chosen
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += NT) hist[i] = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int e = j * NT + tid;
        const uint32_t k = score_key(w[j]);
        if (e >= lo && e < hi && (shift == 24 || k >> ((shift + 8) & 31) == key))
          atomicAdd(&hist[k >> shift & 255], 1u);
      }
      __syncthreads();
      // lane l sums the digits 255 - 4 l .. 252 - 4 l, the largest first
      const int l = tid & 63;
      uint32_t d[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = hist[255 - 4 * l - i];
      const uint32_t sum = d[0] + d[1] + d[2] + d[3], incl = wave_incl_scan(sum);
      const int at = __ffsll((unsigned long long)__ballot(incl >= (uint32_t)need)) - 1;
      uint32_t above = incl - sum;
      int digit = 255 - 4 * l;
      uint32_t count = d[0];
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (above + d[i] < (uint32_t)need && digit == 255 - 4 * l - i) above += d[i], --digit, count = d[i + 1];
      key = key << 8 | (uint32_t)__builtin_amdgcn_readlane(digit, at);
      need -= (int)__builtin_amdgcn_readlane((int)above, at);
      all_ties = (int)__builtin_amdgcn_readlane((int)count, at) == need;
      __syncthreads();
    }
  }
  const bool by_weight = keep - first - recent > 0;
  uint32_t ties = 0, kept_before = 0, gone_before = 0;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (j * NT >= MB) break;
    const int e = j * NT + tid;
    const uint32_t k = score_key(w[j]);
    const bool mid = e >= lo && e < hi;
    const bool tie = mid && by_weight && k == key;
    uint32_t total, rank = 0;
    if (!all_ties) {
      rank = ties + excl_scan<NT>(tie, tmp[2], &total);
      ties += total;
    }
    const bool kept = e < m && (!mid || (by_weight && (k > key || (tie && rank < (uint32_t)need))));
    const bool out = e < m && !kept;
    const uint32_t r = excl_scan<NT>((kept ? 1u : 0u) | (out ? 0x10000u : 0u), tmp[j & 1], &total);
    const int at = kept ? (int)(kept_before + (r & 0xffffu))
                   : out ? MB - gone + (int)(gone_before + (r >> 16)) : e - gone;
    kept_before += total & 0xffffu;
    gone_before += total >> 16;
    if (e < MB) {  // every entry was read before the first barrier
      to[at] = page[j];
      wo[at] = out ? 0.0f : w[j];
    }
  }
  if (!inplace) {
    if (head == 0 && tid == 0) len_out[s] = len - gone * BT;
  } else if (tid == 0) {
    // the last head's workgroup to get here writes the length that all have read
    if (atomicAdd(&C.arrive[s], 1) == C.n_kv_heads - 1) {
      C.arrive[s] = 0;
      C.len[s] = len - gone * BT;
    }
  }
}

}  // namespace

hipError_t launch_kv_evict(const KvView& C, const int32_t* seqs, int n, int keep, int first,
                           int recent, int32_t* table_out, float* weight_out, int32_t* len_out,
                           hipStream_t stream) {
  const dim3 grid((uint32_t)(n * C.n_kv_heads));
#define M2C_EVICT(NT, J)                                                                      \
  hipLaunchKernelGGL((evict_kernel<NT, J>), grid, dim3(NT), 0, stream, C, seqs, keep, first, \
                     recent, table_out, weight_out, len_out)
  if (C.max_blocks <= 256) M2C_EVICT(256, 1);
  else if (C.max_blocks <= 1024) M2C_EVICT(1024, 1);
  else if (C.max_blocks <= 4096) M2C_EVICT(1024, 4);
  else M2C_EVICT(1024, 16);
#undef M2C_EVICT
  return hipGetLastError();
}

}  // namespace m2c
