// Key/value cache: append, read back, reset. Memory-bound movers: a workgroup
// takes one block of tokens of one key/value head, keys and values.
#include "kv_device.h"

namespace m2c {

namespace {

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// Larger of two pairs of magnitudes (16-bit patterns without the sign order
// like the magnitudes, with infinities above every number and NaN above them).
__device__ __forceinline__ uint32_t max_mag(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a),
                                                                __builtin_bit_cast(us2, b)));
}

// code = clamp(rne(x / s), -127, 127) with the fp32 quotient; 0 where the scale
// is 0 or not finite.
__device__ __forceinline__ uint32_t code8(float x, float s) {
  const float r = fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.0f), 127.0f);
  return (uint32_t)(int)r & 0xffu;
}

template <bool BF>
__device__ __forceinline__ u32x2 codes_of(u32x4 x, float s, bool any) {
  u32x2 c = {0, 0};
  if (any) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t a = code8(unpack16<BF>(x[w] & 0xffffu), s), b = code8(unpack16<BF>(x[w] >> 16), s);
      c[w / 2] |= (a | b << 8) << (16 * (w & 1));
    }
  }
  return c;
}

// One block of one sequence and key/value head. Thread t holds chunk t % (D/8)
// of tokens t / (D/8), + 256 / (D/8), ..
template <bool BF, int D, int BT>
__global__ void __launch_bounds__(256) append_kernel(const KvView C, const int32_t* seqs, int n,
                                                     const int32_t* cu, int64_t total,
                                                     const int32_t* pos, const uint8_t* k,
                                                     const uint8_t* v, int64_t k_tok, int64_t k_head,
                                                     int64_t v_tok, int64_t v_head) {
  constexpr int CH = D / 8, TP = 256 / CH;  // chunks of a token, tokens a pass of 256 threads takes
  constexpr int NP = BT / TP;
  __shared__ uint32_t mags[2][4];
  const int x = blockIdx.x / C.n_kv_heads, head = blockIdx.x - x * C.n_kv_heads, tid = threadIdx.x;
  int b = x, item = 0, items = 1;
  int64_t row0 = b;
  int nb = 1;
  if (cu) {
    b = find_item(cu, n, total, x, BT, 2);
    if (b < 0) return;
    row0 = clamp64(cu[b], 0, total);
    const int64_t row1 = clamp64(cu[b + 1], row0, total);
    nb = (int)(row1 - row0);
    const int64_t s0 = item_start(row0, b, BT, 2);
    item = (int)(x - s0);
    items = (int)(item_start(row1, b + 1, BT, 2) - s0);
    if (item >= items) return;  // past the last sequence's
  }
  if (nb == 0) return;  // nothing of this sequence changes
  const int s = seqs ? seqs[b] : b;
  if (s < 0 || s >= C.n_seqs) {
    if (tid == 0) atomicOr(C.status, kKvBadIndex);
    return;
  }
  const int len = C.len[s];
  const int p0 = pos ? pos[b] : len;
  const bool placed = p0 >= 0 && p0 <= len && (p0 % BT == 0 || p0 / BT == (len - 1) / BT);
  const bool fits = (int64_t)p0 + nb <= (int64_t)C.max_blocks * BT;
  const int end = p0 + nb;
  if (placed && fits) {
    const int first = p0 / BT, last = (end - 1) / BT;
    const int64_t sh = (int64_t)s * C.n_kv_heads + head;
    uint8_t* tk = C.tail_k + sh * BT * (D * 2);
    uint8_t* tv = C.tail_v + sh * BT * (D * 2);
    const uint8_t* kr = k + row0 * k_tok + head * k_head;
    const uint8_t* vr = v + row0 * v_tok + head * v_head;
    const int ch = tid % CH, t0 = tid / CH;
    // Item 0 takes the first block, which may begin in the tail, and then
    // writes the tail of the last block; the others never touch the tail.
    for (int blk = first + item; blk <= last; blk += items) {
      const int at = blk * BT;  // first token of the block
      if (tid == 0 && at >= p0) C.weight[sh * C.max_blocks + blk] = 0.0f;
      if (at + BT > end) continue;  // stays open
      u32x4 xk[NP], xv[NP];
      uint32_t mk = 0, mv = 0;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int t = t0 + i * TP;
        const bool old = at + t < p0;
        const int64_t r = at + t - p0;
        xk[i] = *(const u32x4*)((old ? tk + t * (D * 2) : kr + r * k_tok) + ch * 16);
        xv[i] = *(const u32x4*)((old ? tv + t * (D * 2) : vr + r * v_tok) + ch * 16);
      }
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          mk = max_mag(mk, xk[i][w] & 0x7fff7fffu);
          mv = max_mag(mv, xv[i][w] & 0x7fff7fffu);
        }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        mk = max_mag(mk, __shfl_xor(mk, o));
        mv = max_mag(mv, __shfl_xor(mv, o));
      }
      __syncthreads();  // the last block's magnitudes are read
      if ((tid & 63) == 0) {
        mags[0][tid >> 6] = mk;
        mags[1][tid >> 6] = mv;
      }
      __syncthreads();
      mk = max_mag(max_mag(mags[0][0], mags[0][1]), max_mag(mags[0][2], mags[0][3]));
      mv = max_mag(max_mag(mags[1][0], mags[1][1]), max_mag(mags[1][2], mags[1][3]));
      const float sk = __fdiv_rn(unpack16<BF>(max(mk & 0xffffu, mk >> 16)), 127.0f);
      const float sv = __fdiv_rn(unpack16<BF>(max(mv & 0xffffu, mv >> 16)), 127.0f);
      const int page = C.table[sh * C.max_blocks + blk];
      if (page < 0 || page >= C.n_pages) {
        if (tid == 0) atomicOr(C.status, kKvBadIndex);
        continue;
      }
      const bool ak = sk > 0.0f && sk < INFINITY, av = sv > 0.0f && sv < INFINITY;
      int8_t* ck = C.k_codes + (int64_t)page * (BT * D);
      int8_t* cv = C.v_codes + (int64_t)page * (BT * D);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int t = t0 + i * TP;
        *(u32x2*)(ck + t * D + ch * 8) = codes_of<BF>(xk[i], sk, ak);
        *(u32x2*)(cv + t * D + ch * 8) = codes_of<BF>(xv[i], sv, av);
      }
      if (tid == 0) {
        C.k_scale[page] = sk;
        C.v_scale[page] = sv;
      }
    }
    if (item == 0) {
      __syncthreads();  // the first block's old tokens are in registers
      const int at = last * BT;
      for (int t = t0; t < BT; t += TP) {
        if (at + t < p0 || at + t >= end) continue;
        const int64_t r = at + t - p0;
        *(u32x4*)(tk + t * (D * 2) + ch * 16) = *(const u32x4*)(kr + r * k_tok + ch * 16);
        *(u32x4*)(tv + t * (D * 2) + ch * 16) = *(const u32x4*)(vr + r * v_tok + ch * 16);
      }
    }
  }
  // Every thread of every workgroup of the sequence has read the length before
  // the workgroup arrives; the last one to arrive writes the new one.
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(&C.arrive[s], 1) == items * C.n_kv_heads - 1) {
      C.arrive[s] = 0;
      if (placed && fits) C.len[s] = end;
      else atomicOr(C.status, placed ? kKvCapacity : kKvState);
    }
  }
}

template <bool BF, int D, int BT>
__global__ void __launch_bounds__(256) read_kernel(const KvView C, const int32_t* seqs, int n,
                                                   const int32_t* cu, int64_t total, uint8_t* k,
                                                   uint8_t* v, int64_t k_tok, int64_t k_head,
                                                   int64_t v_tok, int64_t v_head) {
  constexpr int CH = D / 8, TP = 256 / CH;
  constexpr int NP = BT / TP;
  const int x = blockIdx.x / C.n_kv_heads, head = blockIdx.x - x * C.n_kv_heads, tid = threadIdx.x;
  const int b = find_item(cu, n, total, x, BT, 1);
  if (b < 0) return;
  const int64_t row0 = clamp64(cu[b], 0, total), row1 = clamp64(cu[b + 1], row0, total);
  const int blk = (int)(x - item_start(row0, b, BT, 1));
  const int s = seqs ? seqs[b] : b;
  if (s < 0 || s >= C.n_seqs) {
    if (tid == 0) atomicOr(C.status, kKvBadIndex);
    return;
  }
  const int64_t cap = (int64_t)C.max_blocks * BT;
  const int len = (int)clamp64(C.len[s], 0, cap);
  const int count = (int)(row1 - row0 < len ? row1 - row0 : len);
  if (blk * BT >= count) return;
  const int64_t sh = (int64_t)s * C.n_kv_heads + head;
  const int ch = tid % CH, t0 = tid / CH;
  uint8_t* kr = k + (row0 + blk * BT) * k_tok + head * k_head + ch * 16;
  uint8_t* vr = v + (row0 + blk * BT) * v_tok + head * v_head + ch * 16;
  const int upto = min(BT, count - blk * BT);
  if ((blk + 1) * BT > len) {  // the open block
    const uint8_t* tk = C.tail_k + sh * BT * (D * 2) + ch * 16;
    const uint8_t* tv = C.tail_v + sh * BT * (D * 2) + ch * 16;
    for (int t = t0; t < upto; t += TP) {
      *(u32x4*)(kr + t * k_tok) = *(const u32x4*)(tk + t * (D * 2));
      *(u32x4*)(vr + t * v_tok) = *(const u32x4*)(tv + t * (D * 2));
    }
    return;
  }
  const int page = C.table[sh * C.max_blocks + blk];
  if (page < 0 || page >= C.n_pages) {
    if (tid == 0) atomicOr(C.status, kKvBadIndex);
    for (int t = t0; t < upto; t += TP) *(u32x4*)(kr + t * k_tok) = *(u32x4*)(vr + t * v_tok) = u32x4{0, 0, 0, 0};
    return;
  }
  const float sk = C.k_scale[page], sv = C.v_scale[page];
  const int8_t* ck = C.k_codes + (int64_t)page * (BT * D) + ch * 8;
  const int8_t* cv = C.v_codes + (int64_t)page * (BT * D) + ch * 8;
  auto value = [](u32x2 c, float sc) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = c[i / 2] >> (16 * (i & 1));
      w[i] = pack16<BF>((float)(int8_t)(two & 0xff) * sc, (float)(int8_t)(two >> 8 & 0xff) * sc);
    }
    return w;
  };
  u32x2 qk[NP], qv[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = t0 + i * TP;
    qk[i] = *(const u32x2*)(ck + t * D);
    qv[i] = *(const u32x2*)(cv + t * D);
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = t0 + i * TP;
    if (t >= upto) continue;
    *(u32x4*)(kr + t * k_tok) = value(qk[i], sk);
    *(u32x4*)(vr + t * v_tok) = value(qv[i], sv);
  }
}

__global__ void reset_kernel(int32_t* len, int32_t* status, const int32_t* seqs, int n, int n_seqs) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int s = seqs ? seqs[i] : i;
  if (s >= 0 && s < n_seqs) len[s] = 0;
  else atomicOr(status, kKvBadIndex);
}

template <typename F>
hipError_t by_shape(const KvView& C, F f) {
  const auto by_block = [&](auto bf, auto d) {
    switch (C.block_tokens) {
      case 32: return f(bf, d, std::integral_constant<int, 32>());
      case 64: return f(bf, d, std::integral_constant<int, 64>());
      default: return f(bf, d, std::integral_constant<int, 128>());
    }
  };
  const auto by_dim = [&](auto bf) {
    return C.head_dim == 128 ? by_block(bf, std::integral_constant<int, 128>())
                             : by_block(bf, std::integral_constant<int, 64>());
  };
  return C.bf ? by_dim(std::true_type()) : by_dim(std::false_type());
}

}  // namespace

hipError_t launch_kv_append(const KvView& C, const int32_t* seqs, int n, const int32_t* cu,
                            int64_t total, const int32_t* pos, const void* k, const void* v,
                            const int64_t* ks, const int64_t* vs, hipStream_t stream) {
  const int64_t items = cu ? total / C.block_tokens + 2 * (int64_t)n : n;
  if (items * C.n_kv_heads > INT32_MAX) return hipErrorInvalidValue;
  return by_shape(C, [&](auto bf, auto d, auto bt) {
    hipLaunchKernelGGL((append_kernel<decltype(bf)::value, decltype(d)::value, decltype(bt)::value>),
                       dim3((uint32_t)(items * C.n_kv_heads)), dim3(256), 0, stream, C, seqs, n, cu,
                       total, pos, (const uint8_t*)k, (const uint8_t*)v, ks[0] * 2, ks[1] * 2,
                       vs[0] * 2, vs[1] * 2);
    return hipGetLastError();
  });
}

hipError_t launch_kv_read(const KvView& C, const int32_t* seqs, int n, const int32_t* cu,
                          int64_t total, void* k, void* v, const int64_t* ks, const int64_t* vs,
                          hipStream_t stream) {
  const int64_t items = total / C.block_tokens + n;
  if (items * C.n_kv_heads > INT32_MAX) return hipErrorInvalidValue;
  return by_shape(C, [&](auto bf, auto d, auto bt) {
    hipLaunchKernelGGL((read_kernel<decltype(bf)::value, decltype(d)::value, decltype(bt)::value>),
                       dim3((uint32_t)(items * C.n_kv_heads)), dim3(256), 0, stream, C, seqs, n, cu,
                       total, (uint8_t*)k, (uint8_t*)v, ks[0] * 2, ks[1] * 2, vs[0] * 2, vs[1] * 2);
    return hipGetLastError();
  });
}

hipError_t launch_kv_reset(const KvView& C, const int32_t* seqs, int n, hipStream_t stream) {
  hipLaunchKernelGGL(reset_kernel, dim3((n + 255) / 256), dim3(256), 0, stream, C.len, C.status,
                     seqs, n, C.n_seqs);
  return hipGetLastError();
}

}  // namespace m2c
