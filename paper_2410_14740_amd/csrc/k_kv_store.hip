// Key/value cache: append, read back, reset. Movers, bound by memory: a
// workgroup takes one block of tokens of one key/value head, keys and values,
// with the whole block in registers between the search for its largest
// magnitude and the codes. Measured, 61344 tokens of 8 heads of 128 in bf16:
// append 73 us and read 65 us, each 377 MB (5.2 and 5.8 TB/s; a 1 GiB copy:
// 5.1). One token for each of 8 sequences of 32 heads: 5 to 7 us, a chain of
// dependent loads (length, tail, table) and the arrivals at the length.
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

// Codes of a chunk of 8 elements: rne of the correctly rounded fp32 quotient x /
// s, as two words. With r the rounded 1 / s, q = x r and one correction by the
// exact remainder give that quotient (three operations instead of a division's
// dozen, which would take longer than the memory); the tests compare every pair
// of fp16 and of bf16 significands. Adding 1.5 2^23 rounds it to an integer, ties
// to even, in the low byte. |x| <= 127 s (1 + 2^-23) for a normal s, so nothing
// has to be clamped.
template <bool BF>
__device__ __forceinline__ u32x2 codes_of(u32x4 x, float s, float r) {
  uint32_t t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = unpack16<BF>(i & 1 ? x[i / 2] >> 16 : x[i / 2] & 0xffffu);
    const float q = v * r;
    t[i] = __float_as_uint(fmaf(fmaf(-q, s, v), r, q) + 12582912.0f);
  }
  u32x2 c;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    c[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0c0c0400u), 0x05040100u);
  return c;
}

// The same by a division, for scales whose reciprocal is not a normal number
// (bf16 blocks below 2^-93 or above 2^107). A subnormal s is 2^-133 / 127, 516 of
// the smallest fp32 number, or more, so |x| <= 127 s (1 + 2^-10): still 127.
template <bool BF>
__device__ __forceinline__ u32x2 codes_divided(u32x4 x, float s) {
  u32x2 c = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = unpack16<BF>(i & 1 ? x[i / 2] >> 16 : x[i / 2] & 0xffffu);
    const uint32_t t = __float_as_uint(__fdiv_rn(v, s) + 12582912.0f) & 0xffu;
    c[i / 4] |= t << (8 * (i & 3));
  }
  return c;
}

// A thread's chunks of a block (see append_kernel) as codes. A block without a
// magnitude, or with one that is not finite, has codes 0.
template <bool BF, int D, int BT>
__device__ __forceinline__ void store_codes(int8_t* page, const u32x4 (&x)[BT * D / 2048], float s) {
  u32x2* to = (u32x2*)page + threadIdx.x;
  const bool normal = s >= 0x1p-100f && s <= 0x1p100f;
  const float r = __fdiv_rn(1.0f, s);
  if (normal) {
#pragma unroll
    for (int i = 0; i < BT * D / 2048; ++i) to[i * 256] = codes_of<BF>(x[i], s, r);
  } else {
    const bool any = s > 0.0f && s < INFINITY;
#pragma unroll
    for (int i = 0; i < BT * D / 2048; ++i) to[i * 256] = any ? codes_divided<BF>(x[i], s) : u32x2{0, 0};
  }
}

// Where an append of nb tokens goes: from p0 to end, if that is a place of the
// sequence (the start of a block, or in the last block) and it fits.
struct Place {
  int p0, end;
  bool placed, fits;
};

__device__ __forceinline__ Place place_of(const KvView& C, int s, const int32_t* pos, int nb) {
  const int BT = C.block_tokens, len = C.len[s];
  Place p;
  p.p0 = pos ? *pos : len;
  p.placed = p.p0 >= 0 && p.p0 <= len && (p.p0 % BT == 0 || p.p0 / BT == (len - 1) / BT);
  p.fits = (int64_t)p.p0 + nb <= (int64_t)C.max_blocks * BT;
  p.end = p.fits ? p.p0 + nb : 0;
  return p;
}

__device__ __forceinline__ void set_length(const KvView& C, int s, bool placed, bool fits, int end) {
  if (placed && fits) C.len[s] = end;
  else atomicOr(C.status, placed ? kKvCapacity : kKvState);
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
    if (item < 0 || item >= items) return;  // past the last sequence's, or starts that do not ascend
  }
  if (nb == 0) return;  // nothing of this sequence changes
  const int s = seqs ? seqs[b] : b;
  if (s < 0 || s >= C.n_seqs) {
    if (tid == 0) atomicOr(C.status, kKvBadIndex);
    return;
  }
  const Place p = place_of(C, s, pos ? &pos[b] : nullptr, nb);
  const int p0 = p.p0, end = p.end;
  if (p.placed && p.fits) {
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
      const int page = C.table[sh * C.max_blocks + blk];
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
      if (page < 0 || page >= C.n_pages) {
        if (tid == 0) atomicOr(C.status, kKvBadIndex);
        continue;
      }
      store_codes<BF, D, BT>(C.k_codes + (int64_t)page * (BT * D), xk, sk);
      store_codes<BF, D, BT>(C.v_codes + (int64_t)page * (BT * D), xv, sv);
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
  // The new length is written when every workgroup of the sequence has read the
  // old one: with one token each, by the last of the heads' workgroups to
  // arrive; with many workgroups, whose arrivals at one counter would take
  // longer (25 ns each) than the memory, by a second launch.
  if (cu) return;
  __syncthreads();
  if (tid == 0 && atomicAdd(&C.arrive[s], 1) == C.n_kv_heads - 1) {
    C.arrive[s] = 0;
    set_length(C, s, p.placed, p.fits, p.end);
  }
}

__global__ void __launch_bounds__(256) length_kernel(const KvView C, const int32_t* seqs, int n,
                                                     const int32_t* cu, int64_t total,
                                                     const int32_t* pos) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= n) return;
  if (cu[b + 1] < cu[b]) atomicOr(C.status, kKvBadIndex);
  const int64_t row0 = clamp64(cu[b], 0, total);
  const int nb = (int)(clamp64(cu[b + 1], row0, total) - row0);
  const int s = seqs ? seqs[b] : b;
  if (nb == 0 || s < 0 || s >= C.n_seqs) return;
  const Place p = place_of(C, s, pos ? &pos[b] : nullptr, nb);
  set_length(C, s, p.placed, p.fits, p.end);
}

template <bool BF, int D, int BT>
__global__ void __launch_bounds__(256) read_kernel(const KvView C, const int32_t* seqs, int n,
                                                   const int32_t* cu, int64_t total, uint8_t* k,
                                                   uint8_t* v, int64_t k_tok, int64_t k_head,
                                                   int64_t v_tok, int64_t v_head) {
  constexpr int CH = D / 8, TP = 256 / CH;
  constexpr int NP = BT / TP;
  const int x = blockIdx.x / C.n_kv_heads, head = blockIdx.x - x * C.n_kv_heads, tid = threadIdx.x;
  // there are n workgroups or more
  if (tid == 0 && (int)blockIdx.x < n && cu[blockIdx.x + 1] < cu[blockIdx.x]) atomicOr(C.status, kKvBadIndex);
  const int b = find_item(cu, n, total, x, BT, 1);
  if (b < 0) return;
  const int64_t row0 = clamp64(cu[b], 0, total), row1 = clamp64(cu[b + 1], row0, total);
  const int blk = (int)(x - item_start(row0, b, BT, 1));
  if (blk < 0) return;  // starts that do not ascend
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
  const hipError_t e = by_shape(C, [&](auto bf, auto d, auto bt) {
    hipLaunchKernelGGL((append_kernel<decltype(bf)::value, decltype(d)::value, decltype(bt)::value>),
                       dim3((uint32_t)(items * C.n_kv_heads)), dim3(256), 0, stream, C, seqs, n, cu,
                       total, pos, (const uint8_t*)k, (const uint8_t*)v, ks[0] * 2, ks[1] * 2,
                       vs[0] * 2, vs[1] * 2);
    return hipGetLastError();
  });
  if (e != hipSuccess || !cu) return e;
  hipLaunchKernelGGL(length_kernel, dim3((n + 255) / 256), dim3(256), 0, stream, C, seqs, n, cu, total, pos);
  return hipGetLastError();
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
