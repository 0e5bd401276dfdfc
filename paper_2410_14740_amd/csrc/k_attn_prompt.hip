// Attention over whole prompts: packed sequences, grouped heads, causal
// (bottom-right aligned) or not.
//
// Per query row, over the keys it sees, with c = scale * log2 e:
//   m = max c s_j,  p_j = 2^(c s_j - m),  l = sum p_j,  O = sum p_j v_j / l,
//   lse = (m + log2 l) ln 2,  in one pass over tiles of 64 keys: when a tile
// raises m, the l and O so far are multiplied by 2^(m_old - m_new).
//
// Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, on
// 32x32x16 instructions: a lane's column is then one query row throughout, so
// that the softmax runs down registers (one exchange with the lane 32 away per
// tile), and the registers of S^T, rounded in pairs, are the second product's B
// operand as they lie: the 8 tokens a lane holds per step of 16 are
// {4h .. 4h + 3, 8 + 4h .. 8 + 4h + 3} of the 16, h = lane / 32, and V^T's A
// operand is read in that order (transposing LDS reads, 4 tokens each).
#include "attn_device.h"

namespace m2c {

struct PromptArgs {
  const uint8_t *q, *k, *v;
  uint8_t* out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int64_t total_q, total_k;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;  // bytes
  float c;     // scale * log2 e
  int n_seqs, n_heads, group, causal;
  int items;   // tiles of query rows over all sequences (find_item)
};

namespace {

constexpr int kTileK = 64;  // keys per tile

// Zeros for the rows of a tile that are no keys of the sequence (0 * what lies
// there in memory could be NaN).
__device__ const u32x4 zero_row[16] = {};

// 16 bytes per lane from global memory straight into LDS (lane i's land at
// dst + 16 i).
__device__ __forceinline__ void load_lds16(const uint8_t* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) void*)(src),
      (__attribute__((address_space(3))) void*)(dst), 16, 0, 0);
}

__device__ __forceinline__ u32x2 read_tr(const uint8_t* lds) {
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(lds)));
}

// Tiles lie in LDS as [64][D] 16-bit rows, the 16-byte chunks of a row permuted
// by an xor so that the rows a read takes at once fall on different banks (a
// row of 128 elements spans all 64 banks, one of 64 elements half of them).
template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) {
  return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1;
}

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// The rows of one wave again, key by key, each row over the keys it sees only:
// taken where a value that some of the rows must not see is an infinity or a
// NaN, which a product with p = 0 would carry into them.
template <bool BF, int D>
__device__ __noinline__ void wave_rows_plain(const PromptArgs& A, const uint8_t* qb, const uint8_t* kb,
                                             const uint8_t* vb, uint8_t* ob, float* lse, int r0,
                                             int ql, int kl) {
  const int lane = threadIdx.x & 63;
  constexpr int E = D / 64;
  for (int r = r0; r < r0 + 32 && r < ql; ++r) {
    const int seen = min(kl, max(0, A.causal ? kl - ql + r + 1 : kl));
    float q[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = unpack16<BF>(*(const uint16_t*)(qb + r * A.q_tok + (lane + 64 * e) * 2));
      o[e] = 0.0f;
    }
    for (int j = 0; j < seen; ++j) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e)
        s += q[e] * unpack16<BF>(*(const uint16_t*)(kb + j * A.k_tok + (lane + 64 * e) * 2));
      s = wave_add(s) * A.c;
      const float mn = fmaxf(m, s), mu = mn == -INFINITY ? 0.0f : mn;
      const float a = exp2_fast(m - mu), p = exp2_fast(s - mu);
      l = l * a + p;
#pragma unroll
      for (int e = 0; e < E; ++e)
        o[e] = o[e] * a + p * unpack16<BF>(*(const uint16_t*)(vb + j * A.v_tok + (lane + 64 * e) * 2));
      m = mn;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e)
      *(uint16_t*)(ob + r * A.o_tok + (lane + 64 * e) * 2) = (uint16_t)pack16<BF>(o[e] * inv, 0.0f);
    if (lse && lane == 0)
      lse[(int64_t)r * A.n_heads] = (m + log2_fast(l)) * kLn2;
  }
}

template <bool BF, int D, int NW>
__global__ void __launch_bounds__(NW * 64, 2) prompt_attention_kernel(const PromptArgs A) {
  constexpr int kRows = NW * 32;           // query rows per workgroup
  constexpr int kRowBytes = D * 2, kChunks = D / 8;
  constexpr int kTileBytes = kTileK * kRowBytes;
  constexpr int kLoads = kTileBytes / (NW * 1024);  // per wave, for K and for V
  constexpr int kLoadRows = 1024 / kRowBytes;       // rows one load of a wave covers
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __align__(1024) uint8_t lds[2][2][kTileBytes];

  // The items of one key/value head follow each other and go to one XCD
  // (consecutive workgroups go round the eight), so that its L2 serves the
  // head's keys and values to all of them.
  const int G = A.group, per_kv = A.items * G, total = per_kv * (A.n_heads / G);
  const int per_xcd = (total + 7) / 8;
  const int item = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (item >= total) return;
  const int kvh = item / per_kv, in_kv = item - kvh * per_kv;
  const int x = in_kv / G, head = kvh * G + (in_kv - x * G);
  const int b = find_item(A.cu_q, A.n_seqs, A.total_q, x, kRows, 1);
  if (b < 0) return;
  const int64_t q_lo = clamp64(A.cu_q[b], 0, A.total_q), q_hi = clamp64(A.cu_q[b + 1], q_lo, A.total_q);
  const int64_t k_lo = clamp64(A.cu_k[b], 0, A.total_k), k_hi = clamp64(A.cu_k[b + 1], k_lo, A.total_k);
  const int ql = (int)(q_hi - q_lo), kl = (int)(k_hi - k_lo);
  const int n_tiles = (ql + kRows - 1) / kRows;
  const int j = x - (int)item_start(q_lo, b, kRows, 1);
  if (j >= n_tiles) return;
  const int qt = A.causal ? n_tiles - 1 - j : j;  // longest rows first

  const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint8_t* qb = A.q + q_lo * A.q_tok + head * A.q_head;
  const uint8_t* kb = A.k + k_lo * A.k_tok + kvh * A.k_head;
  const uint8_t* vb = A.v + k_lo * A.v_tok + kvh * A.v_head;
  uint8_t* ob = A.out + q_lo * A.o_tok + head * A.o_head;
  float* lse = A.lse ? A.lse + q_lo * A.n_heads + head : nullptr;

  const int r0 = qt * kRows + wave * 32;  // the wave's first row
  const int row = r0 + col;               // the lane's
  // keys the workgroup, the wave's first and last row, and the lane's row see
  const int off = kl - ql;
  const int wg_seen = A.causal ? min(kl, max(0, off + min(ql, (qt + 1) * kRows))) : kl;
  const int wv_lo = A.causal ? min(kl, max(0, off + r0 + 1)) : kl;
  const int wv_hi = r0 >= ql ? 0 : A.causal ? min(kl, max(0, off + min(ql, r0 + 32))) : kl;
  const int seen = A.causal ? min(kl, max(0, off + row + 1)) : kl;
  const int nt = (wg_seen + kTileK - 1) / kTileK;

  // global -> LDS: load i of a wave takes rows (i NW + wave) kLoadRows .. of a tile
  const int ld_row = wave * kLoadRows + lane / kChunks;
  const int ld_ck = ((lane % kChunks) ^ swz_k<D>(ld_row)) * 16;
  const int ld_cv = ((lane % kChunks) ^ swz_v<D>(ld_row)) * 16;
  auto load_tile = [&](int t, int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = t * kTileK + i * NW * kLoadRows + ld_row;
      const bool in = r < kl;
      const uint8_t* ks = in ? kb + r * A.k_tok + ld_ck : (const uint8_t*)zero_row;
      const uint8_t* vs = in ? vb + r * A.v_tok + ld_cv : (const uint8_t*)zero_row;
      load_lds16(ks, &lds[buf][0][(i * NW + wave) * 1024]);
      load_lds16(vs, &lds[buf][1][(i * NW + wave) * 1024]);
    }
  };

  u32x4 qf[KS];
  {
    const uint8_t* qr = qb + (int64_t)min(row, ql - 1) * A.q_tok + h * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const u32x4*)(qr + s * 32);
  }

  // LDS read addresses: K row = token col (+ 32), V rows = tokens 4h + i / 4
  // of a 16-lane group, 16 dimensions from 16 (group & 1)
  const int k_base = col * kRowBytes, k_x = swz_k<D>(col);
  const int vr = 4 * h + ((lane & 15) >> 2);
  int v_addr[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const int ch = dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    v_addr[dt] = vr * kRowBytes + (ch ^ swz_v<D>(vr)) * 16 + (lane & 1) * 8;
  }

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  uint32_t worst = 0;  // largest |value| bits seen in masked tiles, per half word
  bool bad = false;

  if (nt > 0) load_tile(0, 0);
  for (int t = 0; t < nt; ++t) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < nt) load_tile(t + 1, (t + 1) & 1);
    const int k0 = t * kTileK;
    if (k0 < wv_hi) {
      const uint8_t* kt = lds[t & 1][0];
      const uint8_t* vt = lds[t & 1][1];
      f32x16 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int a = k_base + (((ks * 2 + h) ^ k_x) * 16);
        const u32x4 k_0 = *(const u32x4*)(kt + a);
        const u32x4 k_1 = *(const u32x4*)(kt + a + 32 * kRowBytes);
        s[0] = mfma32<BF>(k_0, qf[ks], s[0]);
        s[1] = mfma32<BF>(k_1, qf[ks], s[1]);
      }
      const bool masked = k0 + kTileK > wv_lo;  // some row of the wave misses some key
      if (masked) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (k0 + 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= seen) s[i][r] = -INFINITY;
      }
      float mt = s[0][0];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[i][r]);
      mt = max_xor32(mt) * A.c;  // c > 0
      const float mn = fmaxf(m, mt), mu = mn == -INFINITY ? 0.0f : mn;
      const float alpha = exp2_fast(m - mu);
      m = mn;
      const float base = mu - kLift;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[i][r] = exp2_fast(fmaf(s[i][r], A.c, -base));
          sum += s[i][r];
        }
      l = l * alpha + sum;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        u32x4 p;
#pragma unroll
        for (int w = 0; w < 4; ++w)
          p[w] = pack16<BF>(s[u / 2][(u & 1) * 8 + 2 * w], s[u / 2][(u & 1) * 8 + 2 * w + 1]);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const u32x2 lo = read_tr(vt + v_addr[dt] + (16 * u) * kRowBytes);
          const u32x2 hi = read_tr(vt + v_addr[dt] + (16 * u + 8) * kRowBytes);
          const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
          if (masked) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              typedef unsigned short us2 __attribute__((ext_vector_type(2)));
              worst = __builtin_bit_cast(
                  uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, worst),
                                                      __builtin_bit_cast(us2, vf[w] & 0x7fff7fffu)));
            }
          }
          o[dt] = mfma32<BF>(vf, p, o[dt]);
        }
      }
      if (masked) {
        constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
        bad = bad || __ballot((worst & 0xffffu) >= kInf || (worst >> 16) >= kInf) != 0;
      }
    }
  }
  if (r0 >= ql) return;
  if (bad && A.causal) {
    wave_rows_plain<BF, D>(A, qb, kb, vb, ob, lse, r0, ql, kl);
    return;
  }
  if (row >= ql) return;
  l = add_xor32(l);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint8_t* orow = ob + (int64_t)row * A.o_tok + h * 8;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x2 w;
      w[0] = pack16<BF>(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv);
      w[1] = pack16<BF>(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv);
      *(u32x2*)(orow + dt * 64 + i * 16) = w;
    }
  if (lse && h == 0) lse[(int64_t)row * A.n_heads] = (m - kLift + log2_fast(l)) * kLn2;
}

template <bool BF, int D, int NW>
hipError_t launch_tile(PromptArgs& A, hipStream_t stream) {
  const int64_t items = A.total_q / (NW * 32) + A.n_seqs;
  const int64_t grid = (items * A.n_heads + 7) / 8 * 8;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  A.items = (int)items;
  hipLaunchKernelGGL((prompt_attention_kernel<BF, D, NW>), dim3((uint32_t)grid), dim3(NW * 64), 0,
                     stream, A);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(const m2c_attn_desc* D, const void* q, const void* k,
                                   const void* v, const int32_t* cu_q, const int32_t* cu_k,
                                   int n_seqs, int64_t total_q, int64_t total_k, void* out,
                                   float* lse, hipStream_t stream) {
  PromptArgs A;
  A.q = (const uint8_t*)q;
  A.k = (const uint8_t*)k;
  A.v = (const uint8_t*)v;
  A.out = (uint8_t*)out;
  A.lse = lse;
  A.cu_q = cu_q;
  A.cu_k = cu_k;
  A.total_q = total_q;
  A.total_k = total_k;
  A.q_tok = D->q_stride[0] * 2, A.q_head = D->q_stride[1] * 2;
  A.k_tok = D->k_stride[0] * 2, A.k_head = D->k_stride[1] * 2;
  A.v_tok = D->v_stride[0] * 2, A.v_head = D->v_stride[1] * 2;
  A.o_tok = D->out_stride[0] * 2, A.o_head = D->out_stride[1] * 2;
  A.c = (D->scale > 0.0f ? D->scale : 1.0f / sqrtf((float)D->head_dim)) * kLog2e;
  A.n_seqs = n_seqs;
  A.n_heads = D->n_heads;
  A.group = D->n_heads / D->n_kv_heads;
  A.causal = D->causal;
  if (D->dtype == M2C_DTYPE_BF16)
    return D->head_dim == 128 ? launch_tile<true, 128, 4>(A, stream) : launch_tile<true, 64, 4>(A, stream);
  return D->head_dim == 128 ? launch_tile<false, 128, 4>(A, stream) : launch_tile<false, 64, 4>(A, stream);
}

}  // namespace m2c
