// Attention of one query token per sequence over the 8-bit key/value cache.
//
// Per query head over the tokens the sequence holds, in units of 2^: with
// c = scale * log2 e, x_t = c <q, code_t> s_k (s_k the block's key scale),
//   m = max x_t, p_t = 2^(x_t - m), l = sum p_t, O = sum_blocks s_v sum p_t code_t / l.
// Every code byte is read once, by one wave, for all query heads of its
// key/value head: bound by the bytes of the pages.
//
// Transposed products on 16x16x32 instructions: S^T = K Q^T (rows tokens,
// columns the up to 16 query heads of the group), O^T = V^T P^T. A lane's
// column is one query head, the softmax runs down registers and across the
// four lanes of a column, and S^T's registers, rounded in pairs, are the second
// product's B operand as they lie: a lane of quarter c = l / 16 holds tokens
// {4c .. 4c + 3, 16 + 4c .. 16 + 4c + 3} of each 32, and V's rows are loaded in
// that order. Codes become fp16 exactly; queries of bf16 caches are scaled by a
// power of two per head into fp16's range (exact but for elements 2^-24 of the
// head's largest). So both products sum exact products in fp32, p alone is
// rounded (relative 2^-11 in fp16; 2^-8 over the open block of a bf16 cache, whose
// values are bf16).
//
// The units of all rows (a row: a sequence, key/value head and tile of 16 query
// heads), one after another, are cut into even shares, one per workgroup of a
// grid that runs at once; the lengths are on the device, so each workgroup finds
// its share itself. A share may end inside a row: the parts of a row are joined
// by a second launch. Within a share the four waves take the units in turn, each
// with its own running m, l, O, joined through LDS. Short rows are a workgroup's
// each, which then adds the block weights too; rows between those, and calls with
// more sequences than a wave has lanes, are cut into chunks (see split_of).
//
// Measured (kernel times): 131071 tokens of 8 heads of 128 (268 MB) 42 us, 6.4
// TB/s with the Infinity Cache's share, and a join of 5; 32 sequences of 500 ..
// 23254 tokens (707 MB) 136 us, 5.2 TB/s, where a plain read of that size
// reaches 6.3; 8 sequences of up to 2048 tokens of 32 heads (69 MB) 17.4 us.
// Arithmetic takes a third of the cycles; a CU alone takes 45 GB/s of pages, with
// eight waves on a row or with fewer instructions too. Two waves per SIMD (a unit's codes,
// sums and queries take 190 registers); three by a smaller register budget
// spilled (191 us instead of 146), and codes through LDS in whole cache lines
// were no faster (145 instead of 138).
#include <algorithm>

#include "ffn_device.h"
#include "kv_device.h"
#include "wave_ops.h"

namespace m2c {

struct AttendArgs {
  KvView C;
  const int32_t* seqs;
  const uint8_t* q;
  uint8_t* out;
  float* lse;
  int64_t q_row, q_head, o_row, o_head;  // bytes
  float* part_o;    // [parts of rows][min(group, 16)][D] unnormalized outputs
  float2* part_ml;  // [parts of rows][min(group, 16)] their m and l
  float2* fin;      // [n][n_heads] m and 1 / l of whole rows (track)
  float2* wsum;     // [n][n_kv_heads][units of max_blocks][group] m and sum of p by unit (track)
  float c;
  int n, n_heads, group, tiles;  // tiles: head tiles of 16 per key/value head
  int splits, chunk;             // chunk: units per workgroup (where shares are not even)
  int whole_fin;                 // attend writes fin of the rows that it has whole
  int weigh_here;                // attend adds the block weights (a row is one workgroup's)
};

namespace {

constexpr int kWaves = 4;
constexpr int kMaxHeads = 1024;  // query heads of a key/value head

// Weights are taken as 2^(x - m + kLift), l and O alike: rounded to fp16 the
// largest is 2^14 and those down to 2^-28 of it keep all their bits (2^-14
// without the lift; a long sequence of small weights beside one large one would
// lose them). It cancels in O / l and is taken out of the log-sum-exp.
constexpr float kLift = 14.0f;

// p of a unit's tokens from its scores, and the running statistics. s: scores
// in units of 2^ (masked ones -infinity). Returns the factor for what was
// summed before; *unit_sum the lane's sum of p.
template <int T>
__device__ __forceinline__ float softmax_step(f32x4 (&s)[T], float& m, float& l, float* unit_sum) {
  float mt = s[0][0];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) mt = fmaxf(mt, s[t][r]);
  mt = max_xor16(max_xor32(mt));
  const float mn = fmaxf(m, mt), mu = mn == -INFINITY ? 0.0f : mn;
  const float alpha = exp2_fast(m - mu);
  m = mn;
  const float base = mu - kLift;
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] = exp2_fast(s[t][r] - base);
      sum += s[t][r];
    }
  l = l * alpha + sum;
  *unit_sum = sum;
  return alpha;
}

// 32 tokens' p as the B operand of the value product.
template <bool BF>
__device__ __forceinline__ u32x4 pack_p(const f32x4& a, const f32x4& b) {
  return u32x4{pack16<BF>(a[0], a[1]), pack16<BF>(a[2], a[3]), pack16<BF>(b[0], b[1]),
               pack16<BF>(b[2], b[3])};
}

// Byte i of two rows' words as a pair of fp16 (offset-binary codes, see
// i8x4_to_h2).
template <int I>
__device__ __forceinline__ uint32_t pair_of(uint32_t lo, uint32_t hi) {
  constexpr uint32_t sel = 0x0c000c00u | (uint32_t)I | (uint32_t)(4 + I) << 16;
  const uint32_t u = __builtin_amdgcn_perm(hi, lo, sel) | 0x64006400u;
  const half2v bias = {(_Float16)1152.0f, (_Float16)1152.0f};
  return __builtin_bit_cast(uint32_t, (half2v)(as_h2(u) - bias));
}

constexpr int kShares = 512;  // workgroups that run at once: two per CU

// What a row costs a workgroup beside its units, in units: queries, the first
// loads' latency, the waves' join. (32 heads, 8 ragged sequences of up to 16000
// tokens: 57 us with 1, 39 with 4, 36 with 8, 38 with 16.)
constexpr int kRowCost = 8;

// The even shares: lane b of a wave holds sequence b of the call, its rows'
// [start, start + cost * rows of a sequence) in the flat order, each row's
// kRowCost before its units.
struct Shares {
  int s, len;           // sequence id (-1: no such), tokens
  uint32_t cost, start; // cost of a row, the first in the flat order
  uint32_t total;
  int count;            // shares: share p is [p total / count, (p + 1) total / count)

  __device__ __forceinline__ uint32_t first_of(int p) const {
    return (uint32_t)((uint64_t)p * total / count);
  }
  __device__ __forceinline__ int owner_of(uint32_t f) const {
    return (int)((((uint64_t)f + 1) * count - 1) / total);
  }
};

__device__ __forceinline__ int units_of(int len, int BT, int unit) {
  return len / BT * (BT / unit) + (len % BT + unit - 1) / unit;
}

__device__ __forceinline__ Shares shares_of(const AttendArgs& A, int unit) {
  const KvView& C = A.C;
  const int lane = threadIdx.x & 63, rows = C.n_kv_heads * A.tiles;
  Shares S;
  S.s = -1;
  S.len = 0;
  S.cost = 0;
  if (lane < A.n) {
    const int id = A.seqs ? A.seqs[lane] : lane;
    if (id >= 0 && id < C.n_seqs) {
      S.s = id;
      S.len = (int)clamp64(C.len[id], 0, (int64_t)C.max_blocks * C.block_tokens);
    }
    S.cost = kRowCost + units_of(S.len, C.block_tokens, unit);
  }
  const uint32_t all = S.cost * rows, incl = wave_incl_scan(all);
  S.start = incl - all;
  S.total = __builtin_amdgcn_readlane(incl, 63);
  S.count = min(kShares, max(A.n * rows, (int)(S.total / kWaves)));
  return S;
}

// Attention weight of a block: the sum over its units and the group's heads of
// (sum of p) 2^(m of the unit - m) / l. fin: m and 1 / l of the group's heads.
__device__ __forceinline__ float block_weight(const AttendArgs& A, int rk, int blk, int units, int per_block,
                                              const float2* fin) {
  float w = 0.0f;
  for (int u = blk * per_block; u < min(units, (blk + 1) * per_block); ++u) {
    const float2* p = A.wsum + ((int64_t)rk * A.C.max_blocks * per_block + u) * A.group;
    for (int g = 0; g < A.group; ++g) {
      const float m = fin[g].x == -INFINITY ? 0.0f : fin[g].x;
      w += p[g].y * exp2_fast(p[g].x - m) * fin[g].y;
    }
  }
  return w;
}

template <bool BF, int D, int UNIT, bool EVEN>
__global__ void __launch_bounds__(kWaves * 64, 2) attend_kernel(const AttendArgs A) {
  constexpr int T = UNIT / 16;   // token tiles of a unit
  constexpr int KS = D / 32;     // steps of the score product
  constexpr int KL = D / 64;     // 16-byte loads of a key row per lane
  constexpr int E = D / 16;      // dimensions of a lane in the value product
  constexpr int VW = E / 4;      // code words of those
  constexpr int V2 = UNIT / 32;  // steps of the value product
  __shared__ __align__(16) float mrg[kWaves][16][D + 4];
  __shared__ float2 mls[kWaves][16], fins[16];

  const KvView& C = A.C;
  const int lane = threadIdx.x & 63, col = lane & 15, qr = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int BT = C.block_tokens;
  const int halves = BT / UNIT - 1;  // a block is one unit, or two: 0 or 1
  Shares S;
  uint32_t flat = 0, flat_end = 0;
  if constexpr (EVEN) {
    S = shares_of(A, UNIT);
    if ((int)blockIdx.x >= S.count) return;
    flat = S.first_of(blockIdx.x);
    flat_end = S.first_of(blockIdx.x + 1);
  }
  do {  // the rows of a share
    int b, rt, s_id, len, ua, ub, chunk, step, page0 = -1, unit0 = -1;
    int64_t part;
    bool whole;
    if constexpr (EVEN) {
      const int rows = C.n_kv_heads * A.tiles;
      b = __ffsll((unsigned long long)__ballot(flat >= S.start && flat < S.start + S.cost * rows)) - 1;
      const uint32_t cost = __builtin_amdgcn_readlane(S.cost, b);
      const uint32_t at = flat - __builtin_amdgcn_readlane(S.start, b);
      s_id = __builtin_amdgcn_readlane(S.s, b);
      len = __builtin_amdgcn_readlane(S.len, b);
      rt = (int)(at / cost);
      const int in = (int)(at - rt * cost);
      const uint32_t take = min(cost - in, flat_end - flat);
      whole = take == cost;
      ua = max(0, in - kRowCost);
      ub = max(0, in + (int)take - kRowCost);
      chunk = step = 64 * kWaves;
      part = (int64_t)b * rows + rt + blockIdx.x;  // a next row or a next share: one more
      flat += take;
    } else {
      const int row = blockIdx.x / A.splits, split = blockIdx.x - row * A.splits;
      const int rows = C.n_kv_heads * A.tiles;
      b = row / rows, rt = row - b * rows;
      s_id = A.seqs ? A.seqs[b] : b;
      if (s_id < 0 || s_id >= C.n_seqs) s_id = -1;
      // The first chunk's pages, asked for before the length is known: lane i of
      // a wave has its i-th unit's.
      unit0 = split * A.chunk + wave + kWaves * lane;
      const int64_t at = ((int64_t)max(s_id, 0) * C.n_kv_heads + rt / A.tiles) * C.max_blocks;
      page0 = (unit0 >> halves) < C.max_blocks ? C.table[at + (unit0 >> halves)] : -1;
      len = s_id >= 0 ? (int)clamp64(C.len[s_id], 0, (int64_t)C.max_blocks * BT) : 0;
      ua = split * A.chunk, ub = units_of(len, BT, UNIT);
      chunk = A.chunk, step = A.splits * A.chunk;
      part = blockIdx.x;
      whole = A.splits == 1;
      if (!whole && ua >= ub) return;  // a part without tokens; the join knows
    }
    if (s_id < 0 && threadIdx.x == 0) atomicOr(C.status, kKvBadIndex);
    const int s = max(s_id, 0);
    const int kvh = rt / A.tiles, ht = rt - kvh * A.tiles, rk = b * C.n_kv_heads + kvh;
    const int heads = min(16, A.group - ht * 16);           // query heads of this tile
    const int h0 = kvh * A.group + ht * 16;                 // the first
    const int64_t sh = (int64_t)s * C.n_kv_heads + kvh;
    const int32_t* table = C.table + sh * C.max_blocks;
    const int full = (len / BT) << halves;                  // units that lie in pages
    float2* wsum = A.wsum ? A.wsum + (((int64_t)rk * C.max_blocks) << halves) * A.group + ht * 16 + col
                          : nullptr;

    // queries: column = head, a step's elements where the key loads have them
    u32x4 qf[KS];
    const uint8_t* qrow = A.q + b * A.q_row + (h0 + min(col, heads - 1)) * A.q_head;
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *(const u32x4*)(qrow + ((k / 2) * 64 + qr * 16 + (k & 1) * 8) * 2);
    float qc = A.c;
    if constexpr (BF) {
      uint32_t big = 0;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t u = qf[k][w];
          const uint32_t a = u & 0x7fffu, d = u >> 16 & 0x7fffu;
          big = max(big, max(a < 0x7f80u ? a : 0u, d < 0x7f80u ? d : 0u));
        }
      big = max(big, (uint32_t)__shfl_xor((int)big, 16));
      big = max(big, (uint32_t)__shfl_xor((int)big, 32));
      const int ex = big >= 0x80u ? (int)(big >> 7) - 127 : big ? -126 : 14;  // the largest is below 2^(ex + 1)
      // By 2^116 at most: every bf16 number is a multiple of 2^-133, so all are
      // exact then, and c 2^-up keeps its bits (scales of 2^-10 and more).
      const int up = min(14 - ex, 116);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t u = qf[k][w];
          qf[k][w] = pack16<false>(ldexpf(unpack16<true>(u & 0xffffu), up), ldexpf(unpack16<true>(u >> 16), up));
        }
      qc = ldexpf(A.c, -up);
    }

    f32x4 o[E];
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;

    for (int u0 = ua; u0 < ub; u0 += step) {
      const int u1 = min(ub, u0 + chunk);
      // A wave's units of the chunk are u0 + wave, + kWaves, .. (at most 64);
      // lane i holds the page of its i-th, -1 for one that does not exist: page 0
      // stands in with scales of 0, a block of zeros.
      const int mine = u0 + wave + kWaves * lane;
      int page = 0;
      if (mine < min(u1, full)) {
        page = mine == unit0 ? page0 : table[mine >> halves];
        if (page < 0 || page >= C.n_pages) {
          atomicOr(C.status, kKvBadIndex);
          page = -1;
        }
      }
      // Each register set is loaded for the next unit as soon as the products have
      // taken it, so a wave keeps up to a unit's bytes in flight while it computes.
      u32x4 kw[T][KL];
      uint32_t vw[V2][8][VW];
      auto unit_at = [&](int u, int pg) {
        return ((int64_t)max(pg, 0) * BT + (u & halves) * UNIT) * D;
      };
      auto load_k = [&](int64_t at) {
        const int8_t* kp = C.k_codes + at + col * D + qr * 16;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int k = 0; k < KL; ++k) kw[t][k] = *(const u32x4*)(kp + t * 16 * D + k * 64);
      };
      auto load_v = [&](int64_t at) {
        const int8_t* vp = C.v_codes + at + qr * 4 * D + col * E;
#pragma unroll
        for (int v = 0; v < V2; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int8_t* p = vp + (v * 32 + (j / 4) * 16 + j % 4) * D;
            if constexpr (VW == 2) {
              const u32x2 w = *(const u32x2*)p;
              vw[v][j][0] = w[0], vw[v][j][1] = w[1];
            } else {
              vw[v][j][0] = *(const uint32_t*)p;
            }
          }
      };
      // Scales come by scalar loads: a wait for them does not wait for the pages.
      typedef const __attribute__((address_space(4))) float* Scales;
      const Scales k_scale = (Scales)(uintptr_t)C.k_scale, v_scale = (Scales)(uintptr_t)C.v_scale;
      // One unit, page pg; MORE: then loads the one at `next`. (The last unit is a
      // copy of the code, not a condition in it: where a load may be left out the
      // compiler has to wait for all that may be in flight.)
      auto process = [&](int u, int pg, int64_t next, auto more_t) {
        constexpr bool MORE = decltype(more_t)::value;
        const float ks = pg < 0 ? 0.0f : k_scale[pg], vs = pg < 0 ? 0.0f : v_scale[pg];
        f32x4 x[T];
        const float f = ks * qc;
#pragma unroll
        for (int t = 0; t < T; ++t) {
          x[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            half2v a, d, e, g;
            i8x4_to_h2(kw[t][k / 2][(k & 1) * 2], a, d);
            i8x4_to_h2(kw[t][k / 2][(k & 1) * 2 + 1], e, g);
            const u32x4 kf = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, d),
                              __builtin_bit_cast(uint32_t, e), __builtin_bit_cast(uint32_t, g)};
            x[t] = mfma16<false>(kf, qf[k], x[t]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][r] *= f;
        }
        if constexpr (MORE) load_k(next);
        asm volatile("" ::: "memory");
        float sum;
        const float alpha = softmax_step<T>(x, m, l, &sum);
        if (wsum) {
          sum = add_xor16(add_xor32(sum));
          if (lane < heads) wsum[(int64_t)u * A.group] = make_float2(m, sum);
        }
        u32x4 pf[V2];
#pragma unroll
        for (int v = 0; v < V2; ++v) pf[v] = pack_p<false>(x[2 * v], x[2 * v + 1]);
#pragma unroll
        for (int w = 0; w < VW; ++w) {
          f32x4 acc[4];
#pragma unroll
          for (int v = 0; v < V2; ++v) {
            uint32_t c[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = vw[v][j][w] ^ 0x80808080u;
            auto frag = [&](auto idx) {
              constexpr int I = decltype(idx)::value;
              const u32x4 vf = {pair_of<I>(c[0], c[1]), pair_of<I>(c[2], c[3]), pair_of<I>(c[4], c[5]),
                                pair_of<I>(c[6], c[7])};
              acc[I] = mfma16<false>(vf, pf[v], v == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[I]);
            };
            frag(std::integral_constant<int, 0>());
            frag(std::integral_constant<int, 1>());
            frag(std::integral_constant<int, 2>());
            frag(std::integral_constant<int, 3>());
          }
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              o[w * 4 + i2][r] = fmaf(acc[i2][r], vs, o[w * 4 + i2][r] * alpha);
        }
        if constexpr (MORE) load_v(next);
      };
      const int end = min(u1, full);
      if (u0 + wave < end) {
        int pg = __builtin_amdgcn_readlane(page, 0);
        const int64_t at = unit_at(u0 + wave, pg);
        load_k(at);
        asm volatile("" ::: "memory");  // in this order, so that a wait for the keys is for them alone
        load_v(at);
        int u = u0 + wave;
        for (int i = 1; u + kWaves < end; u += kWaves, ++i) {
          const int next = __builtin_amdgcn_readlane(page, i);
          process(u, pg, unit_at(u + kWaves, next), std::true_type());
          pg = next;
        }
        process(u, pg, 0, std::false_type());
      }
      // Units of the open block, from the 16-bit tail, 32 tokens at a time; rows
      // past the length are zeros, whatever the tail holds there.
      for (int u = max(u0 + wave, full + ((u0 + wave - full) & (kWaves - 1))); u < u1; u += kWaves) {
        const int t_first = (u - full) * UNIT, rest = min(UNIT, len % BT - t_first);
        float sum = 0.0f;
#pragma unroll 1
        for (int part = 0; part < rest; part += 32) {
          const int left = rest - part;
          const uint8_t* kt = C.tail_k + (sh * BT + t_first + part) * (D * 2);
          const uint8_t* vt = C.tail_v + (sh * BT + t_first + part) * (D * 2);
          // every load is issued before the first is used, from the last token
          // where there is none
          typedef uint32_t Row __attribute__((ext_vector_type(E / 2)));
          u32x4 qw[KS], kl[2][KS];
          Row vl[8];
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const int el = (k / 2) * 64 + qr * 16 + (k & 1) * 8;
            qw[k] = *(const u32x4*)(qrow + el * 2);
#pragma unroll
            for (int t = 0; t < 2; ++t)
              kl[t][k] = *(const u32x4*)(kt + (min(t * 16 + col, left - 1) * D + el) * 2);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            vl[j] = *(const Row*)(vt + (min((j / 4) * 16 + qr * 4 + j % 4, left - 1) * D + col * E) * 2);
          __builtin_amdgcn_sched_barrier(0);
          f32x4 x[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            x[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const bool in = t * 16 + col < left;
#pragma unroll
            for (int k = 0; k < KS; ++k)
              x[t] = mfma16<BF>(in ? kl[t][k] : u32x4{0, 0, 0, 0}, qw[k], x[t]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              x[t][r] = t * 16 + qr * 4 + r < left ? x[t][r] * A.c : -INFINITY;
          }
          float part_sum;
          const float alpha = softmax_step<2>(x, m, l, &part_sum);
          sum = sum * alpha + part_sum;
#pragma unroll
          for (int i = 0; i < E; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] *= alpha;
          const u32x4 pf = pack_p<BF>(x[0], x[1]);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if ((j / 4) * 16 + qr * 4 + j % 4 >= left) vl[j] = Row{};
#pragma unroll
          for (int i = 0; i < E; ++i) {
            const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
            const u32x4 vf = {__builtin_amdgcn_perm(vl[1][i / 2], vl[0][i / 2], sel),
                              __builtin_amdgcn_perm(vl[3][i / 2], vl[2][i / 2], sel),
                              __builtin_amdgcn_perm(vl[5][i / 2], vl[4][i / 2], sel),
                              __builtin_amdgcn_perm(vl[7][i / 2], vl[6][i / 2], sel)};
            o[i] = mfma16<BF>(vf, pf, o[i]);
          }
        }
        if (wsum) {
          sum = add_xor16(add_xor32(sum));
          if (lane < heads) wsum[(int64_t)u * A.group] = make_float2(m, sum);
        }
      }
    }

    // Join the waves. Lane (col, qr) holds dimensions (4 qr + r) E + i of head col.
    l = add_xor16(add_xor32(l));
    if (lane < 16) mls[wave][col] = make_float2(m, l);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < E; i += 4)
        *(f32x4*)&mrg[wave][col][(qr * 4 + r) * E + i] = f32x4{o[i][r], o[i + 1][r], o[i + 2][r], o[i + 3][r]};
    __syncthreads();
    const int hd = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * E;
    if (hd < heads) {
      float M = -INFINITY, L = 0.0f, fac[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, mls[w][hd].x);
      const float mu = M == -INFINITY ? 0.0f : M;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        fac[w] = exp2_fast(mls[w][hd].x - mu);
        L += mls[w][hd].y * fac[w];
      }
      float y[E];
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < E; ++i) y[i] = fmaf(mrg[w][hd][d0 + i], fac[w], y[i]);
      if (whole) {
        const int64_t at = (int64_t)b * A.n_heads + h0 + hd;
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        uint32_t* po = (uint32_t*)(A.out + b * A.o_row + (h0 + hd) * A.o_head + d0 * 2);
#pragma unroll
        for (int i = 0; i < E; i += 2) po[i / 2] = pack16<BF>(y[i] * inv, y[i + 1] * inv);
        if ((threadIdx.x & 15) == 0) {
          if (A.lse) A.lse[at] = (M - kLift + log2_fast(L)) * kLn2;
          if (A.weigh_here) fins[hd] = make_float2(M, inv);
          else if (A.fin) A.fin[at] = make_float2(M, inv);
        }
      } else {
        const int64_t at = part * min(A.group, 16) + hd;
        if ((threadIdx.x & 15) == 0) A.part_ml[at] = make_float2(M, L);
        float* po = A.part_o + at * D + d0;
#pragma unroll
        for (int i = 0; i < E; i += 4) *(f32x4*)(po + i) = f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]};
      }
    }
    if constexpr (EVEN) {
      __syncthreads();  // the next row writes the same LDS
    } else if (A.weigh_here) {
      __syncthreads();
      if (s_id < 0) return;
      float* weight = C.weight + sh * C.max_blocks;
      for (int blk = threadIdx.x; blk * BT < len; blk += kWaves * 64)
        weight[blk] += block_weight(A, rk, blk, ub, halves + 1, fins);
    }
  } while (EVEN && flat < flat_end);
}

// The parts of row (b, rt): how many, and the place of the first.
template <bool EVEN>
__device__ __forceinline__ int parts_of(const AttendArgs& A, const Shares& S, int unit, int b, int rt,
                                        int64_t* first) {
  const KvView& C = A.C;
  const int rows = C.n_kv_heads * A.tiles;
  if constexpr (EVEN) {
    const uint32_t cost = __builtin_amdgcn_readlane(S.cost, b);
    const uint32_t at = __builtin_amdgcn_readlane(S.start, b) + rt * cost;
    const int p = S.owner_of(at);
    *first = (int64_t)b * rows + rt + p;
    return S.owner_of(at + cost - 1) - p + 1;
  } else {
    const int s_id = A.seqs ? A.seqs[b] : b;
    const int len = s_id >= 0 && s_id < C.n_seqs
                        ? (int)clamp64(C.len[s_id], 0, (int64_t)C.max_blocks * C.block_tokens) : 0;
    const int units = units_of(len, C.block_tokens, unit);
    *first = ((int64_t)b * rows + rt) * A.splits;
    return min(A.splits, (units + A.chunk - 1) / A.chunk);  // those with tokens
  }
}

// The second launch. The first `weighs` workgroups add the block weights,
// `per_row` of them for a key/value head; the others join the parts of one query
// head's row each, 256 threads, D / 4 of them per part. Both read the parts' m
// and l, so that neither waits for the other (32 sequences x 8 heads, 64 query
// heads: 9.3 us; as two launches 7.5 and 4.9).
template <bool BF, int D, bool EVEN>
__global__ void __launch_bounds__(256) join_kernel(const AttendArgs A, int unit, int weighs, int per_row) {
  constexpr int TS = D / 4, GR = 256 / TS;
  __shared__ __align__(16) f32x4 acc[GR][TS];
  __shared__ float2 fins[kMaxHeads];
  const KvView& C = A.C;
  const int tid = threadIdx.x, th = min(A.group, 16);
  Shares S;
  if constexpr (EVEN) S = shares_of(A, unit);
  int64_t first;
  if ((int)blockIdx.x < weighs) {
    const int rk = blockIdx.x / per_row, part = blockIdx.x - rk * per_row;
    const int b = rk / C.n_kv_heads, kvh = rk - b * C.n_kv_heads;
    const int s = A.seqs ? A.seqs[b] : b;
    if (s < 0 || s >= C.n_seqs) return;
    for (int t = 0; t < A.tiles; ++t) {
      const int parts = A.part_ml ? parts_of<EVEN>(A, S, unit, b, kvh * A.tiles + t, &first) : 1;
      // 16 threads to a head
      const int hd = tid >> 4, h = t * 16 + hd, mine = h < A.group ? parts : 0;
      float M = -INFINITY, L = 0.0f, inv;
      if (A.whole_fin && parts == 1) {
        const float2 f = mine ? A.fin[(int64_t)b * A.n_heads + kvh * A.group + h] : make_float2(0.0f, 0.0f);
        M = f.x, inv = f.y;
      } else {
        const float2* ml = A.part_ml + first * th + hd;
        for (int p = tid & 15; p < mine; p += 16) M = fmaxf(M, ml[(int64_t)p * th].x);
        M = fmaxf(M, row_xor<1>(M)), M = fmaxf(M, row_xor<2>(M));
        M = fmaxf(M, row_xor<4>(M)), M = fmaxf(M, row_xor<8>(M));
        const float mu = M == -INFINITY ? 0.0f : M;
        for (int p = tid & 15; p < mine; p += 16) L += ml[(int64_t)p * th].y * exp2_fast(ml[(int64_t)p * th].x - mu);
        L += row_xor<1>(L), L += row_xor<2>(L), L += row_xor<4>(L), L += row_xor<8>(L);
        inv = L == 0.0f ? 0.0f : 1.0f / L;
      }
      if ((tid & 15) == 0 && mine) fins[h] = make_float2(M, inv);
    }
    __syncthreads();
    const int len = (int)clamp64(C.len[s], 0, (int64_t)C.max_blocks * C.block_tokens);
    const int units = units_of(len, C.block_tokens, unit);
    float* weight = C.weight + ((int64_t)s * C.n_kv_heads + kvh) * C.max_blocks;
    for (int blk = part * 256 + tid; blk * C.block_tokens < len; blk += per_row * 256)
      weight[blk] += block_weight(A, rk, blk, units, C.block_tokens / unit, fins);
    return;
  }
  const int row = blockIdx.x - weighs, b = row / A.n_heads, h = row - b * A.n_heads;
  const int kvh = h / A.group, hg = h - kvh * A.group, hd = hg % 16;
  const int parts = parts_of<EVEN>(A, S, unit, b, kvh * A.tiles + hg / 16, &first);
  if (EVEN && parts == 1) return;  // its workgroup had all of it
  const float2* ml = A.part_ml + first * th + hd;
  float M = -INFINITY, L = 0.0f;
  for (int s = tid & 63; s < parts; s += 64) M = fmaxf(M, ml[s * th].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  const float mu = M == -INFINITY ? 0.0f : M;
  for (int s = tid & 63; s < parts; s += 64) L += ml[s * th].y * exp2_fast(ml[s * th].x - mu);
  L = wave_sum(L);
  f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* po = A.part_o + (first * th + hd) * D + (tid % TS) * 4;
#pragma unroll 4
  for (int s = tid / TS; s < parts; s += GR) {
    const float f = exp2_fast(ml[s * th].x - mu);
    const f32x4 v = *(const f32x4*)(po + (int64_t)s * th * D);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fmaf(v[i], f, y[i]);
  }
  acc[tid / TS][tid % TS] = y;
  __syncthreads();
  if (tid >= TS) return;
#pragma unroll
  for (int g = 1; g < GR; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] += acc[g][tid][i];
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  uint32_t* out = (uint32_t*)(A.out + b * A.o_row + h * A.o_head + tid * 8);
  out[0] = pack16<BF>(y[0] * inv, y[1] * inv);
  out[1] = pack16<BF>(y[2] * inv, y[3] * inv);
  if (tid == 0 && A.lse) A.lse[row] = (M - kLift + log2_fast(L)) * kLn2;
}

int unit_of(const KvView& C) { return C.block_tokens < 64 ? 32 : 64; }

struct Split {
  int tiles, splits, chunk;
  bool even;
  int64_t parts;  // of rows, that the join reads
};

Split split_of(const KvView& C, int n, int n_heads, int max_len) {
  const int unit = unit_of(C), group = n_heads / C.n_kv_heads;
  const int64_t cap = (int64_t)C.max_blocks * C.block_tokens;
  const int64_t most = max_len > 0 && max_len < cap ? max_len : cap;
  const int units = (int)((most + unit - 1) / unit);
  Split S;
  S.tiles = (group + 15) / 16;
  const int64_t rows = (int64_t)n * C.n_kv_heads * S.tiles;
  // Whole rows where they are short, the longer the more of them: the join's
  // launch takes longer than what it saves (us whole and in parts: 8 rows of 13
  // units 9.3 and 9.3, of 18 11.1 and 9.4; 64 rows of 24 13.3 and 13.5, of 32
  // 16.6 and 14.4; 128 rows of 32 18.6 and 20.4).
  const int64_t share = (rows * units + kShares - 1) / kShares;
  const bool whole = units <= (rows >= 128 ? 32 : rows >= 64 ? 24 : 16);
  // Else even shares, where they are long and a wave can hold the sequences, or
  // chunks of a row of 4 to 32 units, 16 and more where that is more than a round
  // of workgroups (shares and chunks: 8 ragged sequences of up to 20000 tokens x 32
  // heads 74 and 83, x 8 heads of up to 16000 25 and 35, of up to 4000, 8 units a
  // share, 15.6 and 16.3; 32 of one head of up to 4000, 4 a share, 12.3 and 12.1;
  // 8 of 6000 each x 8 heads 26 and 24).
  S.even = !whole && share >= 8 && n <= 64 && rows * (cap / unit + kRowCost) < INT32_MAX;
  // With chunks of 16 for any number of rows the parts would grow with the longest
  // length that the caller allows. So there are at most kRounds rounds of
  // them, and the rows' number of parts is odd, so that the first parts, all that
  // short rows have, fall on every XCD (us and MB of workspace with chunks of 16 and
  // so, 64 / 8 heads: 96 ragged sequences of up to 16000 tokens 406, 51 and 314, 35;
  // one of 100000 among 127 short ones 247, 417 and 181, 38; 128 of up to 2000 where
  // 131072 are allowed 256, 550 and 79, 38; 1100 of up to 2100 624, 110 and 450, 0).
  constexpr int kRounds = 16;
  int64_t chunk = whole ? units : share > 32 ? std::max<int64_t>(16, (share + kRounds - 1) / kRounds) : share;
  chunk = (chunk + kWaves - 1) / kWaves * kWaves;
  S.splits = (int)((units + chunk - 1) / chunk);
  if (share > 32 && !whole) S.splits |= 1;
  S.chunk = (int)std::min<int64_t>(chunk, 64 * kWaves);  // a lane holds one page of a wave's
  S.parts = S.even ? rows + kShares : S.splits == 1 ? 0 : rows * S.splits;
  return S;
}

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int64_t kv_attend_workspace(const KvView& C, int n, int n_heads, int track, int max_len) {
  const Split S = split_of(C, n, n_heads, max_len);
  int64_t bytes = 0;
  const int64_t part_heads = S.parts * std::min(n_heads / C.n_kv_heads, 16);
  if (S.parts) bytes += round256(part_heads * 8) + round256(part_heads * C.head_dim * 4);
  if (track)
    bytes += round256((int64_t)n * n_heads * 8) +
             round256((int64_t)n * n_heads * C.max_blocks * (C.block_tokens / unit_of(C)) * 8);
  return bytes;
}

hipError_t launch_kv_attend(const KvView& C, const int32_t* seqs, int n, int n_heads, float scale,
                            const void* q, const int64_t* qs, void* out, const int64_t* os,
                            float* lse, int track, int max_len, void* workspace, hipStream_t stream) {
  const Split S = split_of(C, n, n_heads, max_len);
  AttendArgs A = {};
  A.C = C;
  A.seqs = seqs;
  A.q = (const uint8_t*)q;
  A.out = (uint8_t*)out;
  A.lse = lse;
  A.q_row = qs[0] * 2, A.q_head = qs[1] * 2;
  A.o_row = os[0] * 2, A.o_head = os[1] * 2;
  A.c = (scale > 0.0f ? scale : 1.0f / sqrtf((float)C.head_dim)) * kLog2e;
  A.n = n;
  A.n_heads = n_heads;
  A.group = n_heads / C.n_kv_heads;
  A.tiles = S.tiles;
  A.splits = S.splits;
  A.chunk = S.chunk;
  uint8_t* ws = (uint8_t*)workspace;
  const int64_t part_heads = S.parts * std::min(A.group, 16);
  if (S.parts) {
    A.part_ml = (float2*)ws;
    ws += round256(part_heads * 8);
    A.part_o = (float*)ws;
    ws += round256(part_heads * C.head_dim * 4);
  }
  if (track) {
    A.fin = (float2*)ws;
    ws += round256((int64_t)n * n_heads * 8);
    A.wsum = (float2*)ws;
  }
  const int unit = unit_of(C);
  A.weigh_here = track && !S.parts && S.tiles == 1;
  A.whole_fin = S.even || !S.parts;
  const int64_t grid = S.even ? kShares : (int64_t)n * C.n_kv_heads * S.tiles * S.splits;
  const int64_t cap = (int64_t)C.max_blocks * C.block_tokens;
  const int64_t most = max_len > 0 && max_len < cap ? max_len : cap;
  const int per_row = (int)((most + 256 * C.block_tokens - 1) / (256 * C.block_tokens));
  const int64_t weighs = track && !A.weigh_here ? (int64_t)n * C.n_kv_heads * per_row : 0;
  const int64_t second = weighs + (S.parts ? n * n_heads : 0);
  if (grid > INT32_MAX || second > INT32_MAX) return hipErrorInvalidValue;
  const auto launch = [&](auto bf, auto d, auto u, auto even) {
    constexpr bool BF = decltype(bf)::value, EVEN = decltype(even)::value;
    constexpr int D = decltype(d)::value, UNIT = decltype(u)::value;
    hipLaunchKernelGGL((attend_kernel<BF, D, UNIT, EVEN>), dim3((uint32_t)grid), dim3(kWaves * 64), 0,
                       stream, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !second) return e;
    hipLaunchKernelGGL((join_kernel<BF, D, EVEN>), dim3((uint32_t)second), dim3(256), 0, stream, A, UNIT,
                       (int)weighs, per_row);
    return hipGetLastError();
  };
  const auto by_even = [&](auto bf, auto d, auto u) {
    return S.even ? launch(bf, d, u, std::true_type()) : launch(bf, d, u, std::false_type());
  };
  const auto by_unit = [&](auto bf, auto d) {
    return unit == 64 ? by_even(bf, d, std::integral_constant<int, 64>())
                      : by_even(bf, d, std::integral_constant<int, 32>());
  };
  const auto by_dim = [&](auto bf) {
    return C.head_dim == 128 ? by_unit(bf, std::integral_constant<int, 128>())
                             : by_unit(bf, std::integral_constant<int, 64>());
  };
  return C.bf ? by_dim(std::true_type()) : by_dim(std::false_type());
}

}  // namespace m2c
