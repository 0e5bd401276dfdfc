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
//
// A row is one token's query head. The heads that share a key/value head lie in
// the same tiles of rows, token by token, so that few tokens of many heads fill
// them too and read their keys once (16 tokens of 64 / 8 heads on 65536 keys: 157
// us with a head's rows to a tile, 86 so).
// 128 rows per workgroup, 32 per wave, two workgroups per CU (64 KB of LDS and
// up to 256 registers each): the four waves share the key and value tiles,
// loaded straight into LDS one tile ahead. The next tile's score products are in
// the same stretch of code as this tile's softmax, which runs beside them. Few
// rows of many keys are cut along the keys (see Plan).
//
// Measured: 64 / 8 heads of 128, bf16, causal, 8192 + 2500 tokens 1105 to 1230 us
// by the machine's clock, 0.98 to 1.09 PFLOP/s (a bf16 product of 8192^3 by the
// library: 1.25); 32 heads, fp16, seven prompts of 1 .. 2380 tokens 82 to 88 us; 40
// heads, chunks of 512, 300 and 77 rows against up to 3584 keys 76 us and a join
// of 4 that finds nothing to do. What bounds it: the matrix instructions are busy
// in 59% of the cycles, some vector or matrix instruction in 80%; a workgroup alone
// on its CU takes 1.4 us per tile of keys, two together 1.9 us for both, so the last
// two cases, whose longest rows are 38 and 56 tiles, wait for those rows.
#include <algorithm>
#include <type_traits>

#include "attn_device.h"
#include "wave_ops.h"

namespace m2c {

struct PromptArgs {
  const uint8_t *q, *k, *v;
  uint8_t* out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int64_t total_q, total_k;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;  // bytes
  float* part_o;    // [2 extra][units][kRows][D] unnormalized outputs of parts of rows
  float2* part_ml;  // [2 extra][units][kRows] their m and l
  int32_t* cut;     // whether any row tile is cut
  float c;          // scale * log2 e
  int n_seqs, n_heads, causal;
  int pack;    // query heads of a key/value head whose rows lie in one tile: all, or 1
  int units;   // n_heads / pack: what a row tile is taken for
  int shared;  // of those, the ones with the same key/value head
  int extra;   // parts beyond the first of a row tile that there is room for, per unit; 0: none are cut
};

namespace {

constexpr int kTileK = 64;  // keys per tile
constexpr int kWaves = 4, kRows = kWaves * 32;  // query rows per workgroup
// Weights are taken as 2^(x - m + kLift), l and O alike, and m may stay up to
// kSlack below the largest x. Rounded to fp16 the largest is then 2^14, and
// weights down to 2^-24 of 2^m keep all their bits (2^-14 without the lift; a
// long sequence of small weights beside one large one would lose them). It
// cancels in O / l and is taken out of the log-sum-exp.
constexpr float kSlack = 4.0f, kLift = 10.0f;

constexpr int kShares = 512;    // workgroups that run at once: two per CU
constexpr int kLeast = 8;       // tiles of a part at least, where rows are split
constexpr int kJoins = 1024;    // workgroups of the join
constexpr float kUneven = 3.0f;
constexpr int kExtra = 1024;    // parts beyond the first of a row tile, all units

// A raw buffer over `bytes` bytes at p: loads past its end give zeros.
__device__ __forceinline__ u32x4 buffer_of(const uint8_t* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, bytes, 0x00020000u};
}

// 16 bytes per lane from buffer offset `off` (per lane) straight into LDS (lane
// i's land at dst + 16 i, dst the same in every lane, in m0, which is an operand
// so that the compiler knows what it holds). Written out so that the
// compiler does not wait for it at every LDS read that follows: the loads of
// one tile run while the tile before it is used, and one explicit wait and a
// barrier stand between the two.
__device__ __forceinline__ void load_lds16(u32x4 buf, uint32_t off, uint32_t dst) {
  asm volatile(
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %0, 0 offen lds"
      :
      : "s"(buf), "v"(off), "{m0}"(dst)
      : "memory");
}

// LDS reads by byte address.
template <typename T>
__device__ __forceinline__ const __attribute__((address_space(3))) T* lds_at(uint32_t addr) {
  return (const __attribute__((address_space(3))) T*)(uintptr_t)addr;
}
__device__ __forceinline__ u32x2 read_tr(uint32_t addr) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) short4v*)(uintptr_t)addr));
}

// Tiles lie in LDS as [64][D] 16-bit rows, the 16-byte chunks of a row permuted
// by an xor so that the rows a read takes at once fall on different banks (a
// row of 128 elements spans all 64 banks, one of 64 elements half of them).
template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) {
  return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// The rows of one wave again, key by key, each row over the keys it sees only:
// taken where a value that some of the rows must not see is an infinity or a
// NaN, which a product with p = 0 would carry into them. part_o, part_ml (NULL
// for whole rows): the wave's place of a part, which has the first `most` keys.
template <bool BF, int D>
__device__ __forceinline__ void wave_rows_plain(const PromptArgs& A, const uint8_t* qb, const uint8_t* kb,
                                             const uint8_t* vb, uint8_t* ob, float* lse, int r0,
                                             int rows, int off, int kl, int most, float* part_o,
                                             float2* part_ml) {
  const int lane = threadIdx.x & 63;
  constexpr int E = D / 64;
  for (int r = r0; r < r0 + 32 && r < rows; ++r) {
    const int tok = r / A.pack, hd = r - tok * A.pack;
    const int seen = min(most, A.causal ? off + tok + 1 : kl);
    float q[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = unpack16<BF>(*(const uint16_t*)(qb + tok * A.q_tok + hd * A.q_head + (lane + 64 * e) * 2));
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
    if (part_o) {
      const int col = r - r0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = lane + 64 * e;  // where the lane that has it in the products puts it
        part_o[(d / 8 * 64 + (d / 4 & 1) * 32 + col) * 4 + d % 4] = ldexpf(o[e], (int)kLift);
      }
      if (lane == 0) part_ml[col] = make_float2(m, ldexpf(l, (int)kLift));
      continue;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e)
      *(uint16_t*)(ob + tok * A.o_tok + hd * A.o_head + (lane + 64 * e) * 2) = (uint16_t)pack16<BF>(o[e] * inv, 0.0f);
    if (lse && lane == 0)
      lse[(int64_t)tok * A.n_heads + hd] = (m + log2_fast(l)) * kLn2;
  }
}

// The sequence and tile of query rows of tile index x, or -1. Workgroups start
// in index order, and a tile costs what its rows see: sequences go by their
// keys, longest first, and in each a causal mask's longest rows first, so that
// the last workgroups to start are short ones. More than 64 sequences (a lane
// each) are taken as they come.
__device__ __forceinline__ int find_tile(const PromptArgs& A, int x, int* qt) {
  const int lane = threadIdx.x & 63, n = A.n_seqs;
  int b, j, tiles;
  if (n <= 64) {
    int kl = -1, nt = 0;
    if (lane < n) {
      const int64_t lo = clamp64(A.cu_q[lane], 0, A.total_q), hi = clamp64(A.cu_q[lane + 1], lo, A.total_q);
      const int64_t k0 = clamp64(A.cu_k[lane], 0, A.total_k), k1 = clamp64(A.cu_k[lane + 1], k0, A.total_k);
      nt = ((int)(hi - lo) * A.pack + kRows - 1) / kRows;
      kl = (int)(k1 - k0);
    }
    int start = 0;  // tiles of the sequences before the lane's
    for (int i = 0; i < n; ++i) {
      const int k2 = __builtin_amdgcn_readlane(kl, i), n2 = __builtin_amdgcn_readlane(nt, i);
      if (k2 > kl || (k2 == kl && i < lane)) start += n2;
    }
    const unsigned long long own = __ballot(x >= start && x < start + nt);
    if (!own) return -1;
    b = __builtin_amdgcn_readfirstlane(__ffsll(own) - 1);
    j = x - __builtin_amdgcn_readlane(start, b);
    tiles = __builtin_amdgcn_readlane(nt, b);
  } else {
    b = find_item(A.cu_q, n, A.total_q, x, kRows, 1, A.pack);
    if (b < 0) return -1;
    const int64_t lo = clamp64(A.cu_q[b], 0, A.total_q), hi = clamp64(A.cu_q[b + 1], lo, A.total_q);
    tiles = ((int)(hi - lo) * A.pack + kRows - 1) / kRows;
    j = x - (int)item_start(lo, b, kRows, 1, A.pack);
    if (j < 0 || j >= tiles) return -1;  // below 0: starts that do not ascend
  }
  *qt = A.causal ? tiles - 1 - j : j;
  return b;
}

// Where a row tile sees kUneven times as many tiles of keys as each of the
// workgroups that run at once has to take, row tiles are cut along their keys
// into parts of such a share, joined by a second launch. Lane b of a wave holds
// sequence b: the last `keyed` of its row tiles see some key, and each is cut
// into at most `per` parts of up to `most` tiles; the sequence's items are start
// .. in the order of find_tile, a row tile's parts one after another. (Measured,
// in us without and with cuts: 1 head, 6000 rows, longest 21 shares 98, 33; 32 / 8
// heads, 512 rows on 16384 keys, 4 shares 258, 144; 8 heads of 64, 4000 rows, 3.8
// shares 51, 48; 40 heads, 2.2 shares 71, 94. Parts of a half share are as fast or
// slower by up to a tenth.)
struct Plan {
  int rows, keyed, per, start;
  int row_start, slot_start;  // its first among the row tiles and parts of the sequences that are cut
  int most;
  bool any;
};

__device__ __forceinline__ Plan plan_of(const PromptArgs& A) {
  const int lane = threadIdx.x & 63, n = A.n_seqs;
  Plan P = {};
  int kl = -1, kt = 0;
  float work = 0.0f;
  if (lane < n) {
    const int64_t lo = clamp64(A.cu_q[lane], 0, A.total_q), hi = clamp64(A.cu_q[lane + 1], lo, A.total_q);
    const int64_t k0 = clamp64(A.cu_k[lane], 0, A.total_k), k1 = clamp64(A.cu_k[lane + 1], k0, A.total_k);
    const int rows = (int)(hi - lo) * A.pack;
    kl = (int)(k1 - k0);
    P.rows = (rows + kRows - 1) / kRows;
    kt = (kl + kTileK - 1) / kTileK;
    const int off = kl - (int)(hi - lo);
    const int empty = kl == 0 ? P.rows : A.causal && off < 0 ? -off * A.pack / kRows : 0;
    P.keyed = P.rows - empty;
    int first = kt;  // tiles the first of them sees
    if (A.causal) {
      const int last = min(rows, (empty + 1) * kRows) - 1;
      first = (min(kl, max(0, off + last / A.pack + 1)) + kTileK - 1) / kTileK;
    }
    work = 0.5f * (float)P.keyed * ((float)first + (float)kt);
  }
  work = add_xor32(add_xor16(work));
  work += row_xor<1>(work), work += row_xor<2>(work), work += row_xor<4>(work), work += row_xor<8>(work);
  const float share = work * (float)A.units * (1.0f / kShares);
  const bool even = (float)wave_max((uint32_t)kt) <= kUneven * share;
  P.most = even ? 1 << 25 : (int)fminf(fmaxf((float)kLeast, ceilf(share)), 0x1p25f);
  P.most = __builtin_amdgcn_readfirstlane(P.most);
  int cut;
  for (;; P.most *= 2) {  // ends: no sequence has more than 2^24 tiles
    P.per = P.keyed > 0 ? (kt + P.most - 1) / P.most : 1;
    cut = P.per > 1 ? P.keyed * P.per : 0;
    const uint32_t extra = P.per > 1 ? (uint32_t)(cut - P.keyed) : 0u;
    const int all = __builtin_amdgcn_readlane(wave_incl_scan(extra), 63);
    P.any = all > 0;
    if (all <= A.extra) break;
  }
  const int items = P.per > 1 ? cut + P.rows - P.keyed : P.rows;
  const int cut_rows = P.per > 1 ? P.keyed : 0;
  for (int i = 0; i < n; ++i) {
    const int k2 = __builtin_amdgcn_readlane(kl, i), n2 = __builtin_amdgcn_readlane(items, i);
    const int r2 = __builtin_amdgcn_readlane(cut_rows, i), c2 = __builtin_amdgcn_readlane(cut, i);
    if (k2 > kl || (k2 == kl && i < lane)) P.start += n2, P.row_start += r2, P.slot_start += c2;
  }
  return P;
}

// The kernel's arguments by a pointer that the compiler cannot tell from others.
__device__ __forceinline__ const PromptArgs* args_again() {
  uint64_t p = (uint64_t)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return (const PromptArgs*)(const __attribute__((address_space(4))) PromptArgs*)(uintptr_t)p;
}

template <bool BF, int D, bool SPLIT>
__global__ void __launch_bounds__(kWaves * 64, 2) prompt_attention_kernel(const PromptArgs A) {
  constexpr int NW = kWaves;
  constexpr int kRowBytes = D * 2, kChunks = D / 8;
  constexpr int kTileBytes = kTileK * kRowBytes;
  constexpr int kLoads = kTileBytes / (NW * 1024);  // per wave, for K and for V
  constexpr int kLoadRows = 1024 / kRowBytes;       // rows one load of a wave covers
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __align__(1024) uint8_t lds[2][2][kTileBytes];

  // Consecutive workgroups go round the eight XCDs: they take the heads of one
  // query tile, and where the key/value heads divide by eight, each XCD keeps
  // the same ones, so that its L2 holds their keys and values for all tiles.
  const int n_kv = A.units / A.shared;
  const int x = blockIdx.x / A.units, r = blockIdx.x - x * A.units;
  const int unit = n_kv % 8 == 0 ? (r & 7) * (A.units / 8) + (r >> 3) : r;
  const int kvh = unit / A.shared, head = unit * A.pack;
  int qt, b, part = 0, most = 0, slot = 0;
  if constexpr (SPLIT) {
    const Plan P = plan_of(A);
    if (blockIdx.x == 0 && threadIdx.x == 0) *A.cut = P.any;
    const int items = P.per > 1 ? P.keyed * P.per + P.rows - P.keyed : P.rows;
    const unsigned long long own = __ballot(x >= P.start && x < P.start + items);
    if (!own) return;
    b = __builtin_amdgcn_readfirstlane(__ffsll(own) - 1);
    const int j = x - __builtin_amdgcn_readlane(P.start, b), per = __builtin_amdgcn_readlane(P.per, b);
    const int rows = __builtin_amdgcn_readlane(P.rows, b), keyed = __builtin_amdgcn_readlane(P.keyed, b);
    int i = j;
    if (per > 1 && j < keyed * per) {
      i = j / per;
      part = j - i * per;
      most = P.most;
      slot = __builtin_amdgcn_readlane(P.slot_start, b) + j;
    } else if (per > 1) {
      i = j - keyed * per + keyed;
    }
    qt = rows - 1 - i;
  } else {
    b = find_tile(A, x, &qt);
    if (b < 0) return;
  }
  const int64_t q_lo = clamp64(A.cu_q[b], 0, A.total_q), q_hi = clamp64(A.cu_q[b + 1], q_lo, A.total_q);
  const int64_t k_lo = clamp64(A.cu_k[b], 0, A.total_k), k_hi = clamp64(A.cu_k[b + 1], k_lo, A.total_k);
  const int ql = (int)(q_hi - q_lo);
  int kl = (int)(k_hi - k_lo);

  const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint8_t* qb = A.q + q_lo * A.q_tok + head * A.q_head;
  const uint8_t* kb = A.k + k_lo * A.k_tok + kvh * A.k_head;
  const uint8_t* vb = A.v + k_lo * A.v_tok + kvh * A.v_head;

  const int rows = ql * A.pack;
  const int r0 = qt * kRows + wave * 32;  // the wave's first row
  const int row = r0 + col;               // the lane's
  const int tok = min(row, rows - 1) / A.pack, hd = min(row, rows - 1) - tok * A.pack;
  // keys the workgroup, the wave's first and last row, and the lane's row see
  int off = kl - ql;
  auto seen_by = [&](int r) { return A.causal ? min(kl, max(0, off + r / A.pack + 1)) : kl; };
  const int wg_seen = seen_by(min(rows, (qt + 1) * kRows) - 1);
  const int tiles = (wg_seen + kTileK - 1) / kTileK;
  int nt = tiles, parts = 1;
  if constexpr (SPLIT) {
    if (most) parts = max(1, (tiles + most - 1) / most);
    if (part >= parts) return;
    // from here on the keys count from the part's first
    const int ta = (int)((int64_t)part * tiles / parts);
    nt = (int)((int64_t)(part + 1) * tiles / parts) - ta;
    kb += (int64_t)ta * kTileK * A.k_tok;
    vb += (int64_t)ta * kTileK * A.v_tok;
    kl -= ta * kTileK, off -= ta * kTileK;
  }
  const int wv_lo = seen_by(r0);
  const int wv_hi = r0 >= rows ? 0 : seen_by(min(rows, r0 + 32) - 1);
  int seen = 0;  // the lane's, set before the masked tiles

  // global -> LDS: load i of a wave takes rows (i NW + wave) kLoadRows .. of a
  // tile; the tile's buffer ends with the sequence, so rows past it are zeros
  const int ld_row = wave * kLoadRows + lane / kChunks;
  const uint32_t ld_k = (uint32_t)(ld_row * A.k_tok) + ((lane % kChunks) ^ swz_k<D>(ld_row)) * 16;
  const uint32_t ld_v = (uint32_t)(ld_row * A.v_tok) + ((lane % kChunks) ^ swz_v<D>(ld_row)) * 16;
  const uint32_t step_k = (uint32_t)(NW * kLoadRows * A.k_tok), step_v = (uint32_t)(NW * kLoadRows * A.v_tok);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[0][0][0] + wave * 1024;
  auto load_tile = [&](const uint8_t* rows, int64_t tok, uint32_t off, uint32_t step, int t, uint32_t at) {
    const int left = min(kTileK, kl - t * kTileK) - 1;
    const u32x4 buf = buffer_of(rows + (int64_t)t * kTileK * tok, (uint32_t)(left * tok) + kRowBytes);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      load_lds16(buf, off + i * step, lds0 + at + (t & 1) * (2 * kTileBytes) + i * (NW * 1024));
  };
  auto load_k = [&](int t) { load_tile(kb, A.k_tok, ld_k, step_k, t, 0); };
  auto load_v = [&](int t) { load_tile(vb, A.v_tok, ld_v, step_v, t, kTileBytes); };

  u32x4 qf[KS];
  {
    const uint8_t* qr = qb + tok * A.q_tok + hd * A.q_head + h * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const u32x4*)(qr + s * 32);
    // wait for them here: a wait inside the loop would also wait for its tiles
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));
  }

  // LDS read addresses: K row = token col (+ 32), step ks's chunk 2 ks + h; V
  // rows = tokens 4h + i / 4 of a 16-lane group, 16 dimensions from 16 (group &
  // 1) of each 32. The swizzles are xors, so a step is an xor of address bits.
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[0][0][0];
  const uint32_t k_lane = lds_base + col * kRowBytes + ((h ^ swz_k<D>(col)) * 16);
  const int vr = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_lane = lds_base + kTileBytes + vr * kRowBytes +
                          (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ swz_v<D>(vr)) * 16) + (lane & 1) * 8;

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  uint32_t worst = 0;  // largest |value| bits seen in masked tiles, per half word

  // S^T of tile t.
  auto scores = [&](int t, f32x16 (&s)[2]) {
    const uint32_t ka = k_lane + (t & 1) * (2 * kTileBytes);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 k_0 = *lds_at<u32x4>(ka ^ (ks * 32));
      const u32x4 k_1 = *lds_at<u32x4>((ka ^ (ks * 32)) + 32 * kRowBytes);
      s[0] = mfma32<BF>(k_0, qf[ks], s[0]);
      s[1] = mfma32<BF>(k_1, qf[ks], s[1]);
    }
  };
  // Tile t from its scores s, and the scores of the next one into sn: those
  // products do not wait for the softmax, and the softmax runs beside them.
  // MASKED: some row of the wave misses some key of the tile.
  auto compute = [&](int t, f32x16 (&s)[2], f32x16 (&sn)[2], auto masked_t) {
    constexpr bool MASKED = decltype(masked_t)::value;
    const uint32_t va = v_lane + (t & 1) * (2 * kTileBytes);
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * kTileK + 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= seen) s[i][r] = -INFINITY;
    }
    float mt = s[0][0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[i][r]);
    mt = max_xor32(mt) * A.c;  // c > 0
    // m follows the largest score only when that is 2^kSlack above it: the
    // largest weight is then 2^(kLift + kSlack), and most tiles leave l and O as
    // they are.
    if (__ballot(mt > m + kSlack)) {
      const float mn = fmaxf(m, mt);
      const float alpha = exp2_fast(m - (mn == -INFINITY ? 0.0f : mn));
      m = mn;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
    scores(t + 1, sn);
    const float base = (m == -INFINITY ? 0.0f : m) - kLift;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[i][r] = exp2_fast(fmaf(s[i][r], A.c, -base));
        sum[r & 3] += s[i][r];
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    u32x4 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        p[u][w] = pack16<BF>(s[u / 2][(u & 1) * 8 + 2 * w], s[u / 2][(u & 1) * 8 + 2 * w + 1]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u32x2 lo = read_tr((va ^ (dt * 64)) + (16 * u) * kRowBytes);
        const u32x2 hi = read_tr((va ^ (dt * 64)) + (16 * u + 8) * kRowBytes);
        const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
        if constexpr (MASKED) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            typedef unsigned short us2 __attribute__((ext_vector_type(2)));
            worst = __builtin_bit_cast(
                uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, worst),
                                                    __builtin_bit_cast(us2, vf[w] & 0x7fff7fffu)));
          }
        }
        o[dt] = mfma32<BF>(vf, p[u], o[dt]);
      }
    }
  };

  // Tile t needs V(t) and K(t + 1). Waves pass the barriers of the loops
  // together, each with its own number of tiles in the first.
  const int plain = r0 >= rows ? 0 : min(nt, wv_lo / kTileK);  // tiles that every row of the wave sees whole
  auto arrive = [&](int t) {
    // this wave's loads have landed, and its reads of K(t) and V(t - 1) are done
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + 2 < nt) load_k(t + 2);
    if (t + 1 < nt) load_v(t + 1);
  };
  f32x16 s0[2], s1[2];
  if (nt > 0) {
    load_k(0);
    load_v(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (nt > 1) load_k(1);
    scores(0, s0);
  }
  int t = 0;
  for (; t + 1 < plain; t += 2) {
    arrive(t);
    compute(t, s0, s1, std::false_type());
    arrive(t + 1);
    compute(t + 1, s1, s0, std::false_type());
  }
  // What only the masked tiles and the end need is computed again, not kept in
  // registers through the loop above (the compiler, short of them, would order
  // its score products before the softmax instead of beside it).
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int row2 = r0 + (tid & 31);
  seen = seen_by(min(row2, rows - 1));
  for (; t < nt; ++t) {
    arrive(t);
    if (t * kTileK < wv_hi) {
      compute(t, s0, s1, std::true_type());
#pragma unroll
      for (int i = 0; i < 2; ++i) s0[i] = s1[i];
    }
  }
  const PromptArgs& B = *args_again();
  const int64_t first = clamp64(B.cu_q[b], 0, B.total_q);
  uint8_t* ob = B.out + first * B.o_tok + head * B.o_head;
  float* lse = B.lse ? B.lse + first * B.n_heads + head : nullptr;
  constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
  const bool bad = __ballot((worst & 0xffffu) >= kInf || (worst >> 16) >= kInf) != 0;
  if (r0 >= rows) return;
  float* part_o = nullptr;
  float2* part_ml = nullptr;
  if (SPLIT && parts > 1) {
    const int64_t at = ((int64_t)slot * B.units + unit) * kWaves + wave;
    part_o = B.part_o + at * (32 * D);
    part_ml = B.part_ml + at * 32;
  }
  if (bad && B.causal) {
    wave_rows_plain<BF, D>(B, B.q + first * B.q_tok + head * B.q_head, kb, vb, ob, lse, r0, rows, off, kl,
                           min(kl, nt * kTileK), part_o, part_ml);
    return;
  }
  l = add_xor32(l);
  if (SPLIT && parts > 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(part_o + ((dt * 4 + i) * 64 + lane) * 4) =
            f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    if (h == 0) part_ml[col] = make_float2(m, l);
    return;
  }
  if (row2 >= rows) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int o_tok = row2 / B.pack, o_hd = row2 - o_tok * B.pack;
  uint8_t* orow = ob + o_tok * B.o_tok + o_hd * B.o_head + h * 8;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x2 w;
      w[0] = pack16<BF>(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv);
      w[1] = pack16<BF>(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv);
      *(u32x2*)(orow + dt * 64 + i * 16) = w;
    }
  if (lse && h == 0) lse[(int64_t)o_tok * B.n_heads + o_hd] = (m - kLift + log2_fast(l)) * kLn2;
}

// Joins the parts of the row tiles that were cut: 32 dimensions of 128 rows per
// workgroup, each lane with the elements it had as a lane of the parts.
template <bool BF, int D>
__global__ void __launch_bounds__(kWaves * 64) prompt_join_kernel(const PromptArgs A) {
  constexpr int DT = D / 32;
  if (!*A.cut) return;
  const Plan P = plan_of(A);
  for (int id = blockIdx.x;; id += gridDim.x) {  // ends past the row tiles that were cut
    const int x = id / (A.units * DT), r = id - x * (A.units * DT);
    const int unit = r / DT, dt = r - unit * DT;
    const unsigned long long own = __ballot(P.per > 1 && x >= P.row_start && x < P.row_start + P.keyed);
    if (!own) return;
    const int b = __builtin_amdgcn_readfirstlane(__ffsll(own) - 1);
    const int i = x - __builtin_amdgcn_readlane(P.row_start, b), per = __builtin_amdgcn_readlane(P.per, b);
    const int qt = __builtin_amdgcn_readlane(P.rows, b) - 1 - i;
    const int64_t q_lo = clamp64(A.cu_q[b], 0, A.total_q), q_hi = clamp64(A.cu_q[b + 1], q_lo, A.total_q);
    const int64_t k_lo = clamp64(A.cu_k[b], 0, A.total_k), k_hi = clamp64(A.cu_k[b + 1], k_lo, A.total_k);
    const int ql = (int)(q_hi - q_lo), kl = (int)(k_hi - k_lo);
    const int rows = ql * A.pack, last = min(rows, (qt + 1) * kRows) - 1;
    const int seen = A.causal ? min(kl, max(0, kl - ql + last / A.pack + 1)) : kl;
    const int tiles = (seen + kTileK - 1) / kTileK, parts = (tiles + P.most - 1) / P.most;
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = qt * kRows + wave * 32 + col;
    if (parts > 1 && row < rows) {
      const int64_t slot = ((int64_t)__builtin_amdgcn_readlane(P.slot_start, b) + i * per) * A.units + unit;
      const float2* ml = A.part_ml + (slot * kWaves + wave) * 32 + col;
      const float* po = A.part_o + (slot * kWaves + wave) * (32 * D) + (dt * 256 + lane) * 4;
      const int64_t step = (int64_t)A.units * kWaves * 32;  // rows from part to part
      float M = -INFINITY, L = 0.0f;
      for (int p = 0; p < parts; ++p) M = fmaxf(M, ml[p * step].x);
      const float mu = M == -INFINITY ? 0.0f : M;
      f32x4 y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
      for (int p = 0; p < parts; ++p) {
        const float2 v = ml[p * step];
        const float f = exp2_fast(v.x - mu);
        L = fmaf(v.y, f, L);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f32x4 a = *(const f32x4*)(po + p * step * D + k * 256);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[k][e] = fmaf(a[e], f, y[k][e]);
        }
      }
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      const int64_t tok = q_lo + row / A.pack;
      const int head = unit * A.pack + row % A.pack;
      uint8_t* orow = A.out + tok * A.o_tok + head * A.o_head + dt * 64 + h * 8;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const u32x2 w = {pack16<BF>(y[k][0] * inv, y[k][1] * inv), pack16<BF>(y[k][2] * inv, y[k][3] * inv)};
        *(u32x2*)(orow + k * 16) = w;
      }
      if (A.lse && h == 0 && dt == 0)
        A.lse[tok * A.n_heads + head] = (M - kLift + log2_fast(L)) * kLn2;
    }
  }
}

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

int pack_of(const m2c_attn_desc* D, int64_t total_q) {
  const int group = D->n_heads / D->n_kv_heads;
  return total_q * group <= 1 << 30 ? group : 1;  // rows of a sequence fit 32 bits
}

// Parts beyond the first of a row tile to make room for, per unit, or 0. (A row
// tile that is cut has at least one, so there are at most twice as many parts.
// With a share a part they are at most 1024: a sequence's row tiles see half of
// its longest's tiles or more on average.)
int extra_of(const m2c_attn_desc* D, bool self, int n_seqs, int64_t total_q, int64_t total_k) {
  if (n_seqs > 64) return 0;
  const int pack = pack_of(D, total_q), units = D->n_heads / pack;
  const int64_t tiles = (total_k + kTileK - 1) / kTileK, rows = total_q * pack / kRows + n_seqs;
  if (tiles <= kLeast) return 0;
  // Of lq queries with as many keys or more a row tile sees half the longest's
  // tiles or more on average: where they are so many, none is cut. As many keys
  // as queries in all are taken to be the same sequences.
  const int64_t lq = n_seqs == 1 && total_q <= total_k ? total_q
                     : self || total_q == total_k      ? D->max_q
                                                       : 0;
  if ((float)(lq * D->n_heads) * kUneven >= (float)(kShares * 2 * kRows)) return 0;
  const int64_t most = rows * ((tiles - 1) / kLeast);
  return (int)std::min<int64_t>((kExtra + units - 1) / units, most);
}

template <bool BF, int D>
hipError_t launch_rows(PromptArgs& A, hipStream_t stream) {
  const int64_t grid = (A.total_q * A.pack / kRows + A.n_seqs + A.extra) * A.units;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (!A.extra) {
    hipLaunchKernelGGL((prompt_attention_kernel<BF, D, false>), dim3((uint32_t)grid), dim3(kWaves * 64), 0,
                       stream, A);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((prompt_attention_kernel<BF, D, true>), dim3((uint32_t)grid), dim3(kWaves * 64), 0,
                     stream, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prompt_join_kernel<BF, D>), dim3(kJoins), dim3(kWaves * 64), 0, stream, A);
  return hipGetLastError();
}

}  // namespace

int64_t prompt_workspace(const m2c_attn_desc* D, bool self, int n_seqs, int64_t total_q, int64_t total_k) {
  const int64_t parts = 2 * (int64_t)extra_of(D, self, n_seqs, total_q, total_k) *
                        (D->n_heads / pack_of(D, total_q));
  return parts ? 256 + round256(parts * kRows * 8) + parts * kRows * D->head_dim * 4 : 0;
}

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
  A.pack = pack_of(D, total_q);
  A.units = D->n_heads / A.pack;
  A.shared = A.units / D->n_kv_heads;
  A.causal = D->causal;
  A.extra = D->workspace ? extra_of(D, cu_q == cu_k, n_seqs, total_q, total_k) : 0;
  uint8_t* ws = (uint8_t*)D->workspace;
  A.cut = (int32_t*)ws;
  A.part_ml = (float2*)(ws + 256);
  A.part_o = (float*)(ws + 256 + round256(2 * (int64_t)A.extra * A.units * kRows * 8));
  if (D->dtype == M2C_DTYPE_BF16)
    return D->head_dim == 128 ? launch_rows<true, 128>(A, stream) : launch_rows<true, 64>(A, stream);
  return D->head_dim == 128 ? launch_rows<false, 128>(A, stream) : launch_rows<false, 64>(A, stream);
}

}  // namespace m2c
