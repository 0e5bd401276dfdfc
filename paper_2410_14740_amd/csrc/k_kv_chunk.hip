// Attention of chunks of tokens over the 8-bit key/value cache: many query rows a
// sequence, which see the tokens that the cache holds and, where the chunk is not
// in it yet, its own keys and values, causally.
//
// Per query row over the keys it sees, with c = scale * log2 e:
//   x_j = c <q, k_j>,  m = max x_j,  p_j = 2^(x_j - m),  l = sum p_j,
//   O = sum p_j v_j / l,  lse = (m + log2 l) ln 2,
// in one pass over tiles of 64 keys. A page's keys are codes with one scale, and
// its values too: x_j = (c s_k) <q, code_j>, and s_v goes into the weight,
// p_j s_v = 2^(x_j + g - m), g = log2(s_v / 2^u): m is then the largest x_j + g, l
// sums the weights of a block times 2^-g, and O is in units of 2^u. Codes become
// fp16 exactly on their way into LDS; queries of bf16 caches are scaled by a power
// of two per row into fp16's range (exact but for elements 2^-24 of the row's
// largest). So both products sum exact products in fp32 and a weight alone is
// rounded, relative 2^-11 (2^-8 over the 16-bit keys of bf16 caches).
//
// Rows, products and LDS tiles lie as in the attention of prompts; the 16-bit keys
// (the open block, the chunk's own) go straight into LDS as there, codes by way of
// registers: a tile's are loaded while the one before it is written to LDS and the
// one before that is computed.
//
// Bound by matrix instructions (43% of the cycles) and vector ones (59%), which
// hardly run at the same time, and by the codes' way into LDS, a quarter of a tile's
// time. 64 query heads on 8 of 128, 2048 and 700 rows after 30000 and 16385 tokens:
// 2.75 to 2.9 ms (0.85 to 0.9 PFLOP/s, by the machine's clock). Five rows on each of
// 16 sequences of 700 to 31870 tokens: 160 us, 525 MB; a tile takes 1.2 us however
// few of its rows there are. 40 heads, 512, 300 and 77 rows after 3500, 1511 and 2323:
// 117 us. The bf16 kernel of 128 spills 62 registers, nearly all in the key-by-key sum
// of tiles that hold a value that is not finite, none in the loops over pages and
// over whole tiles.
#include <type_traits>

#include "attn_tiles.h"
#include "ffn_device.h"
#include "kv_device.h"

namespace m2c {

struct ChunkArgs : RowArgs {
  static constexpr bool kOneRound = true;
  KvView C;
  const int32_t* seqs;
  const uint8_t *k, *v;  // the chunk's keys and values, or NULL: the cache has them
  int64_t k_tok, k_head, v_tok, v_head;  // bytes

  __device__ __forceinline__ int seq(int b) const {  // its sequence in the cache, or -1
    const int s = seqs ? seqs[b] : b;
    return s >= 0 && s < C.n_seqs ? s : -1;
  }
  __device__ __forceinline__ Keys keys(int b) const {
    const int64_t lo = clamp64(cu_q[b], 0, total_q), hi = clamp64(cu_q[b + 1], lo, total_q);
    const int s = seq(b), ql = (int)(hi - lo);
    if (s < 0) return {ql, 0, 0, 0};
    const int len = (int)clamp64(C.len[s], 0, (int64_t)C.max_blocks * C.block_tokens);
    return {ql, k ? len + ql : len, len - len % C.block_tokens, len};
  }
};

namespace {

// Values lie in LDS as in the attention of prompts, but that odd rows (of 64: the
// second two of four) swap neighbouring chunks, for the writes of codes.
template <int D>
__device__ __forceinline__ int swz_values(int row) {
  return D == 128 ? (row & 3) << 2 | (row & 1) : ((row >> 1) & 1) * 5;
}

// A block's key scale and the logarithm of its value scale, -1000 for a scale of 0;
// NaN for scales that are not finite.
struct Block {
  float ks, g;
};

constexpr int kUnitF16 = -24;  // u of fp16 caches: their scales are 2^-31 and more, or 0

template <bool BF, int D, bool SPLIT>
__global__ void __launch_bounds__(kWaves * 64, 2) chunk_attention_kernel(const ChunkArgs A) {
  constexpr int NW = kWaves;
  constexpr int kRowBytes = D * 2, kChunks = D / 8;
  constexpr int kTileBytes = kTileK * kRowBytes;
  constexpr int kLoads = kTileBytes / (NW * 1024);  // per wave, for K and for V
  constexpr int kLoadRows = 1024 / kRowBytes;       // rows one load of a wave covers
  constexpr int kCodeChunks = D / 16;               // 16-byte chunks of a row of codes
  constexpr int CL = 16 * kCodeChunks / 64;         // loads of a lane for a wave's 16 rows of codes
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __align__(1024) uint8_t lds[2][2][kTileBytes];
  __shared__ float weights[NW][16][32];  // of 16 keys, where a value is not finite
  __shared__ Block blocks[2][64];        // of 64 blocks each, the even and the odd 64s
  __shared__ int pages[2][64];

  // What is wrong with the call is reported once.
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < A.n_seqs; i += NW * 64)
      if (A.seq(i) < 0 || A.cu_q[i + 1] < A.cu_q[i]) atomicOr(A.C.status, kKvBadIndex);

  const int n_kv = A.units / A.shared;
  const int x = blockIdx.x / A.units, r = blockIdx.x - x * A.units;
  const int unit = n_kv % 8 == 0 ? (r & 7) * (A.units / 8) + (r >> 3) : r;  // a head's pages in one XCD's L2
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
  const Keys K = A.keys(b);
  const int64_t q_lo = clamp64(A.cu_q[b], 0, A.total_q);
  const int s_id = max(A.seq(b), 0);

  const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = K.ql * A.pack, off = K.kl - K.ql;
  const int r0 = qt * kRows + wave * 32;  // the wave's first row
  const int row = r0 + col;               // the lane's
  const int tok = min(row, rows - 1) / A.pack, hd = min(row, rows - 1) - tok * A.pack;
  auto seen_by = [&](int r) { return min(K.kl, max(0, off + r / A.pack + 1)); };
  const int tiles = K.tiles(seen_by(min(rows, (qt + 1) * kRows) - 1));
  int ta = 0, tb = tiles, parts = 1;
  if constexpr (SPLIT) {
    if (most) parts = max(1, (tiles + most - 1) / most);
    if (part >= parts) return;
    ta = (int)((int64_t)part * tiles / parts);
    tb = (int)((int64_t)(part + 1) * tiles / parts);
  }
  const int wv_lo = seen_by(r0);
  const int wv_hi = r0 >= rows ? 0 : seen_by(min(rows, r0 + 32) - 1);
  const int seen = seen_by(min(row, rows - 1));

  const int BT = A.C.block_tokens, shift = __ffs(BT) - 1;
  const int64_t sh = (int64_t)s_id * A.C.n_kv_heads + kvh;
  const int page_tiles = (K.paged + kTileK - 1) / kTileK, open_tiles = (K.held - K.paged + kTileK - 1) / kTileK;

  u32x4 qf[KS];
  {
    const uint8_t* qr = A.q + (q_lo + tok) * A.q_tok + (head + hd) * A.q_head + h * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const u32x4*)(qr + s * 32);
    // wait for them here: a wait inside the loop would also wait for its tiles
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));
  }

  // LDS read addresses, see the attention of prompts
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[0][0][0];
  const uint32_t k_lane = lds_base + col * kRowBytes + ((h ^ swz_k<D>(col)) * 16);
  const int vr = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_lane = lds_base + kTileBytes + vr * kRowBytes +
                          (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ swz_values<D>(vr)) * 16) + (lane & 1) * 8;

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  // The tile in slot t & 1. f, g, inv: of its two halves; left: the keys of it that
  // the lane's row sees (used if MASKED); beside: called between scores and softmax.
  auto compute = [&](int t, const float (&f)[2], const float (&g)[2], const float (&inv)[2], int left,
                     auto codes_t, auto masked_t, auto&& beside) {
    constexpr bool CODES = decltype(codes_t)::value, MASKED = decltype(masked_t)::value, B16 = BF && !CODES;
    const uint32_t ka = k_lane + (t & 1) * (2 * kTileBytes), va = v_lane + (t & 1) * (2 * kTileBytes);
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 k_0 = *lds_at<u32x4>(ka ^ (ks * 32));
      const u32x4 k_1 = *lds_at<u32x4>((ka ^ (ks * 32)) + 32 * kRowBytes);
      s[0] = mfma32<B16>(k_0, qf[ks], s[0]);
      s[1] = mfma32<B16>(k_1, qf[ks], s[1]);
    }
    beside();
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * i + 8 * (r / 4) + 4 * h + r % 4 >= left) s[i][r] = -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float mi = s[i][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mi = fmaxf(mi, s[i][r]);
      // f >= 0: of a block of zero keys it is 0, and -infinity times it NaN where all of
      // this half is masked, which the maximum drops
      mt = fmaxf(mt, fmaf(mi, f[i], g[i]));
    }
    mt = max_xor32(mt);
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
    const float base = (m == -INFINITY ? 0.0f : m) - kLift;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float sum[2] = {0.0f, 0.0f};
      const float at = g[i] - base;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[i][r] = exp2_fast(fmaf(s[i][r], f[i], at));
        // a block that reads back as NaN makes NaN of the rows that see it alone
        if (MASKED && 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= left) s[i][r] = 0.0f;
        sum[r & 1] += s[i][r];
      }
      l = CODES ? fmaf(sum[0] + sum[1], inv[i], l) : l + (sum[0] + sum[1]);
    }
    if constexpr (MASKED && !CODES) {
      // An infinity or NaN among the values must not come to the rows that do not
      // see it, as a product with p = 0 would: such a tile is added key by key.
      uint32_t worst = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          typedef unsigned short us2 __attribute__((ext_vector_type(2)));
          const u32x2 w = read_tr((va ^ (dt * 64)) + (8 * u) * kRowBytes);
#pragma unroll
          for (int e = 0; e < 2; ++e)
            worst = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, worst),
                                                                          __builtin_bit_cast(us2, w[e] & 0x7fff7fffu)));
        }
      constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
      if (__ballot((worst & 0xffffu) >= kInf || (worst >> 16) >= kInf)) {
        const uint32_t vt = lds_base + (t & 1) * (2 * kTileBytes) + kTileBytes;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int r = 0; r < 8; ++r) weights[wave][8 * (r / 4) + 4 * h + r % 4][col] = s[u / 2][(u & 1) * 8 + r];
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own, in order
#pragma unroll 1
          for (int j = 0; j < 16; ++j) {
            const int key = 16 * u + j;
            const float p = weights[wave][j][col];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const u32x2 w = *lds_at<u32x2>(vt + key * kRowBytes + (((dt * 4 + i) ^ swz_values<D>(key)) * 16) + h * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float v = unpack16<BF>(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
                  o[dt][4 * i + e] = key < left ? fmaf(p, v, o[dt][4 * i + e]) : o[dt][4 * i + e];
                }
              }
          }
          asm volatile("" ::: "memory");
        }
        return;
      }
    }
    u32x4 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        p[u][w] = pack16<B16>(s[u / 2][(u & 1) * 8 + 2 * w], s[u / 2][(u & 1) * 8 + 2 * w + 1]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u32x2 lo = read_tr((va ^ (dt * 64)) + (16 * u) * kRowBytes);
        const u32x2 hi = read_tr((va ^ (dt * 64)) + (16 * u + 8) * kRowBytes);
        o[dt] = mfma32<B16>(u32x4{lo[0], lo[1], hi[0], hi[1]}, p[u], o[dt]);
      }
    }
  };
  auto barrier = [&] {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // The 16-bit keys: tiles of the open block, then of the chunk's own.
  {
    const int t0 = max(ta, page_tiles), nt = tb - t0;
    const uint8_t* tk = A.C.tail_k + sh * BT * kRowBytes;
    const uint8_t* tv = A.C.tail_v + sh * BT * kRowBytes;
    const int64_t new_k = q_lo * A.k_tok + kvh * A.k_head, new_v = q_lo * A.v_tok + kvh * A.v_head;
    // first key of local tile t and the end of the keys that lie with it
    auto first_of = [&](int t) {
      const int i = t0 + t - page_tiles;
      return i < open_tiles ? K.paged + i * kTileK : K.held + (i - open_tiles) * kTileK;
    };
    auto end_of = [&](int t) { return t0 + t - page_tiles < open_tiles ? K.held : K.kl; };
    const int ld_row = wave * kLoadRows + lane / kChunks;
    const uint32_t lds0 = lds_base + wave * 1024;
    auto load_tile = [&](int t, bool values) {
      const int k0 = first_of(t), left = min(kTileK, end_of(t) - k0) - 1;
      const bool open = k0 < K.held;
      const int64_t step = open ? kRowBytes : values ? A.v_tok : A.k_tok;
      const uint8_t* at = open ? (values ? tv : tk) + (int64_t)(k0 - K.paged) * kRowBytes
                               : (values ? A.v + new_v : A.k + new_k) + (k0 - K.held) * step;
      const u32x4 buf = buffer_of(at, (uint32_t)(left * step) + kRowBytes);  // rows past the end are zeros
      const int swz = values ? swz_values<D>(ld_row) : swz_k<D>(ld_row);
      const uint32_t first = (uint32_t)(ld_row * step) + ((lane % kChunks) ^ swz) * 16;
      const uint32_t row_step = (uint32_t)(NW * kLoadRows * step);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        load_lds16(buf, first + i * row_step,
                   lds0 + (values ? kTileBytes : 0) + (t & 1) * (2 * kTileBytes) + i * (NW * 1024));
    };
    const float f[2] = {A.c, A.c}, none[2] = {0.0f, 0.0f};
    if (nt > 0) {
      load_tile(0, false);
      load_tile(0, true);
    }
    auto arrive = [&](int t) {
      // this wave's loads have landed, and its reads of the tile before are done
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      barrier();
      if (t + 1 < nt) {
        load_tile(t + 1, false);
        load_tile(t + 1, true);
      }
    };
    auto some = [&](int from, int to) {
      for (int t = from; t < to; ++t) {
        arrive(t);
        if (first_of(t) < wv_hi)
          compute(t, f, none, none, min(seen, end_of(t)) - first_of(t), std::false_type(), std::true_type(), [] {});
      }
    };
    // tiles of the chunk's own keys that every row of the wave sees whole
    const int own = max(0, page_tiles + open_tiles - t0), before = max(0, t0 - page_tiles - open_tiles);
    const int whole = r0 >= rows ? 0 : max(0, (wv_lo - K.held) / kTileK - before);
    const int from = min(max(nt, 0), own), to = min(max(nt, 0), own + whole);
    some(0, from);
    for (int t = from; t < to; ++t) {
      arrive(t);
      compute(t, f, none, none, 0, std::false_type(), std::false_type(), [] {});
    }
    some(max(from, to), nt);
  }

  // The pages.
  int u = 0;  // O is in units of 2^u
  const int nt = min(tb, page_tiles) - ta;
  if (nt > 0) {
    float qc = A.c;
    if constexpr (BF) {
      uint32_t big = 0;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t a = qf[k][w] & 0x7fffu, d = qf[k][w] >> 16 & 0x7fffu;
          big = max(big, max(a < 0x7f80u ? a : 0u, d < 0x7f80u ? d : 0u));
        }
      big = max(big, (uint32_t)__shfl_xor((int)big, 32));
      const int ex = big >= 0x80u ? (int)(big >> 7) - 127 : big ? -126 : 14;  // the largest is below 2^(ex + 1)
      // by 2^116 at most: all are exact then, and c 2^-up keeps its bits
      const int up = min(14 - ex, 116);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t v = qf[k][w];
          qf[k][w] = pack16<false>(ldexpf(unpack16<true>(v & 0xffffu), up), ldexpf(unpack16<true>(v >> 16), up));
        }
      qc = ldexpf(A.c, -up);
    }
    const ChunkArgs& P = *args_again<ChunkArgs>();
    const int32_t* table = P.C.table + sh * P.C.max_blocks;
    const int n_blocks = K.paged >> shift, n_pages = (int)P.C.n_pages;
    // What a block's scales come to is looked up for 64 blocks at a time, by one wave,
    // a lane each. A page out of range, or none, is -1.
    auto look_page = [&](int w) {
      const int blk = w * 64 + lane, page = table[min(blk, n_blocks - 1)];
      const bool in = page >= 0 && page < n_pages;
      if (blk < n_blocks && !in) atomicOr(P.C.status, kKvBadIndex);
      return blk < n_blocks && in ? page : -1;
    };
    auto look_up = [&](int w, int page, float ks, float vs) {
      const float g = log2_fast(__builtin_amdgcn_frexp_mantf(vs)) + (float)__builtin_amdgcn_frexp_expf(vs);
      pages[w & 1][lane] = page;
      blocks[w & 1][lane] = page < 0 ? Block{0.0f, -1000.0f} : Block{fmaf(ks, 0.0f, ks), vs == 0.0f ? -1000.0f : fmaf(vs, 0.0f, g)};
    };
    const int w0 = (ta * kTileK) >> shift >> 6;
    if (wave < 2) {
      const int page = look_page(w0 + wave);
      look_up(w0 + wave, page, P.C.k_scale[max(page, 0)], P.C.v_scale[max(page, 0)]);
    }
    if constexpr (!BF) {
      u = kUnitF16;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = ldexpf(o[dt][r], -u);
    }
    // u of bf16 caches: 2^-20 of the first block's scale that is not 0, or 2^-100 of
    // what O has by then, and a larger one should a later scale be 2^40 times as large.
    // In a larger unit every x + g so far is as much less, and so is m, which later
    // weights are to be measured by; l, a sum of 2^(x - m), grows. Where l would pass
    // 2^100 (a sum of blocks 2^-80 of the new one's size) O takes the rest.
    bool unit_set = !BF;
    auto set_unit = [&](int e) __attribute__((always_inline)) {  // for a scale in [2^(e - 1), 2^e)
      int up = e - 20 - u;
      if (!unit_set) {
        int top = -1000;  // O's numbers are below 2^top
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int x = __float_as_uint(o[dt][r]) >> 23 & 0xff;
            top = max(top, x < 255 ? x - 126 : -1000);
          }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, __shfl_xor(top, d));
        up = max(up, __builtin_amdgcn_readfirstlane(top) - 100);
        unit_set = true;
      }
      u += up;
      const int most = 227 - (int)(__float_as_uint(max_xor32(l)) >> 23);  // the row's l stays below 2^101
      const int by = max(0, min(up, most));
      m -= (float)by;
      l = ldexpf(l, by);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = ldexpf(o[dt][r], by - up);
    };
    // A wave's rows of a tile are 16 wave .. + 15. A load covers 1024 bytes of them, 16
    // codes a lane, which become two chunks of 16 bytes in LDS. LDS takes 128 bytes of
    // a write at a time, eight lanes': four of one row, whose chunks are even, and four
    // of another, whose are odd by the swizzle (all eight of one row: half as fast).
    const int c_row = D == 128 ? (lane >> 4) * 2 + (lane >> 2 & 1)
                               : (lane >> 4) * 4 + (lane >> 2 & 1) * 2 + (lane >> 3 & 1);
    const int c_chunk = D == 128 ? (lane >> 3 & 1) * 4 + (lane & 3) : lane & 3;
    const int c_at = c_row * D + c_chunk * 16;
    u32x4 rk[CL], rv[CL];
    auto load_codes = [&](int t, int page) {  // a page of -1 loads zeros
      const int64_t at = (((int64_t)max(page, 0) << shift) + (((ta + t) * kTileK + 16 * wave) & (BT - 1))) * D;
      const int bytes = page < 0 ? 0 : 16 * D;
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(P.C.k_codes + at, 0, bytes, 0x00020000);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(P.C.v_codes + at, 0, bytes, 0x00020000);
#pragma unroll
      for (int i = 0; i < CL; ++i) rk[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, c_at + i * 1024, 0, 0));
#pragma unroll
      for (int i = 0; i < CL; ++i) rv[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, c_at + i * 1024, 0, 0));
    };
    auto write_codes = [&](int t, const u32x4 (&x)[CL], bool values) {
#pragma unroll
      for (int i = 0; i < CL; ++i) {
        const int row = 16 * wave + c_row + i * (64 / kCodeChunks);
        const int swz = values ? swz_values<D>(row) : swz_k<D>(row);
        const uint32_t at = lds_base + (t & 1) * (2 * kTileBytes) + (values ? kTileBytes : 0) + row * kRowBytes;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          half2v a, b, c, d;
          i8x4_to_h2(x[i][2 * j], a, b);
          i8x4_to_h2(x[i][2 * j + 1], c, d);
          *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(at + ((2 * c_chunk + j) ^ swz) * 16) =
              u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                    __builtin_bit_cast(uint32_t, d)};
        }
      }
    };
    auto block_of = [&](int t, int key) { return ((ta + t) * kTileK + key) >> shift; };
    // Tile t is computed while t + 1 goes into LDS and t + 2 comes into registers.
    int page_of = -1;  // that of the wave's rows of tile t + 3
    auto ask_page = [&](int t) {
      const int blk = block_of(t, 16 * wave);
      page_of = pages[blk >> 6 & 1][blk & 63];
    };
    int next_at = -1, next_page = -1;  // the following 64 blocks: which, their pages and scales
    float next_ks = 0.0f, next_vs = 0.0f;
    auto look_ahead = [&](int t) {  // in three steps, so that none has to wait
      const int blk = block_of(t, 0), w = blk >> 6;
      if ((w & 3) != wave) return;
      if ((blk & 63) == 8) {
        next_page = look_page(next_at = w + 1);
      } else if (next_at != w + 1) {
        return;  // begun after the first step: looked up before the first tile
      } else if ((blk & 63) == 16) {
        next_ks = P.C.k_scale[max(next_page, 0)], next_vs = P.C.v_scale[max(next_page, 0)];
      } else if ((blk & 63) == 24) {
        look_up(w + 1, next_page, next_ks, next_vs);
      }
    };
    auto meet = [&] {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's writes, and its reads of the tile before
      barrier();
    };
    // Beside the score products of tile t (before them 3% slower). Past the last tile
    // it writes what nobody reads.
    auto stage = [&](int t) {
      write_codes(t + 1, rk, false);
      write_codes(t + 1, rv, true);
      load_codes(t + 2, t + 2 < nt ? __builtin_amdgcn_readfirstlane(page_of) : -1);
      ask_page(t + 3);
    };
    auto attend = [&](int t, auto masked_t) {
      Block b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int blk = block_of(t, 32 * i);
        b[i] = blocks[blk >> 6 & 1][blk & 63];
      }
      if constexpr (BF) {
        const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fmaxf(b[0].g, b[1].g))));
        if (top > (unit_set ? (float)(u + 60) : -999.0f)) set_unit((int)floorf(top) + 1);
      }
      float f[2], g[2], inv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[i] = qc * b[i].ks;
        const float e = fmaxf(b[i].g - (float)u, -60.0f);  // scales below 2^-60 units count as 2^-60
        g[i] = fmaf(b[i].g, 0.0f, e), inv[i] = exp2_fast(-e);
      }
      compute(t, f, g, inv, min(seen, K.paged) - (ta + t) * kTileK, std::true_type(), masked_t, [&] { stage(t); });
    };
    const int plain = r0 >= rows ? 0 : min(nt, min(wv_lo, K.paged) / kTileK - ta);  // tiles that all its rows see whole
    meet();  // the tiles before are read, and the first blocks looked up
    ask_page(0);
    load_codes(0, __builtin_amdgcn_readfirstlane(page_of));
    ask_page(1);
    write_codes(0, rk, false);
    write_codes(0, rv, true);
    if (1 < nt) load_codes(1, __builtin_amdgcn_readfirstlane(page_of));
    ask_page(2);
    int t = 0;
    for (; t < plain; ++t) {
      meet();
      attend(t, std::false_type());
      look_ahead(t);
    }
    for (; t < nt; ++t) {
      meet();
      if ((ta + t) * kTileK < wv_hi) attend(t, std::true_type());
      else stage(t);
      look_ahead(t);
    }
  }

  if (r0 >= rows) return;
  l = add_xor32(l);
  if (SPLIT && parts > 1) {
    const int64_t at = ((int64_t)slot * A.units + unit) * kWaves + wave;
    float* part_o = A.part_o + at * (32 * D);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(part_o + ((dt * 4 + i) * 64 + lane) * 4) =
            f32x4{ldexpf(o[dt][4 * i], u), ldexpf(o[dt][4 * i + 1], u), ldexpf(o[dt][4 * i + 2], u),
                  ldexpf(o[dt][4 * i + 3], u)};
    if (h == 0) A.part_ml[at * 32 + col] = make_float2(m, l);
    return;
  }
  if (row >= rows) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint8_t* orow = A.out + (q_lo + tok) * A.o_tok + (head + hd) * A.o_head + h * 8;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = ldexpf(o[dt][4 * i + e] * inv, u);
      *(u32x2*)(orow + dt * 64 + i * 16) = u32x2{pack16<BF>(y[0], y[1]), pack16<BF>(y[2], y[3])};
    }
  if (A.lse && h == 0) A.lse[(q_lo + tok) * A.n_heads + head + hd] = (m - kLift + log2_fast(l)) * kLn2;
}

// Parts beyond the first of a row tile to make room for, per unit, or 0 (see the
// attention of prompts). max_q, max_len: the longest chunk and the most tokens that
// a sequence holds in the cache, 0 if not known. Plans hold a sequence a lane: more
// than 64 are not cut. Five rows of 64 / 8 heads on each of n sequences of 500 to
// 4200 tokens, one of 100000 among them: n 64 218 us, 65 1.91 to 1.96 ms, that one's
// time, 256 1.95 to 2.2; without it 104, 134 and 391.
int extra_of(const KvView& C, int n, int n_heads, int64_t total, int max_q, int max_len) {
  if (n > 64) return 0;
  const int64_t cap = (int64_t)C.max_blocks * C.block_tokens;
  const int64_t keys = (max_len > 0 && max_len < cap ? max_len : cap) + (max_q > 0 && max_q < total ? max_q : total);
  const int pack = pack_of(n_heads, C.n_kv_heads, total), units = n_heads / pack;
  const int64_t tiles = (keys + kTileK - 1) / kTileK + 2, rows = total * pack / kRows + n;
  if (tiles <= kLeast + 2) return 0;
  // a single sequence of enough rows: each sees half the longest's tiles or more on average
  if (n == 1 && (float)(total * n_heads) * kUneven >= (float)(kShares * 2 * kRows)) return 0;
  return (int)std::min<int64_t>((kExtra + units - 1) / units, rows * ((tiles - 1) / kLeast));
}

template <bool BF, int D>
hipError_t launch_chunks(ChunkArgs& A, hipStream_t stream) {
  const int64_t grid = (A.total_q * A.pack / kRows + A.n_seqs + A.extra) * A.units;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (!A.extra) {
    hipLaunchKernelGGL((chunk_attention_kernel<BF, D, false>), dim3((uint32_t)grid), dim3(kWaves * 64), 0, stream, A);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((chunk_attention_kernel<BF, D, true>), dim3((uint32_t)grid), dim3(kWaves * 64), 0, stream, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((row_join_kernel<BF, D, ChunkArgs>), dim3(kJoins), dim3(kWaves * 64), 0, stream, A);
  return hipGetLastError();
}

}  // namespace

int64_t kv_chunk_workspace(const KvView& C, int n, int n_heads, int64_t total, int max_q, int max_len) {
  return parts_bytes(2 * (int64_t)extra_of(C, n, n_heads, total, max_q, max_len) *
                         (n_heads / pack_of(n_heads, C.n_kv_heads, total)), C.head_dim);
}

hipError_t launch_kv_chunk(const KvView& C, const int32_t* seqs, int n, const int32_t* cu, int64_t total,
                           int n_heads, float scale, const void* q, const int64_t* qs, const void* k,
                           const int64_t* ks, const void* v, const int64_t* vs, void* out, const int64_t* os,
                           float* lse, int max_q, int max_len, void* workspace, hipStream_t stream) {
  ChunkArgs A;
  A.C = C;
  A.seqs = seqs;
  A.q = (const uint8_t*)q, A.out = (uint8_t*)out, A.lse = lse;
  A.k = (const uint8_t*)k, A.v = (const uint8_t*)v;
  A.cu_q = cu, A.total_q = total, A.n_seqs = n;
  A.q_tok = qs[0] * 2, A.q_head = qs[1] * 2, A.o_tok = os[0] * 2, A.o_head = os[1] * 2;
  A.k_tok = k ? ks[0] * 2 : 0, A.k_head = k ? ks[1] * 2 : 0;
  A.v_tok = k ? vs[0] * 2 : 0, A.v_head = k ? vs[1] * 2 : 0;
  A.c = (scale > 0.0f ? scale : 1.0f / sqrtf((float)C.head_dim)) * kLog2e;
  A.n_heads = n_heads;
  A.causal = 1;
  A.pack = pack_of(n_heads, C.n_kv_heads, total);
  A.units = n_heads / A.pack;
  A.shared = A.units / C.n_kv_heads;
  A.extra = workspace ? extra_of(C, n, n_heads, total, max_q, max_len) : 0;
  place_parts(A, workspace);
  if (C.bf) return C.head_dim == 128 ? launch_chunks<true, 128>(A, stream) : launch_chunks<true, 64>(A, stream);
  return C.head_dim == 128 ? launch_chunks<false, 128>(A, stream) : launch_chunks<false, 64>(A, stream);
}

}  // namespace m2c
