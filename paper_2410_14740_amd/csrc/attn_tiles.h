// What the kernels share that attend with many query rows: tiles of rows and of
// keys, their places in LDS, and how rows that see many keys are cut along them.
#pragma once

#include <algorithm>

#include "attn_device.h"
#include "wave_ops.h"

namespace m2c {

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

// A sequence's queries and keys. Tiles of keys begin anew where its keys change
// their place: the first `paged` lie in pages of a cache, those up to `held` in its
// open block, the others in rows.
struct Keys {
  int ql, kl, paged, held;

  __device__ __forceinline__ int tiles(int seen) const {  // that the first `seen` keys lie in
    const int a = min(seen, paged), b = min(seen, held) - a, c = seen - a - b;
    return (a + kTileK - 1) / kTileK + (b + kTileK - 1) / kTileK + (c + kTileK - 1) / kTileK;
  }
};

// Arguments of the kernels on tiles of rows. Beside these a kernel's have
//   Keys keys(int b) const     of sequence b of the call
//   kOneRound                  whether parts of rows grow until all run at once
struct RowArgs {
  const uint8_t* q;
  uint8_t* out;
  float* lse;
  const int32_t* cu_q;
  int64_t total_q;
  int64_t q_tok, q_head, o_tok, o_head;  // bytes
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

// The kernel's arguments by a pointer that the compiler cannot tell from others:
// what is read by it is read again, not kept in registers.
template <class Args>
__device__ __forceinline__ const Args* args_again() {
  uint64_t p = (uint64_t)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return (const Args*)(const __attribute__((address_space(4))) Args*)(uintptr_t)p;
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

// The sequence and tile of query rows of tile index x, or -1. Workgroups start
// in index order, and a tile costs what its rows see: sequences go by their
// keys, longest first, and in each a causal mask's longest rows first, so that
// the last workgroups to start are short ones. More than 64 sequences (a lane
// each) are taken as they come.
template <class Args>
__device__ __forceinline__ int find_tile(const Args& A, int x, int* qt) {
  const int lane = threadIdx.x & 63, n = A.n_seqs;
  int b, j, tiles;
  if (n <= 64) {
    int kl = -1, nt = 0;
    if (lane < n) {
      const Keys K = A.keys(lane);
      nt = (K.ql * A.pack + kRows - 1) / kRows;
      kl = K.kl;
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

template <class Args>
__device__ __forceinline__ Plan plan_of(const Args& A) {
  const int lane = threadIdx.x & 63, n = A.n_seqs;
  Plan P = {};
  int kl = -1, kt = 0;
  float work = 0.0f;
  if (lane < n) {
    const Keys K = A.keys(lane);
    const int rows = K.ql * A.pack;
    kl = K.kl;
    P.rows = (rows + kRows - 1) / kRows;
    kt = K.tiles(kl);
    const int off = kl - K.ql;
    const int empty = kl == 0 ? P.rows : A.causal && off < 0 ? -off * A.pack / kRows : 0;
    P.keyed = P.rows - empty;
    int first = kt;  // tiles the first of them sees
    if (A.causal) {
      const int last = min(rows, (empty + 1) * kRows) - 1;
      first = K.tiles(min(kl, max(0, off + last / A.pack + 1)));
    }
    work = 0.5f * (float)P.keyed * ((float)first + (float)kt);
  }
  work = add_xor32(add_xor16(work));
  work += row_xor<1>(work), work += row_xor<2>(work), work += row_xor<4>(work), work += row_xor<8>(work);
  const float share = work * (float)A.units * (1.0f / kShares);
  const bool even = (float)wave_max((uint32_t)kt) <= kUneven * share;
  P.most = even ? 1 << 25 : (int)fminf(fmaxf((float)kLeast, ceilf(share)), 0x1p25f);
  P.most = __builtin_amdgcn_readfirstlane(P.most);
  if constexpr (Args::kOneRound) {
    // Somewhat larger parts where shares come to a few more than run at once: those
    // would run alone afterwards (five rows on each of 16 sequences: 191 us, 167 so).
    const int rows = __builtin_amdgcn_readlane(wave_incl_scan((uint32_t)P.rows), 63);
    const bool grow = rows * A.units <= kShares && !__builtin_amdgcn_readfirstlane(even);
    for (int i = 0; i < 16 && grow; ++i) {
      const int per = P.keyed > 0 ? (kt + P.most - 1) / P.most : 1;
      const int items = per > 1 ? P.keyed * per + P.rows - P.keyed : P.rows;
      if (__builtin_amdgcn_readlane(wave_incl_scan((uint32_t)items), 63) * A.units <= kShares) break;
      P.most = __builtin_amdgcn_readfirstlane(P.most + max(1, P.most >> 4));
    }
  }
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

// Joins the parts of the row tiles that were cut: 32 dimensions of 128 rows per
// workgroup, each lane with the elements it had as a lane of the parts.
template <bool BF, int D, class Args>
__global__ void __launch_bounds__(kWaves * 64) row_join_kernel(const Args A) {
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
    const int64_t q_lo = clamp64(A.cu_q[b], 0, A.total_q);
    const Keys K = A.keys(b);
    const int rows = K.ql * A.pack, last = min(rows, (qt + 1) * kRows) - 1;
    const int seen = A.causal ? min(K.kl, max(0, K.kl - K.ql + last / A.pack + 1)) : K.kl;
    const int tiles = K.tiles(seen), parts = (tiles + P.most - 1) / P.most;
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

inline int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

// Query heads of a key/value head whose rows share tiles: rows of a sequence fit 32 bits.
inline int pack_of(int n_heads, int n_kv_heads, int64_t total_q) {
  const int group = n_heads / n_kv_heads;
  return total_q * group <= 1 << 30 ? group : 1;
}

// Room for the parts of row tiles: `parts` of kRows rows.
inline int64_t parts_bytes(int64_t parts, int head_dim) {
  return parts ? 256 + round256(parts * kRows * 8) + parts * kRows * head_dim * 4 : 0;
}

inline void place_parts(RowArgs& A, void* workspace) {
  uint8_t* ws = (uint8_t*)workspace;
  A.cut = (int32_t*)ws;
  A.part_ml = (float2*)(ws + 256);
  A.part_o = (float*)(ws + 256 + round256(2 * (int64_t)A.extra * A.units * kRows * 8));
}

}  // namespace m2c
