// Rotation of rows by their positions: pair i of a head, (a, b), becomes
//   (a cos w - b sin w, b cos w + a sin w),  w = position * freq[i],
// with the position of the pair's axis. The angle is taken in turns, in 64 bits,
// and its fraction alone goes to the hardware's sine and cosine of a turn (2^-22.9
// off at most, over every multiple of 2^-24): far positions lose nothing.
#pragma once

#include "attn_device.h"

namespace m2c {

struct TurnView {
  const float* freq;
  const int32_t* positions;  // [axes][pos_stride]
  int64_t pos_stride;
  float scale;
  int32_t half, axes;  // pairs, axes
  int32_t end[3];      // first pair of axes 1, 2, 3
};

__device__ __forceinline__ int axis_of(const TurnView& T, int pair) {
  return (pair >= T.end[0]) + (pair >= T.end[1]) + (pair >= T.end[2]);
}

// Turns per position of a pair.
__device__ __forceinline__ double turns_of(const TurnView& T, int pair) {
  return (double)T.freq[pair] * 0.15915494309189533577;  // 1 / 2 pi
}

// Cosine and sine of a pair at a row, times the scale.
__device__ __forceinline__ float2 turn_of(const TurnView& T, double turns, int position) {
  const float f = (float)__builtin_amdgcn_fract(turns * (double)position);
  return make_float2(__builtin_amdgcn_cosf(f) * T.scale, __builtin_amdgcn_sinf(f) * T.scale);
}

__device__ __forceinline__ int position_of(const TurnView& T, int pair, int64_t row) {
  return T.positions[T.axes == 1 ? row : axis_of(T, pair) * T.pos_stride + row];
}

// Two pairs (a0, b0), (a1, b1) whose a's and b's lie in one word each.
template <bool BF>
__device__ __forceinline__ void turn_words(uint32_t& a, uint32_t& b, float2 cs0, float2 cs1) {
  const float a0 = unpack16<BF>(a & 0xffffu), a1 = unpack16<BF>(a >> 16);
  const float b0 = unpack16<BF>(b & 0xffffu), b1 = unpack16<BF>(b >> 16);
  a = pack16<BF>(fmaf(a0, cs0.x, -(b0 * cs0.y)), fmaf(a1, cs1.x, -(b1 * cs1.y)));
  b = pack16<BF>(fmaf(b0, cs0.x, a0 * cs0.y), fmaf(b1, cs1.x, a1 * cs1.y));
}

// A pair that is one word.
template <bool BF>
__device__ __forceinline__ uint32_t turn_word(uint32_t w, float2 cs) {
  const float a = unpack16<BF>(w & 0xffffu), b = unpack16<BF>(w >> 16);
  return pack16<BF>(fmaf(a, cs.x, -(b * cs.y)), fmaf(b, cs.x, a * cs.y));
}

// Rows of one tensor, strides in bytes.
struct TurnRows {
  const uint8_t* from;
  uint8_t* to;
  int64_t from_tok, from_head, to_tok, to_head;
  int32_t heads;
};

constexpr int kTurnTokens = 4;  // of a workgroup of 256 threads

// Heads h0 .. h1 - 1 of tokens tok0 .. tok0 + n - 1 (n <= kTurnTokens) of two
// tensors, q's heads before k's. The angles' cosines and sines are computed once,
// shared by the heads through LDS; a thread takes 16 elements of a head at a time:
// 8 pairs, or 16 that do not turn.
template <bool BF, int D, bool INTER>
__device__ __forceinline__ void turn_rows(const TurnView& T, const TurnRows& Q, const TurnRows& K,
                                          int64_t tok0, int n, int h0, int h1,
                                          float2 (*cs)[64]) {
  constexpr int NI = D / 16;
  const int tid = threadIdx.x;
  {
    const int t = tid >> 6, pair = tid & 63;
    if (t < n && pair < T.half)
      cs[t][pair] = turn_of(T, turns_of(T, pair), position_of(T, pair, tok0 + t));
  }
  __syncthreads();
  const int heads = h1 - h0, items = n * heads * NI;
  const int turned = T.half / 8;  // items of a head that turn
  for (int i = tid; i < items; i += 256) {
    const int c = i % NI, x = i / NI, t = x / heads;
    int h = h0 + x - t * heads;
    const bool is_k = h >= Q.heads;
    const TurnRows& R = is_k ? K : Q;
    h -= is_k ? Q.heads : 0;
    const uint8_t* from = R.from + (tok0 + t) * R.from_tok + h * R.from_head;
    uint8_t* to = R.to + (tok0 + t) * R.to_tok + h * R.to_head;
    const bool turns = c < turned;
    const bool apart = !INTER && turns;  // the two sides of the pairs lie half apart
    const int at = apart ? c * 16 : c * 32, step = apart ? T.half * 2 : 16;  // bytes
    u32x4 a = *(const u32x4*)(from + at), b = *(const u32x4*)(from + at + step);
    if (turns) {
      const float2* f = &cs[t][c * 8];
      if constexpr (INTER) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          a[w] = turn_word<BF>(a[w], f[w]);
          b[w] = turn_word<BF>(b[w], f[4 + w]);
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t aw = a[w], bw = b[w];
          turn_words<BF>(aw, bw, f[2 * w], f[2 * w + 1]);
          a[w] = aw, b[w] = bw;
        }
      }
    }
    *(u32x4*)(to + at) = a;
    *(u32x4*)(to + at + step) = b;
  }
}

// 16 bytes (chunk ch) of a row of keys, turned. The other side of a pair is read
// again by the thread that has it.
template <bool BF, bool INTER>
__device__ __forceinline__ u32x4 turn_chunk(const TurnView& T, const uint8_t* row, int64_t index, int ch) {
  u32x4 x = *(const u32x4*)(row + ch * 16);
  if constexpr (INTER) {
    if (ch * 4 >= T.half) return x;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int pair = ch * 4 + w;
      x[w] = turn_word<BF>(x[w], turn_of(T, turns_of(T, pair), position_of(T, pair, index)));
    }
  } else {
    const int chunks = T.half / 8;
    if (ch >= 2 * chunks) return x;
    const bool second = ch >= chunks;
    const int c = second ? ch - chunks : ch;
    u32x4 y = *(const u32x4*)(row + (second ? c : c + chunks) * 16);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float2 f[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int pair = c * 8 + 2 * w + j;
        f[j] = turn_of(T, turns_of(T, pair), position_of(T, pair, index));
      }
      uint32_t a = second ? y[w] : x[w], b = second ? x[w] : y[w];
      turn_words<BF>(a, b, f[0], f[1]);
      x[w] = second ? b : a;
    }
  }
  return x;
}

}  // namespace m2c
