// Matrix-instruction types and small helpers of the attention kernels.
#pragma once

#include "m2c_internal.h"

namespace m2c {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// D = A B + C on 16-bit inputs held as raw words. 32x32x16: lane l holds row
// (column) l % 32 of A (B), elements 8 (l / 32) .. + 7 of the 16 of the sum;
// D's lane l holds column l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4.
// 16x16x32: row (column) l % 16, elements 8 (l / 16) .. + 7 of 32; D's column
// l % 16, rows 4 (l / 16) + r. The order of the summed elements is free as
// long as A and B agree.
template <bool BF>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, a),
                                                   __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a),
                                                  __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

template <bool BF>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, a),
                                                   __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a),
                                                  __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// Two floats as a pair of the 16-bit type, each rounded to nearest even.
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (BF) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  } else {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
}

template <bool BF>
__device__ __forceinline__ float unpack16(uint32_t bits) {  // the low 16 bits
  if constexpr (BF) return __uint_as_float(bits << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// The larger / the sum of v and the value of the lane 32 away.
__device__ __forceinline__ float max_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The same with the lane 16 away.
__device__ __forceinline__ float max_xor16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_xor16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) {
  return v < lo ? lo : v > hi ? hi : v;
}

// The work items of packed sequences in one flat range without a prefix sum:
// sequence b, of `mul` rows per token, owns items item_start(cu[b], b) ..
// item_start(cu[b + 1], b + 1) - 1, at least rows / per + `more` of them (floor),
// since floor((a + n) / per) - floor(a / per) >= floor(n / per).
__device__ __forceinline__ int64_t item_start(int64_t cu, int b, int per, int more, int mul = 1) {
  return cu * mul / per + (int64_t)b * more;
}

// The sequence that owns item x, or -1 (wave-uniform). Where cu does not ascend
// x may lie before the first item of the one that this names.
__device__ __forceinline__ int find_item(const int32_t* cu, int n, int64_t total, int64_t x,
                                         int per, int more, int mul = 1) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < n; base += 64) {
    const int b = base + lane;
    const bool at_or_before =
        b < n && item_start(clamp64(cu[b], 0, total), b, per, more, mul) <= x;
    const int cnt = __popcll(__ballot(at_or_before));
    if (cnt < 64)  // -1 before the first sequence's items
      return __builtin_amdgcn_readfirstlane(base + cnt - 1);
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

}  // namespace m2c
