// Queries and keys turned by their positions: rows are read and written once, a
// workgroup takes a few tokens and some or all of their heads.
#include <algorithm>
#include <type_traits>

#include "rotary_device.h"
#include "rows_device.h"

namespace m2c {

namespace {

template <bool BF, int D, bool INTER>
__global__ void __launch_bounds__(256) rotate_kernel(const TurnView T, const TurnRows Q, const TurnRows K,
                                                     int64_t total, int parts) {
  __shared__ __align__(16) float2 cs[kTurnTokens][64];
  const int g = blockIdx.x / parts, part = blockIdx.x - g * parts;
  const int64_t tok0 = (int64_t)g * kTurnTokens;
  const int heads = Q.heads + K.heads;
  turn_rows<BF, D, INTER>(T, Q, K, tok0, (int)(total - tok0 < kTurnTokens ? total - tok0 : kTurnTokens),
                          part * heads / parts, (part + 1) * heads / parts, cs);
}

}  // namespace

TurnView turn_view(const m2c_rotary* R, const int32_t* positions, int64_t pos_stride) {
  TurnView T;
  T.freq = R->freq;
  T.positions = positions;
  T.pos_stride = pos_stride;
  T.scale = R->scale == 0.0f ? 1.0f : R->scale;
  T.half = R->rot_dim / 2;
  T.axes = R->n_axes;
  for (int a = 0, end = 0; a < 3; ++a) {
    end += a < R->n_axes ? R->section[a] : 0;
    T.end[a] = a + 1 < R->n_axes ? end : INT32_MAX;
  }
  return T;
}

hipError_t launch_rotate(const TurnView& T, bool interleaved, bool bf, int head_dim, int64_t total,
                         const TurnRows& Q, const TurnRows& K, hipStream_t stream) {
  const int64_t groups = (total + kTurnTokens - 1) / kTurnTokens;
  const int heads = Q.heads + K.heads;
  // few tokens: their heads go to several workgroups
  const int parts = (int)std::min<int64_t>(std::max<int64_t>(512 / groups, 1), (heads + 7) / 8);
  if (groups * parts > INT32_MAX) return hipErrorInvalidValue;
  const auto go = [&](auto b, auto d, auto inter) {
    hipLaunchKernelGGL((rotate_kernel<decltype(b)::value, decltype(d)::value, decltype(inter)::value>),
                       dim3((uint32_t)(groups * parts)), dim3(256), 0, stream, T, Q, K, total, parts);
    return hipGetLastError();
  };
  const auto by_pairs = [&](auto b, auto d) {
    return interleaved ? go(b, d, std::true_type()) : go(b, d, std::false_type());
  };
  const auto by_dim = [&](auto b) {
    return head_dim == 128 ? by_pairs(b, std::integral_constant<int, 128>())
                           : by_pairs(b, std::integral_constant<int, 64>());
  };
  return bf ? by_dim(std::true_type()) : by_dim(std::false_type());
}

}  // namespace m2c
