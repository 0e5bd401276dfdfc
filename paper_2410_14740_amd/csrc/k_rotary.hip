// Queries and keys turned by their positions: rows are read and written once, a
// workgroup takes a few tokens and some or all of their heads. Bound by memory:
// 16385 tokens of 64 query and 8 key heads of 128 are 604 MB in 117 to 120 us (5.1
// TB/s, as a 1 GiB copy), 4096 of 32 and 32 heads 134 MB in 22 us, part of it from
// the caches. One token: 2.2 us.
#include <algorithm>
#include <type_traits>

#include "rotary_device.h"
#include "rows_device.h"

namespace m2c {

namespace {

constexpr int64_t kAcross = 1 << 20;  // groups of tokens along x: a grid has fewer than 2^32 threads there

template <bool BF, int D, bool INTER>
__global__ void __launch_bounds__(256) rotate_kernel(const TurnView T, const TurnRows Q, const TurnRows K,
                                                     int64_t total, int parts) {
  __shared__ __align__(16) float2 cs[kTurnTokens][64];
  const int x = blockIdx.x / parts, part = blockIdx.x - x * parts;
  const int64_t tok0 = ((int64_t)blockIdx.y * kAcross + x) * kTurnTokens;
  if (tok0 >= total) return;
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
  // few tokens: their heads go to several workgroups. 16 tokens of 64 and 8 heads:
  // 2.4 us, by one workgroup 5.6; 257 of 32 and 32: 3.4 and 5.7; 1024: 6.3 and 7.6;
  // 4096 alike; more parts than for 512 workgroups bring nothing.
  const int parts = (int)std::min<int64_t>(std::max<int64_t>(512 / groups, 1), (heads + 7) / 8);
  const dim3 grid((uint32_t)(std::min(groups, kAcross) * parts), (uint32_t)((groups + kAcross - 1) / kAcross));
  const auto go = [&](auto b, auto d, auto inter) {
    hipLaunchKernelGGL((rotate_kernel<decltype(b)::value, decltype(d)::value, decltype(inter)::value>),
                       grid, dim3(256), 0, stream, T, Q, K, total, parts);
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
