// The residual stream between two blocks of a layer: r = x + scale g t, t the
// block's output y, normed or not, and the next block's input N(r) w + b, where
//   N(z) = (z - mean z) / sqrt(mean (z - mean z)^2 + eps)   (mean 0 for M2C_NORM_RMS).
// A row is read once and kept in registers, 8 consecutive elements of it per
// thread and step, between the sums (one for each mean, over the wave by lane
// exchanges and over the waves of a row through LDS) and what is written; of rows
// of more than 32768 elements, 64 a thread, most of that is in scratch memory (350
// to 500 spilled registers). Bound by memory: 10692 rows of 8192, x and what comes of it in fp32, y and N in bf16, are
// 1.05 GB in 185 us from a graph and 200 to 215 between other kernels (5.7 and 4.9
// to 5.3 TB/s; a 1 GiB copy: 5.1). One row: 2.4 us, the two sums one after another.
// x fp32, y fp16: 8000 rows of 5000 86 us, of 5001 or at odd addresses 124 to 130:
// types known at run time only stand as branches between the loads, and take 110
// registers for 70, so a CU holds one row of ten waves, not two. y bf16: 1000 rows of
// 32768 88 us (4.5 TB/s), of 40000 119, of 65536 200 (3.9 TB/s), 65535 270.
#include <type_traits>

#include "attn_device.h"
#include "rows_device.h"
#include "wave_ops.h"

namespace m2c {

namespace {

struct NormArgs {
  const uint8_t *x, *y;
  uint8_t *x_out, *out;
  const uint8_t *weight, *bias, *post_weight, *post_bias, *gate;
  int64_t rows, x_row, y_row, x_out_row, out_row, gate_row;  // bytes
  float scale, eps, inv_d;
  int d, layer, post;
  int x32, y32, o32, w32;  // which are fp32
};

// Elements 8 i .. 8 i + 7 of a row; ones past its end are zeros. VEC: the row is
// aligned to 16 bytes and its length divides by 8. Otherwise the same wide loads,
// which global memory takes at any element's address, and the last few one by one.
template <int ALIGN, typename T>
struct Unaligned {
  typedef T type __attribute__((aligned(ALIGN)));
};

template <bool BF, bool VEC>
__device__ __forceinline__ void load8(const uint8_t* row, bool f32, int i, int d, float (&v)[8]) {
  const int64_t at = (int64_t)i * 8;
  if (VEC ? 8 * i >= d : 8 * i + 8 > d) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = VEC || at + j >= d ? 0.0f
             : f32              ? *(const float*)(row + (at + j) * 4)
                                : unpack16<BF>(*(const uint16_t*)(row + (at + j) * 2));
  } else if (f32) {
    typedef typename Unaligned<VEC ? 16 : 4, f32x4>::type Four;
    const f32x4 a = *(const Four*)(row + at * 4), b = *(const Four*)(row + at * 4 + 16);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < 4 ? a[j % 4] : b[j % 4];
  } else {
    const u32x4 a = *(const typename Unaligned<VEC ? 16 : 2, u32x4>::type*)(row + at * 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = unpack16<BF>(j & 1 ? a[j / 2] >> 16 : a[j / 2] & 0xffffu);
  }
}

template <bool BF, bool VEC>
__device__ __forceinline__ void store8(uint8_t* row, bool f32, int i, int d, const float (&v)[8]) {
  const int64_t at = (int64_t)i * 8;
  if (VEC ? 8 * i >= d : 8 * i + 8 > d) {
    if (VEC) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (at + j >= d) continue;
      if (f32) *(float*)(row + (at + j) * 4) = v[j];
      else *(uint16_t*)(row + (at + j) * 2) = (uint16_t)pack16<BF>(v[j], 0.0f);
    }
  } else if (f32) {
    typedef typename Unaligned<VEC ? 16 : 4, f32x4>::type Four;
    *(Four*)(row + at * 4) = f32x4{v[0], v[1], v[2], v[3]};
    *(Four*)(row + at * 4 + 16) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    *(typename Unaligned<VEC ? 16 : 2, u32x4>::type*)(row + at * 2) =
        u32x4{pack16<BF>(v[0], v[1]), pack16<BF>(v[2], v[3]), pack16<BF>(v[4], v[5]), pack16<BF>(v[6], v[7])};
  }
}

constexpr int kMaxWaves = 16;  // of a row

// The sums over a row's threads, the same in all of them. slot: a part of the
// LDS that the sum before did not use, so that one barrier is enough.
struct RowSum {
  float (*red)[kMaxWaves];
  double* wide;
  int waves, wave, slot;

  __device__ __forceinline__ float add(float v) {
    v += row_xor<1>(v), v += row_xor<2>(v), v += row_xor<4>(v), v += row_xor<8>(v);
    v = add_xor32(add_xor16(v));
    if (waves == 1) return v;
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) red[slot][wave] = v;
    __syncthreads();
    v = 0.0f;
    for (int i = 0; i < waves; ++i) v += red[slot][i];
    return v;
  }
  __device__ __forceinline__ double add(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    if (waves == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) wide[wave] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < waves; ++i) v += wide[i];
    return v;
  }
};

// What takes a row in registers to N of it: z becomes (z size - mean) f. Sums are
// fp32; where they leave its range (a row of numbers near the largest or smallest,
// or of zeros) they are taken again in 64 bits, and the row is brought near 1 by a
// power of two first, as z - mean or 1 / sqrt may leave fp32 too.
struct Norm {
  float size, mean, f;
};

__device__ __forceinline__ int exponent_of(double v) { return (int)(__double_as_longlong(v) >> 52 & 0x7ff) - 1023; }

template <int V>
__device__ __forceinline__ Norm statistics(const NormArgs& A, const float (&v)[V][8], const bool (&in)[V][8],
                                             RowSum& sum) {
  float mean = 0.0f;
  if (A.layer) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[k][j];
    mean = sum.add(s) * A.inv_d;
  }
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < V; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = in[k][j] ? v[k][j] - mean : 0.0f;
      s = fmaf(c, c, s);
    }
  s = sum.add(s);
  if (s > 0x1p-80f && s < 0x1p120f) return {1.0f, mean, __frsqrt_rn(fmaf(s, A.inv_d, A.eps))};
  double m = 0.0;
  if (A.layer) {
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += (double)v[k][j];
    m = sum.add(m) / A.d;
  }
  double q = 0.0;
#pragma unroll
  for (int k = 0; k < V; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double c = in[k][j] ? (double)v[k][j] - m : 0.0;
      q = fma(c, c, q);
    }
  const double rms = sqrt(sum.add(q) / A.d + (double)A.eps);
  // the mean of a row of nearly equal numbers, far larger than rms, stays below 2^121
  const int e = max(min(max(exponent_of(rms), -126), 126), exponent_of(m) - 120);
  const double size = rms > 0.0 && rms < 0x1p200 ? ldexp(1.0, -e) : 1.0;
  return {(float)size, (float)(m * size), (float)(1.0 / (rms * size))};
}

// A workgroup, of `waves` waves, to a row of at most waves * V * 512 elements. X32, Y32, O32: which
// of the arrays are fp32; without VEC they are known at run time only.
template <bool BF, bool X32, bool Y32, bool O32, int V, bool VEC>
__global__ void __launch_bounds__(1024) residual_norm_kernel(const NormArgs A, int waves) {
  __shared__ float red[2][kMaxWaves];
  __shared__ double wide[kMaxWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= A.rows) return;
  const int threads = waves * 64, tid = threadIdx.x;
  RowSum sum = {red, wide, waves, wave, 0};
  const bool x32 = VEC ? X32 : A.x32, y32 = VEC ? Y32 : A.y32, o32 = VEC ? O32 : A.o32;
  auto at = [&](int k) { return tid + k * threads; };

  // x beside y from the start; of long rows x when y's sums are known, in y's registers
  constexpr bool kEarly = V <= 2;
  float x[V][8], y[kEarly ? V : 1][8];
  bool in[V][8];
#pragma unroll
  for (int k = 0; k < V; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) in[k][j] = 8 * at(k) + (VEC ? 0 : j) < A.d;
  if (kEarly || !A.y) {
#pragma unroll
    for (int k = 0; k < V; ++k) load8<BF, VEC>(A.x + row * A.x_row, x32, at(k), A.d, x[k]);
  }
  if (A.y) {
    float (&t)[V][8] = *[&] {
      if constexpr (kEarly) return &y;
      else return &x;
    }();
#pragma unroll
    for (int k = 0; k < V; ++k) load8<BF, VEC>(A.y + row * A.y_row, y32, at(k), A.d, t[k]);
    if (A.post) {
      const Norm st = statistics<V>(A, t, in, sum);
#pragma unroll
      for (int k = 0; k < V; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[k][j] = fmaf(t[k][j], st.size, -st.mean) * st.f;
        float w[8];
        if (A.post_weight) {
          load8<BF, VEC>(A.post_weight, A.w32, at(k), A.d, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) t[k][j] *= w[j];
        }
        if (A.post_bias) {
          load8<BF, VEC>(A.post_bias, A.w32, at(k), A.d, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) t[k][j] += w[j];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (A.gate) {
        float g[8];
        load8<BF, VEC>(A.gate + row * A.gate_row, A.w32, at(k), A.d, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[k][j] *= g[j];
      }
      float late[8];
      if constexpr (!kEarly) load8<BF, VEC>(A.x + row * A.x_row, x32, at(k), A.d, late);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[k][j] = fmaf(A.scale, in[k][j] ? t[k][j] : 0.0f, kEarly ? x[k][j] : late[j]);
    }
  }
  if (A.x_out) {
#pragma unroll
    for (int k = 0; k < V; ++k) store8<BF, VEC>(A.x_out + row * A.x_out_row, x32, at(k), A.d, x[k]);
  }
  if (!A.out) return;
  const Norm st = statistics<V>(A, x, in, sum);
#pragma unroll
  for (int k = 0; k < V; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[k][j] = fmaf(x[k][j], st.size, -st.mean) * st.f;
    float w[8];
    if (A.weight) {
      load8<BF, VEC>(A.weight, A.w32, at(k), A.d, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[k][j] *= w[j];
    }
    if (A.bias) {
      load8<BF, VEC>(A.bias, A.w32, at(k), A.d, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[k][j] += w[j];
    }
    store8<BF, VEC>(A.out + row * A.out_row, o32, at(k), A.d, x[k]);
  }
}

constexpr int64_t kAcross = 1 << 20;  // a grid has fewer than 2^32 threads along x

template <bool BF, bool X32, bool Y32, bool O32, int V, bool VEC>
hipError_t launch_rows(const NormArgs& A, hipStream_t stream) {
  const int waves = (A.d + V * 512 - 1) / (V * 512);
  const int64_t across = A.rows < kAcross ? A.rows : kAcross;
  const dim3 grid((uint32_t)across, (uint32_t)((A.rows + across - 1) / across));
  hipLaunchKernelGGL((residual_norm_kernel<BF, X32, Y32, O32, V, VEC>), grid, dim3(waves * 64), 0, stream, A,
                     waves);
  return hipGetLastError();
}

// As few elements to a thread as a workgroup of 1024 threads allows. 20000 rows of
// 1024: 37.0 us with 8 a thread, 38.5 with 16; 8192 of 4096: 72 and 76; 10692 of
// 8192: 185, 187 and 196 with 32. Rows that come to little more than run at once may
// gain the other way: 889 of 5120, 1.7 times the 512 that do with 8 a thread, 12.1,
// 12.4 and 11.4. Four rows of one wave each to a workgroup took as long as one.
template <bool BF, bool X32, bool Y32, bool O32, bool VEC>
hipError_t launch_typed(const NormArgs& A, hipStream_t stream) {
  if (A.d <= 8192) return launch_rows<BF, X32, Y32, O32, 1, VEC>(A, stream);
  if (A.d <= 16384) return launch_rows<BF, X32, Y32, O32, 2, VEC>(A, stream);
  if (A.d <= 32768) return launch_rows<BF, X32, Y32, O32, 4, VEC>(A, stream);
  return launch_rows<BF, X32, Y32, O32, 8, VEC>(A, stream);
}

}  // namespace

hipError_t launch_residual_norm(const m2c_norm_desc* D, const void* x, const void* y, int64_t rows,
                                void* x_out, void* out, hipStream_t stream) {
  const auto size = [](int dtype) { return dtype == M2C_DTYPE_FP32 ? 4 : 2; };
  NormArgs A;
  A.x = (const uint8_t*)x, A.y = (const uint8_t*)y;
  A.x_out = (uint8_t*)x_out, A.out = (uint8_t*)out;
  A.weight = (const uint8_t*)D->weight, A.bias = (const uint8_t*)D->bias;
  A.post_weight = (const uint8_t*)D->post_weight, A.post_bias = (const uint8_t*)D->post_bias;
  A.gate = (const uint8_t*)D->gate;
  A.rows = rows;
  A.x_row = D->x_stride * size(D->x_dtype), A.y_row = D->y_stride * size(D->y_dtype);
  A.x_out_row = D->x_out_stride * size(D->x_dtype), A.out_row = D->out_stride * size(D->out_dtype);
  A.gate_row = D->gate_stride * size(D->weight_dtype);
  A.scale = D->scale, A.eps = D->eps, A.inv_d = 1.0f / (float)D->d;
  A.d = D->d, A.layer = D->kind == M2C_NORM_LAYER, A.post = D->post;
  A.x32 = D->x_dtype == M2C_DTYPE_FP32, A.y32 = y && D->y_dtype == M2C_DTYPE_FP32;
  A.o32 = out && D->out_dtype == M2C_DTYPE_FP32, A.w32 = D->weight_dtype == M2C_DTYPE_FP32;
  // wide loads where every row of every array begins on 16 bytes
  uintptr_t bits = 0;
  for (const void* p : {(const void*)A.x, (const void*)A.y, (const void*)A.x_out, (const void*)A.out,
                        (const void*)A.weight, (const void*)A.bias, (const void*)A.post_weight,
                        (const void*)A.post_bias, (const void*)A.gate})
    bits |= (uintptr_t)p;
  if (rows > 1) {
    bits |= A.x_row | A.gate_row;
    if (y) bits |= A.y_row;
    if (x_out) bits |= A.x_out_row;
    if (out) bits |= A.out_row;
  }
  const bool vec = A.d % 8 == 0 && bits % 16 == 0;
  const bool weighted = A.weight || A.bias || A.post_weight || A.post_bias || A.gate;
  const bool bf = D->x_dtype == M2C_DTYPE_BF16 || (y && D->y_dtype == M2C_DTYPE_BF16) ||
                  (out && D->out_dtype == M2C_DTYPE_BF16) || (weighted && D->weight_dtype == M2C_DTYPE_BF16);
  const auto flag = [](bool b, auto f) { return b ? f(std::true_type()) : f(std::false_type()); };
  return flag(bf, [&](auto b) {
    constexpr bool BF = decltype(b)::value;
    if (!vec) return launch_typed<BF, false, false, false, false>(A, stream);
    return flag(A.x32, [&](auto x32) {
      return flag(A.y32, [&](auto y32) {
        return flag(A.o32, [&](auto o32) {
          return launch_typed<BF, decltype(x32)::value, decltype(y32)::value, decltype(o32)::value, true>(A, stream);
        });
      });
    });
  });
}

}  // namespace m2c
