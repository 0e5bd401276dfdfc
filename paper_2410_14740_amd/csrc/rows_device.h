// Calls on rows of the residual stream, of queries and of keys.
#pragma once

#include "rotary_device.h"

namespace m2c {

hipError_t launch_residual_norm(const m2c_norm_desc* D, const void* x, const void* y, int64_t rows,
                                void* x_out, void* out, hipStream_t stream);

// What m2c_rotary and the positions say, as the kernels take it.
TurnView turn_view(const m2c_rotary* R, const int32_t* positions, int64_t pos_stride);

hipError_t launch_rotate(const TurnView& T, bool interleaved, bool bf, int head_dim, int64_t total,
                         const TurnRows& Q, const TurnRows& K, hipStream_t stream);

}  // namespace m2c
