// Calls on rows of the residual stream, of queries and of keys.
#pragma once

#include "m2c_internal.h"

namespace m2c {

hipError_t launch_residual_norm(const m2c_norm_desc* D, const void* x, const void* y, int64_t rows,
                                void* x_out, void* out, hipStream_t stream);

}  // namespace m2c
