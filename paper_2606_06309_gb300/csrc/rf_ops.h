// rf_ops.h -- host-side helpers of the operators around the attention (rf_rope, rf_cross_attn,
// rf_linear): element types and tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "rf_div.h"
#include "rf_host.h"

namespace rf {

// Bytes of an element of `dtype` (rf_dtype), 0 if it is none.
inline int dtype_bytes(int dtype) {
  return dtype == RF_BF16 || dtype == RF_FP16 ? 2 : dtype == RF_FP32 ? 4 : 0;
}

// A tiled map of `rank` <= 3 dimensions of `dtype` (innermost first), 128-byte swizzle,
// zeros out of bounds.  strides: bytes, of dimensions 1 .. rank-1.
rf_status make_tensor_map(CUtensorMap* m, int dtype, const void* base, int rank,
                          const uint64_t* dims, const uint64_t* strides, const uint32_t* box);

}  // namespace rf
