// rf_ops.h -- host-side helpers of the operators around the attention (rf_rope, rf_cross_attn,
// rf_linear): element types, tensor maps, and the division used to find a row's frame and token.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "rf_host.h"

namespace rf {

// Bytes of an element of `dtype` (rf_dtype), 0 if it is none.
inline int dtype_bytes(int dtype) {
  return dtype == RF_BF16 || dtype == RF_FP16 ? 2 : dtype == RF_FP32 ? 4 : 0;
}

// A tiled map of `rank` <= 3 dimensions of 16-bit elements (innermost first), 128-byte swizzle,
// zeros out of bounds.  strides: bytes, of dimensions 1 .. rank-1.
rf_status make_tensor_map(CUtensorMap* m, int dtype, const void* base, int rank,
                          const uint64_t* dims, const uint64_t* strides, const uint32_t* box);

// Division by an invariant 31-bit divisor as a multiplication: with l = ceil(log2 d) and
// m = floor(2^32 (2^l - d) / d) + 1, x / d = (mulhi(x, m) + x) >> l for x < 2^31 (Granlund and
// Montgomery, "Division by invariant integers using multiplication", 1994; the sum cannot carry
// for x < 2^31, as mulhi(x, m) <= x).
struct FastDiv {
  uint32_t d = 1, mul = 1, shift = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t divisor) : d(divisor) {
    while ((1ull << shift) < d) ++shift;
    mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ uint32_t div(uint32_t x) const {
    return (__umulhi(x, mul) + x) >> shift;
  }
  __device__ __forceinline__ void divmod(uint32_t x, uint32_t& q, uint32_t& r) const {
    q = div(x);
    r = x - q * d;
  }
#endif
};

}  // namespace rf
