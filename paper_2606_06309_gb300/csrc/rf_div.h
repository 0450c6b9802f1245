// rf_div.h -- division by a divisor that stays the same for a launch.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define RF_HOST_DEVICE __host__ __device__
#else
#define RF_HOST_DEVICE
#endif

namespace rf {

// Division by an invariant 31-bit divisor as a multiplication: with l = ceil(log2 d) and
// m = floor(2^32 (2^l - d) / d) + 1, x / d = (mulhi(x, m) + x) >> l for x < 2^31 (Granlund and
// Montgomery, "Division by invariant integers using multiplication", 1994; the sum cannot carry
// for x < 2^31, as mulhi(x, m) <= x).
struct FastDiv {
  uint32_t d = 1, mul = 1, shift = 0;
  FastDiv() = default;
  RF_HOST_DEVICE explicit FastDiv(uint32_t divisor) : d(divisor) {
    while ((1ull << shift) < d) ++shift;
    mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ int div(int x) const { return static_cast<int>(div(static_cast<uint32_t>(x))); }
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
