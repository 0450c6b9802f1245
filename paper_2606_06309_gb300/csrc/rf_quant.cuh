// rf_quant.cuh -- rows in 8 bits: a row's largest value, its scale, and the digits.
#pragma once
#include <cstdint>

#include "rf_ptx.cuh"
#include "rf_vec.cuh"

namespace rf {

// 127 y / most as the nearest whole number, ties to even.  t = y (k + k_lo) with k + k_lo = 127 / most to 48 bits is
// that quotient rounded once, to nearest: where it is exactly h + 1/2, so is t.  Of 16-bit rows no other
// quotient rounds to a half: t in [2^i, 2^(i+1)) is a quotient of whole numbers with a denominator below
// 2^(20-i), so it differs from a half by 2^(i-20) or more, and t's rounding is 2^(i-24).  Of 32-bit rows one
// may, and is compared exactly: p + pe is c most, c = h + 1/2, and 127 y - p, of numbers that near to each
// other, has no rounding.  Neither overflows: y and most are RowScale's, scaled to 2^28 at most.
__device__ __forceinline__ int exact_digit(float y, float k, float most) {
  const float h = floorf(y * k), c = h + 0.5f;
  const float p = c * most, pe = fmaf(c, most, -p), q = fmaf(127.f, y, -p);
  const int lo = static_cast<int>(h);
  return q > pe || (q == pe && (lo & 1)) ? lo + 1 : lo;
}

// The largest of a value's and a pair's magnitudes, NaN (as 0x7FFFFFFF) above infinity.
__device__ __forceinline__ float largest(float most, float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(most), "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

// The factor and scale of a row whose largest value's bits (without the sign) are most_bits: NaN above
// infinity above the others.  A row with one of those gets the scale NaN and digits 0, so its products are
// NaN.  Rows too small for 127 / most are multiplied by 2^100 first; ones so large that 127 most could pass
// the largest float, by 2^-100 (what that takes below the normal numbers has the digit 0 either way).
struct RowScale {
  float k, k_lo, scale, most, up;
  __device__ __forceinline__ explicit RowScale(uint32_t most_bits) {
    most = __uint_as_float(most_bits);
    up = most < 0x1p-100f ? 0x1p100f : most > 0x1p100f ? 0x1p-100f : 1.f;
    const bool ok = most_bits < 0x7F800000u;
    scale = ok ? most / 127.f : __uint_as_float(0x7FC00000u);
    most *= up;
    k = ok && most > 0.f ? 127.f / most : 0.f;
    k_lo = k != 0.f ? fmaf(-k, most, 127.f) / most : 0.f;
  }
  // EXACT: for the few quotients that land on a half once rounded, and may not be one
  template <bool EXACT, int E>
  __device__ __forceinline__ Vec<int8_t, E> digits(const float (&y)[E]) const {
    // adding 3 2^22 rounds to whole numbers, ties to even, and leaves them in the low bits
    uint32_t w[E + E % 2];
    float worst = 0.f;
    const uint64_t k2 = f2_both(k), lo2 = f2_both(k_lo), up2 = f2_both(up), magic = f2_both(12582912.f);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const uint64_t v = fmul2(f2_pack(y[e], e + 1 < E ? y[e + 1] : 0.f), up2);
      const uint64_t t = ffma2(v, k2, fmul2(v, lo2)), r = fadd2(t, magic);
      float a, b;
      if (EXACT) {
        f2_unpack(fadd2(t, ffma2(r, f2_both(-1.f), magic)), a, b);
        worst = fmaxf(worst, fmaxf(fabsf(a), fabsf(b)));
      }
      f2_unpack(r, a, b);
      w[e] = __float_as_uint(a);
      w[e + 1] = __float_as_uint(b);
    }
    if (EXACT && worst >= 0.5f) {
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = exact_digit(y[e] * up, k, most);
    }
    const uint32_t keep = k == 0.f ? 0 : ~0u;  // (also of rows with an infinity or NaN)
    Vec<int8_t, E> d;
    if constexpr (E % 4 == 0) {
      uint32_t* to = reinterpret_cast<uint32_t*>(&d);
#pragma unroll
      for (int i = 0; i < E / 4; ++i)
        to[i] = keep & __byte_perm(__byte_perm(w[4 * i], w[4 * i + 1], 0x0040),
                                   __byte_perm(w[4 * i + 2], w[4 * i + 3], 0x0040), 0x5410);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d.e[e] = static_cast<int8_t>(keep & w[e]);
    }
    return d;
  }
};

}  // namespace rf
