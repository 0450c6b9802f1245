// rf_quant.cu -- rows of the active frames in 8 bits.
//
//     s[t] = max_k |x[t, k]| / 127,   q[t, k] = the whole number nearest to x[t, k] / s[t], ties to even
//
// One read and one write: a team of 32 to 512 threads keeps its row, as it was loaded, in registers until
// its largest value is known.  The search compares the elements' bits without the sign, two 16-bit ones
// per instruction.  Bound by HBM: 75,600 rows of 5120 bf16 188 to 192 us, 6.1 TB/s; two rows of 64 tokens of
// 128 2.1 us, the launch.  Rows of 5120 fp32 376 us, 5.1 TB/s.  Rows off the 16-byte boundaries go element by
// element: 75,600 of 5117 bf16 792 us, 12,480 of 1149 34.
#include <cuda_runtime.h>

#include <algorithm>

#include "rf_ops.h"
#include "rf_quant.cuh"

namespace rf {
namespace {

constexpr int kThreads = 256, kRaw = 8;  // vectors of a row in a thread's registers

struct QuantParams {
  const void* X;
  int8_t* Y;
  float* scale;
  int64_t x_stride, y_stride;
  const int32_t *active, *counts;
  FastDiv by_N;
  int F, N, C, team, segs, whole;
};

// max of the elements' bits without the sign, as bits of a float
template <typename T, int E>
__device__ __forceinline__ uint32_t top_bits(const Vec<T, E>& v, uint32_t most) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < E; ++e) most = max(most, __float_as_uint(v.e[e]) & 0x7FFFFFFFu);
  } else if constexpr (E == 8) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) most = __vmaxu2(most, w[i] & 0x7FFF7FFFu);
  } else {
    most = max(most, static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(&v) & 0x7FFF));
  }
  return most;
}
template <typename T, int E>
__device__ __forceinline__ uint32_t float_bits(uint32_t most) {
  if constexpr (sizeof(T) == 4) {
    return most;
  } else {
    if (E == 8) most = max(most & 0xFFFFu, most >> 16);
    const uint16_t h = static_cast<uint16_t>(most);
    return __float_as_uint(to_f(*reinterpret_cast<const T*>(&h)));  // (infinity and NaN stay what they are)
  }
}

template <typename T, int E>
__global__ void __launch_bounds__(512, 2) quant_kernel(const __grid_constant__ QuantParams p) {
  __shared__ uint32_t top[2][16];
  const int team = p.team, lane = threadIdx.x & (team - 1), teams = blockDim.x / team, who = threadIdx.x / team;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const int A = p.active ? min(max(p.counts[0], 0), p.F) : p.F;
  const int64_t rows = static_cast<int64_t>(A) * p.N;
  int turn = 0;
  // (teams wider than a warp are the whole block: every thread takes part in each turn)
#pragma unroll 1
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * teams + who; r < rows;
       r += static_cast<int64_t>(gridDim.x) * teams, turn ^= 1) {
    const int a = p.by_N.div(static_cast<int>(r));
    const int64_t row = static_cast<int64_t>(p.active ? p.active[a] : a) * p.N + (static_cast<int>(r) - a * p.N);
    const T* x = static_cast<const T*>(p.X) + row * p.x_stride;
    Vec<T, E> v[kRaw];
    auto fetch = [&](int seg) {
#pragma unroll
      for (int i = 0; i < kRaw; ++i) {
        const int c = ((seg * kRaw + i) * team + lane) * E;
        if (c < p.C) v[i] = load_stream<T, E>(x + c);
      }
    };
    uint32_t most = 0;
#pragma unroll 1
    for (int seg = 0; seg < p.segs; ++seg) {
      fetch(seg);
#pragma unroll
      for (int i = 0; i < kRaw; ++i)
        if (((seg * kRaw + i) * team + lane) * E < p.C) most = top_bits<T, E>(v[i], most);
    }
    most = __reduce_max_sync(0xffffffffu, float_bits<T, E>(most));
    if (team > 32) {
      if ((threadIdx.x & 31) == 0) top[turn][threadIdx.x >> 5] = most;
      __syncthreads();
      for (int w = 0; w < team / 32; ++w) most = max(most, top[turn][w]);
    }
    const RowScale rs(most);
    if (lane == 0) p.scale[row] = rs.scale;
    int8_t* to = p.Y + row * p.y_stride;
#pragma unroll 1
    for (int seg = 0; seg < p.segs; ++seg) {
      if (p.segs > 1) fetch(seg);
#pragma unroll
      for (int i = 0; i < kRaw; ++i) {
        const int c = ((seg * kRaw + i) * team + lane) * E;
        if (c >= p.C) continue;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = to_f(v[i].e[e]);
        const Vec<int8_t, E> d = rs.template digits<sizeof(T) == 4>(y);
        if (p.whole) {
          *reinterpret_cast<Vec<int8_t, E>*>(to + c) = d;
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) to[c + e] = d.e[e];
        }
      }
    }
  }
}

template <typename T, int E>
rf_status launch(QuantParams& p, const DeviceInfo& di, cudaStream_t st) {
  const int nv = p.C / E;
  p.team = 32;
  while (p.team < 512 && p.team * kRaw < nv) p.team *= 2;
  p.segs = (nv + p.team * kRaw - 1) / (p.team * kRaw);
  p.whole = reinterpret_cast<uintptr_t>(p.Y) % E == 0 && p.y_stride % E == 0;
  const int block = p.team == 32 ? kThreads : p.team, teams = block / p.team;
  const int64_t rows = static_cast<int64_t>(p.F) * p.N;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(std::min((rows + teams - 1) / teams, static_cast<int64_t>(di.sm_count) * (8192 / block))));
  cfg.blockDim = dim3(static_cast<unsigned>(block));
  cfg.stream = st;
  return launch_early(cfg, 1, "rf_quantize_rows launch", quant_kernel<T, E>, p);
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" rf_status rf_quantize_rows(int8_t* d_Y, int64_t y_row_stride, float* d_scale,
                                      const void* d_X, int64_t x_row_stride, int dtype, int F, int N,
                                      int d, const int32_t* d_active, const int32_t* d_counts,
                                      rf_stream_t stream) {
  if (!d_Y || !d_scale || !d_X) return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: null pointer");
  const int es = dtype_bytes(dtype);
  if (!es) return fail(RF_ERR_UNSUPPORTED, "rf_quantize_rows: dtype");
  if (F < 1 || N < 1 || d < 1) return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: sizes >= 1");
  if (static_cast<int64_t>(F) * N > 0x7FFFFFFF - 65536 || d > 0x7FFFFFFF - 65536)
    return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: too many tokens or elements");
  if (x_row_stride < d || y_row_stride < d)
    return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: row stride below the row's length");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: active list and counts come together");
  if (static_cast<const void*>(d_Y) == d_X) return fail(RF_ERR_INVALID_ARG, "rf_quantize_rows: in place");
  if (reinterpret_cast<uintptr_t>(d_X) % es || reinterpret_cast<uintptr_t>(d_scale) % 4)
    return fail(RF_ERR_MISALIGNED, "rf_quantize_rows: pointer not on its elements' boundary");
  DeviceInfo di;
  if (rf_status st = current_device_info(&di)) return st;
  if (di.cc_major != 10 || di.cc_minor != 3) return fail(RF_ERR_UNSUPPORTED, "needs sm_103");
  QuantParams p{d_X, d_Y, d_scale, x_row_stride, y_row_stride, d_active, d_counts,
                FastDiv(static_cast<uint32_t>(N)), F, N, d, 32, 1, 1};
  const bool vec = static_cast<int64_t>(d) * es % 16 == 0 && aligned16(d_X) && x_row_stride * es % 16 == 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == RF_FP32) return vec ? launch<float, 4>(p, di, s) : launch<float, 1>(p, di, s);
  if (dtype == RF_FP16) return vec ? launch<__half, 8>(p, di, s) : launch<__half, 1>(p, di, s);
  return vec ? launch<__nv_bfloat16, 8>(p, di, s) : launch<__nv_bfloat16, 1>(p, di, s);
}
