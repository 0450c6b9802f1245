// rf_rope.cu -- rotary positions with three axes (time, height, width) over the active frames.
//
// Token (f, y, x) of a frame grid gh x gw rotates each pair of a head by the angle of the pair's
// axis at the token's position on it:
//     (x0, x1) -> (x0 cos a - x1 sin a, x0 sin a + x1 cos a),   inverse: -sin a.
// (cos, sin) come from one small table per axis (rf_rope_table: 64-bit arithmetic, rounded once),
// so the kernel evaluates no trigonometric function and any positions can be had, also fractional
// ones.  Products and sums in 32 bits, one rounding to the stored type.
//
// The work is one read and one write of the active rows.  A thread keeps its place in the head (16
// bytes of it, or 8 to 16 bytes of each half) and loads the (cos, sin) of its pairs once per token,
// for four heads whose loads are all in flight together; blocks of a fixed grid walk the active
// tokens, since their number is known on the device only (a grid for all F frames would launch F/A
// times the blocks).  Blocks that run together cover all heads of the same tokens, so that rows are
// read and written whole.  A pair's place in the tables is found again for every token, from three
// pointers: kept per pair it took 115 registers.
//
// What bounds it is HBM.  Measured (device time; bytes of one read and one write): 480p, 21
// frames, 12 + 12 heads of 128, bf16, neighbours as pairs: 60.5 us, 6.65 TB/s, as fast as a copy;
// 720p, 40 + 40 heads, fp16, halves: 452 us, 6.85 TB/s.  In halves the loads stand without branches
// between them (with a branch per head and vector they waited for one another: 585 us); with
// neighbours as pairs a branch per head is the better of the two at whole groups of heads (60.5
// against 62.7 us).  Where R/2 is not a multiple of four the halves go element by element: the 480p case
// with R/2 = 45 or 46 takes 104 us, 3.9 TB/s.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "rf_ops.h"

namespace rf {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kHeads = 4;  // of a thread: 64 bytes in flight

struct RopeSide {  // queries or keys
  char* y;
  const char* x;
  int64_t y_stride, x_stride;  // bytes between tokens
  int heads, groups;           // groups of kHeads heads
};

struct RopeParams {
  RopeSide side[2];
  const float2* table[3];  // [positions][half[a]] (cos, sin)
  int half[3];             // pairs of the axis
  int pairs;               // of all axes: R / 2
  const int32_t* active;   // or null: every frame
  const int32_t* counts;
  FastDiv by_N, by_gw;
  int F, N, head_bytes, units;  // units: threads along a head
  float sign;
};

template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f(float v) { return v; }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <typename T, int E>
struct __align__(sizeof(T) * E) Vec {
  T e[E];
};

// E elements per load.  HALF = false: pairs are neighbours, a unit is one vector (E >= 2).
// HALF = true: pair i is (i, i + R/2), a unit is the vectors at i and i + R/2; behind them come
// the units of the elements past R, one vector each, which pass through.
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRopeThreads)
    rope_kernel(const RopeParams p) {
  constexpr int kPairs = HALF ? E : E / 2;  // pairs of a unit
  constexpr int kVecs = HALF ? 2 : 1;
  using V = Vec<T, E>;
  const bool keys = static_cast<int>(blockIdx.x) >= p.side[0].groups;
  const RopeSide s = p.side[keys];
  const int h0 = (blockIdx.x - (keys ? p.side[0].groups : 0)) * kHeads;
  const int nh = min(kHeads, s.heads - h0);
  const int slots = kRopeThreads / p.units;  // tokens of a block at a time
  const int slot = threadIdx.x / p.units, u = threadIdx.x - slot * p.units;
  if (slot >= slots) return;

  // this unit's place in the head
  const int pair0 = u * kPairs;
  const bool through = HALF && pair0 >= p.pairs;  // whole units only (host: pairs % kPairs == 0)
  const int at = (through ? p.pairs * 2 + (u - p.pairs / kPairs) * E : u * E) * sizeof(T);
  // HALF: from i to i + R/2; where nothing is rotated the same vector again
  const int to_other = through ? 0 : p.pairs * static_cast<int>(sizeof(T));
  const int end_t = p.half[0], end_h = end_t + p.half[1];      // the axes' pairs end here

  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const int A = p.active ? min(max(p.counts[0], 0), p.F) : p.F;
  const uint32_t rows = static_cast<uint32_t>(A) * p.N, step = gridDim.y * slots;
  for (uint32_t r = blockIdx.y * slots + slot; r < rows; r += step) {
    uint32_t f, t, y, x;
    p.by_N.divmod(r, f, t);
    p.by_gw.divmod(t, y, x);
    if (p.active) f = p.active[f];
    const int64_t token = static_cast<int64_t>(f) * p.N + t;
    const char* src = s.x + token * s.x_stride + static_cast<int64_t>(h0) * p.head_bytes + at;
    char* dst = s.y + token * s.y_stride + static_cast<int64_t>(h0) * p.head_bytes + at;
    V v[kHeads][kVecs];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (HALF) {  // no branch between the loads: past the last head the last one's again
        const char* q = src + min(h, nh - 1) * p.head_bytes;
        v[h][0] = *reinterpret_cast<const V*>(q);
        v[h][kVecs - 1] = *reinterpret_cast<const V*>(q + to_other);
      } else if (h < nh) {
        v[h][0] = *reinterpret_cast<const V*>(src + h * p.head_bytes);
      }
    }
    // the token's rows of the tables, as if each began with the first pair of all
    const float2* tab_t = p.table[0] + static_cast<int64_t>(f) * p.half[0];
    const float2* tab_h = p.table[1] + (static_cast<int64_t>(y) * p.half[1] - end_t);
    const float2* tab_w = p.table[2] + (static_cast<int64_t>(x) * p.half[2] - end_h);
    float2 cs[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int g = pair0 + i;
      const float2* tab = g < end_t ? tab_t : g < end_h ? tab_h : tab_w;
      cs[i] = g < p.pairs ? __ldg(tab + g) : make_float2(1.f, 0.f);
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (h >= nh) break;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        T& e0 = v[h][0].e[HALF ? i : 2 * i];
        T& e1 = v[h][kVecs - 1].e[HALF ? i : 2 * i + 1];
        const float x0 = to_f(e0), x1 = to_f(e1), sn = p.sign * cs[i].y;
        const float y0 = fmaf(x0, cs[i].x, -(x1 * sn)), y1 = fmaf(x0, sn, x1 * cs[i].x);
        if (pair0 + i < p.pairs) {  // elements past R keep their bits
          e0 = from_f<T>(y0);
          e1 = from_f<T>(y1);
        }
      }
      *reinterpret_cast<V*>(dst + h * p.head_bytes) = v[h][0];
      if (HALF && !through)
        *reinterpret_cast<V*>(dst + h * p.head_bytes + to_other) = v[h][kVecs - 1];
    }
  }
}

template <typename T, int E, bool HALF>
rf_status launch_rope(RopeParams p, int sm_count, cudaStream_t stream) {
  const int d = p.head_bytes / static_cast<int>(sizeof(T));
  p.units = HALF ? p.pairs / E + (d - 2 * p.pairs) / E : d / E;
  for (RopeSide& s : p.side) s.groups = (s.heads + kHeads - 1) / kHeads;
  const int groups = p.side[0].groups + p.side[1].groups, slots = kRopeThreads / p.units;
  const int64_t blocks = (static_cast<int64_t>(p.F) * p.N + slots - 1) / slots;
  // eight blocks of 256 threads fill an SM; four times that many even out the blocks' ends
  const int64_t most = std::max<int64_t>(1, static_cast<int64_t>(sm_count) * 32 / groups);
  const dim3 grid(groups, static_cast<unsigned>(std::min(blocks, most)));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kRopeThreads);
  cfg.stream = stream;
  return launch_early(cfg, 1, "rope_kernel launch", rope_kernel<T, E, HALF>, p);
}

template <typename T>
rf_status launch_rope_type(const RopeParams& p, bool half, int sm_count, cudaStream_t stream) {
  if (!half) return launch_rope<T, 16 / sizeof(T), false>(p, sm_count, stream);
  // Halves: four elements of each at a time, which reach the rate of a copy; eight of a 16-bit type
  // would need the angles of eight pairs in registers.  The second half of the pairs, and what
  // passes through behind it, start on a vector's boundary only where R/2 is a multiple of four.
  if (p.pairs % 4 == 0) return launch_rope<T, 4, true>(p, sm_count, stream);
  return launch_rope<T, 1, true>(p, sm_count, stream);
}

// One side's argument errors.
rf_status check_side(const void* y, const void* x, int64_t ys, int64_t xs, int heads, int d, int es) {
  if (!y || !x) return fail(RF_ERR_INVALID_ARG, "rf_rope: null pointer");
  if (heads < 1 || heads > 16384) return fail(RF_ERR_INVALID_ARG, "rf_rope: heads");
  const int64_t row = static_cast<int64_t>(heads) * d;
  if (ys < row || xs < row) return fail(RF_ERR_INVALID_ARG, "rf_rope: row stride < heads * d");
  if (!aligned16(y) || !aligned16(x) || ys * es % 16 || xs * es % 16)
    return fail(RF_ERR_MISALIGNED, "rf_rope: bases and row strides on 16-byte boundaries");
  if (y == x && ys != xs) return fail(RF_ERR_INVALID_ARG, "rf_rope: in place with two strides");
  return RF_OK;
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" rf_status rf_rope_table(const double* h_pos, int n, int dim, double base,
                                   float* h_table) {
  if (!h_pos || !h_table || n < 1 || dim < 2 || dim % 2 || !(base > 0.0) || !std::isfinite(base))
    return fail(RF_ERR_INVALID_ARG, "rf_rope_table: positions, even dim >= 2, base > 0");
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(h_pos[i])) return fail(RF_ERR_INVALID_ARG, "rf_rope_table: position");
  for (int j = 0; j < dim / 2; ++j) {
    const double freq = std::pow(base, -2.0 * j / dim);
    for (int i = 0; i < n; ++i) {
      float* e = h_table + (static_cast<int64_t>(i) * (dim / 2) + j) * 2;
      e[0] = static_cast<float>(std::cos(h_pos[i] * freq));
      e[1] = static_cast<float>(std::sin(h_pos[i] * freq));
    }
  }
  return RF_OK;
}

extern "C" rf_status rf_rope(void* d_Yq, const void* d_Xq, int64_t yq_row_stride,
                             int64_t xq_row_stride, int Hq, void* d_Yk, const void* d_Xk,
                             int64_t yk_row_stride, int64_t xk_row_stride, int Hk, int dtype, int F,
                             int gh, int gw, int d, int dim_t, int dim_h, int dim_w,
                             const float* d_table_t, const float* d_table_h, const float* d_table_w,
                             int pairing, int inverse, const int32_t* d_active,
                             const int32_t* d_counts, rf_stream_t stream) {
  const int es = dtype_bytes(dtype);
  if (es == 0) return fail(RF_ERR_UNSUPPORTED, "rf_rope: dtype");
  if (F < 1 || gh < 1 || gw < 1) return fail(RF_ERR_INVALID_ARG, "rf_rope: F, gh, gw >= 1");
  if (static_cast<int64_t>(gh) * gw > 0x7FFFFFFF ||
      static_cast<int64_t>(gh) * gw * F > 0x7FFFFFFF - (1 << 24))
    return fail(RF_ERR_INVALID_ARG, "rf_rope: too many tokens");
  if (d < 8 || d > 256 || d % 8) return fail(RF_ERR_UNSUPPORTED, "rf_rope: head dim 8..256, % 8");
  if (pairing != RF_ROPE_INTERLEAVED && pairing != RF_ROPE_HALF)
    return fail(RF_ERR_INVALID_ARG, "rf_rope: pairing");
  const int dims[3] = {dim_t, dim_h, dim_w};
  const float* tables[3] = {d_table_t, d_table_h, d_table_w};
  int64_t R = 0;
  for (int a = 0; a < 3; ++a) {
    if (dims[a] < 0 || dims[a] % 2 || dims[a] > d)
      return fail(RF_ERR_INVALID_ARG, "rf_rope: rotated elements per axis, even, at most d");
    if (dims[a] > 0 && !tables[a]) return fail(RF_ERR_INVALID_ARG, "rf_rope: null table");
    if (reinterpret_cast<uintptr_t>(tables[a]) & 7)
      return fail(RF_ERR_MISALIGNED, "rf_rope: tables on 8-byte boundaries");
    R += dims[a];
  }
  if (R > d) return fail(RF_ERR_INVALID_ARG, "rf_rope: more rotated elements than d");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "rf_rope: active list and counts come together");
  if (rf_status st = check_side(d_Yq, d_Xq, yq_row_stride, xq_row_stride, Hq, d, es)) return st;
  const bool keys = d_Yk || d_Xk || Hk != 0;
  if (keys)
    if (rf_status st = check_side(d_Yk, d_Xk, yk_row_stride, xk_row_stride, Hk, d, es)) return st;
  DeviceInfo di;
  if (rf_status st = current_device_info(&di)) return st;

  RopeParams p{};
  p.side[0] = {static_cast<char*>(d_Yq), static_cast<const char*>(d_Xq), yq_row_stride * es,
               xq_row_stride * es, Hq, 0};
  if (keys)
    p.side[1] = {static_cast<char*>(d_Yk), static_cast<const char*>(d_Xk), yk_row_stride * es,
                 xk_row_stride * es, Hk, 0};
  for (int a = 0; a < 3; ++a) {
    p.table[a] = reinterpret_cast<const float2*>(tables[a]);
    p.half[a] = dims[a] / 2;
  }
  p.pairs = static_cast<int>(R / 2);
  p.active = d_active;
  p.counts = d_counts;
  p.N = gh * gw;
  p.F = F;
  p.by_N = FastDiv(static_cast<uint32_t>(p.N));
  p.by_gw = FastDiv(static_cast<uint32_t>(gw));
  p.head_bytes = d * es;
  p.sign = inverse ? -1.f : 1.f;
  const bool half = pairing == RF_ROPE_HALF;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  switch (dtype) {
    case RF_BF16: return launch_rope_type<__nv_bfloat16>(p, half, di.sm_count, s);
    case RF_FP16: return launch_rope_type<__half>(p, half, di.sm_count, s);
    default: return launch_rope_type<float>(p, half, di.sm_count, s);
  }
}
