// rf_linear.cu -- matrix product with bias, activation, gate and residual, over the active frames.
//
//     Y[t, n] = R[t, n] + g[n] * act(sum_k X[t, k] W[n, k] + b[n])       t: tokens of active frames
//
// Products of 16-bit elements are exact in 32 bits and summed there (tcgen05, fp32 accumulators in
// tensor memory); bias, activation, gate and residual follow in 32 bits on the accumulator as it
// leaves tensor memory, so Y is rounded once and nothing between them goes to memory.
//
// Two kernels, both fed by TMA from 128-byte-swizzled tiles of 64 columns of K:
//   pair_kernel  many rows: a pair of CTAs on one tile of 256 tokens x 256 columns (cta_group::2).
//   split_kernel few rows: 128 columns of W against 16 to 256 tokens, W as the tensor core's M
//                side, and K split over a cluster of CTAs.
//
// Measured (device time, calls one after another):
//   75,600 rows 5120 -> 5120, residual and gate: bounded by the tensor cores, 1.84 PFLOP/s while
//     the clock holds (2.16 ms; 2.57 ms, 1.54 PFLOP/s, when the power limit lowers it).
//   6,240 of 20,280 rows 1536 -> 6144, bias and tanh-GELU: 82 us, 1.44 PFLOP/s (87 to 90 with inputs
//     that change from call to call).  As one frame, or in frames of whole tiles, 72 us, and without the
//     activation 66, eight rounds of the 76 pairs: 6 us are the last tiles' activation, which has no
//     products to hide behind, and 10 to 12 the 72 of 600 tiles that lie across frames of 1560 tokens
//     and are loaded in boxes.
//   1 row 1536 -> 9216: 9.4 us, of which reading W's 28 MB takes 4.2: launch, tensor memory,
//     barriers and one cluster's exchange are the rest.
//   333 rows 1000 -> 777: 10.9 us, the same fixed costs.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "rf_deal.h"
#include "rf_ops.h"
#include "rf_rows.cuh"
#include "rf_stage.cuh"
#include "rf_tc_ptx.cuh"

namespace rf {
namespace {

constexpr uint64_t kDrainLimitNs = 200000000ull;  // 0.2 s for what is in flight at teardown
constexpr int kBlockK = 64;                       // columns of K per stage: 128 bytes, one swizzle atom

// ---------------------------------------------------------------------------------------
// Epilogue
// ---------------------------------------------------------------------------------------
struct Epilogue {
  void* Y;
  const void* R;        // or null; elements of Y's type
  const void* bias;     // or null; elements of X's type
  const float* gate;    // or null
  int64_t y_stride, r_stride, gate_stride;  // elements; gate_stride 0: one row for all frames
  int act, in_dtype, out_dtype;
  int n_out;
  int vec;              // Y and R rows, bias and gate can be moved in 16-byte vectors
  int vec_cols;         // bias and gate alone
};

// 1 / x for x of 2^-126 to 2^126, to a unit in the last place; 0 from there on
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// x * sigmoid(s) = x / (1 + h^2) with h = e^(-s / 2) = 2^t.  The denominator is scaled by 2^-22 and its
// reciprocal back, so that it stays in the range of floats where the value does (SiLU to -100; unscaled
// the quotient is 0 from -87.3 down, where the value is -1e-36).
__device__ __forceinline__ float times_sigmoid(float x, float t) {
  constexpr float kScale = 0x1p-22f;
  const float h = ex2_approx(t);
  return x * (kScale * rcp_approx(fmaf(h * kScale, h, kScale)));  // (x 2^-22 could lose digits)
}
// x Phi(x).  The tail Phi(-|x|) = e^(-x^2 / 2) times a function that falls from 1/2 to 0.03 over the
// numbers where it is not yet lost; that one is t Q(t) with t = 1 / (1 + 0.3 |x|) and Q of degree 7,
// fitted for the least largest relative error, 1.3e-7.  So the digits of negative x stay, which
// 1 + erf(x / sqrt 2) loses (4% of the value at -5), up to the rounding of x^2: 8e-6 at -12.  Fewer
// instructions, too: 6240 rows 1536 -> 6144 81 us, with erff 92, with erfcf 143.
__device__ __forceinline__ float gelu(float x) {
  const float t = __fdividef(1.f, fmaf(0.3f, fabsf(x), 1.f));
  float q = 0.035931736f;
  q = fmaf(q, t, -0.158276007f);
  q = fmaf(q, t, 0.208206624f);
  q = fmaf(q, t, -0.0553938560f);
  q = fmaf(q, t, 0.129469201f);
  q = fmaf(q, t, 0.0996374935f);
  q = fmaf(q, t, 0.120798357f);
  q = fmaf(q, t, 0.119626388f);
  const float tail = t * q * ex2_approx(-0.72134752f * (x * x));
  return x * (x < 0.f ? tail : 1.f - tail);
}
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
  switch (act) {
    case RF_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = gelu(v[i]);
      break;
    case RF_ACT_GELU_TANH:  // 0.5 (1 + tanh u) = sigmoid(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3); t = -u log2 e
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[i] = times_sigmoid(v[i], v[i] * fmaf(-0.051471619f, v[i] * v[i], -1.15110411f));
      break;
    case RF_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = times_sigmoid(v[i], -0.72134752f * v[i]);
      break;
    default:
      break;
  }
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, int dtype) {
  if (dtype == RF_FP32) return static_cast<const float*>(p)[i];
  if (dtype == RF_FP16) return __half2float(static_cast<const __half*>(p)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_elem(void* p, int64_t i, int dtype, float v) {
  if (dtype == RF_FP32) static_cast<float*>(p)[i] = v;
  else if (dtype == RF_FP16) static_cast<__half*>(p)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ void unpack2(uint32_t w, int dtype, float& lo, float& hi) {
  if (dtype == RF_FP16) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
  } else {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
  }
}
// lo, hi += the two elements of a word
__device__ __forceinline__ void add2(uint32_t w, int dtype, float& lo, float& hi) {
  float a, b;
  unpack2(w, dtype, a, b);
  lo += a;
  hi += b;
}

// Gate, residual and store of four columns of a row.  VEC: from n on, as vectors; otherwise n,
// n + 32, ...
template <bool VEC>
__device__ __forceinline__ void finish4(const Epilogue& e, int64_t token, int frame, int n, float* v) {
  constexpr int kApart = VEC ? 1 : 32;
  const int64_t at = token * e.y_stride + n, at_r = token * e.r_stride + n;
  const float* g = e.gate ? e.gate + frame * e.gate_stride + n : nullptr;
  if (!VEC || n + 4 > e.n_out) {
    float res[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i * kApart < e.n_out) {
        if (g) v[i] *= g[i * kApart];
        if (e.R) res[i] = load_elem(e.R, at_r + i * kApart, e.out_dtype);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i * kApart < e.n_out)
        store_elem(e.Y, at + i * kApart, e.out_dtype, e.R ? v[i] + res[i] : v[i]);
    return;
  }
  if (g) {
    const float4 x = *reinterpret_cast<const float4*>(g);
    v[0] *= x.x;
    v[1] *= x.y;
    v[2] *= x.z;
    v[3] *= x.w;
  }
  if (e.out_dtype == RF_FP32) {
    if (e.R) {
      const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(e.R) + at_r);
      v[0] += x.x;
      v[1] += x.y;
      v[2] += x.z;
      v[3] += x.w;
    }
    *reinterpret_cast<float4*>(static_cast<float*>(e.Y) + at) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    if (e.R) {
      const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(e.R) + at_r);
      add2(x.x, e.out_dtype, v[0], v[1]);
      add2(x.y, e.out_dtype, v[2], v[3]);
    }
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(e.Y) + at) =
        e.out_dtype == RF_FP16 ? make_uint2(pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]))
                               : make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

// 32 columns from n, element by element: bias, activation, gate.  Out of line: the last columns of
// a result, and bias or gate rows off the 16-byte boundaries.
static __device__ __noinline__ void finish_cols_each(const Epilogue& e, int frame, int n, float (&v)[32]) {
  const int mine = n + (threadIdx.x & 31);  // a column per lane, then handed round
  if (e.bias) {
    const float b = mine < e.n_out ? load_elem(e.bias, mine, e.in_dtype) : 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] += __shfl_sync(0xffffffffu, b, i);
  }
  activate(e.act, v);
  if (e.gate) {
    const int frame0 = __shfl_sync(0xffffffffu, frame, 0);
    if (__all_sync(0xffffffffu, frame == frame0)) {
      const float g = mine < e.n_out ? e.gate[frame0 * e.gate_stride + mine] : 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= __shfl_sync(0xffffffffu, g, i);
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (n + i < e.n_out) v[i] *= e.gate[frame * e.gate_stride + n + i];
    }
  }
}

// 32 columns from n: bias, activation, gate.
__device__ __forceinline__ void finish_cols(const Epilogue& e, int frame, int n, float (&v)[32]) {
  if (e.bias) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(e.bias) + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w = q[i];
      add2(w.x, e.in_dtype, v[8 * i], v[8 * i + 1]);
      add2(w.y, e.in_dtype, v[8 * i + 2], v[8 * i + 3]);
      add2(w.z, e.in_dtype, v[8 * i + 4], v[8 * i + 5]);
      add2(w.w, e.in_dtype, v[8 * i + 6], v[8 * i + 7]);
    }
  }
  activate(e.act, v);
  if (e.gate) {
    const float4* q = reinterpret_cast<const float4*>(e.gate + frame * e.gate_stride + n);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 g = q[i];
      v[4 * i] *= g.x;
      v[4 * i + 1] *= g.y;
      v[4 * i + 2] *= g.z;
      v[4 * i + 3] *= g.w;
    }
  }
}

// A warp's 32 rows of an accumulator (tensor memory columns from `acc`; a row per lane, its token
// or -1), columns n0 .. n0 + cols - 1 of the result, 128 bytes of them at a time through the warp's
// stage.  ready() is called when the residual's first loads are in flight and the accumulator is
// wanted, read() when it has been read; false from ready() ends it.
template <bool OUT32, typename Ready, typename Read>
__device__ __forceinline__ bool finish_tile(const Epilogue& e, const CUtensorMap* tmY,
                                            uint4* stage, uint32_t acc, int n0, int cols,
                                            int64_t token, int frame, Ready&& ready, Read&& read) {
  constexpr int kCols = OUT32 ? 32 : 64, kBytes = OUT32 ? 4 : 2;
  const int chunks = (min(cols, max(e.n_out - n0, 0)) + kCols - 1) / kCols;
  const int64_t y_bytes = e.y_stride * kBytes, r_bytes = e.r_stride * kBytes;
  const RowSpan span_y = row_span(token < 0 ? -1 : token * y_bytes, y_bytes);
  const RowSpan span_r = row_span(token < 0 ? -1 : token * r_bytes, r_bytes);
  char* Y = static_cast<char*>(e.Y) + static_cast<int64_t>(n0) * kBytes;
  const char* R = static_cast<const char*>(e.R) + static_cast<int64_t>(n0) * kBytes;
  const int lane = threadIdx.x & 31;
  auto stage_free = [&]() {
    if (lane == 0) bulk_wait_read();
    __syncwarp();
  };
  auto in_full = [&](int c) { return n0 + (c + 1) * kCols <= e.n_out; };
  auto whole = [&](int c) { return e.vec && in_full(c); };
  auto fetch = [&](int c) {  // the residual's rows, ahead of their use
    stage_free();
    if (whole(c)) fetch_rows(stage, R + c * 128, span_r, r_bytes);
    else fetch_elems<kBytes>(stage, R + c * 128, span_r.at, e.n_out - n0 - c * kCols);
  };
  // 32 consecutive tokens leave through TMA, in the background
  const bool bulk = span_y.regular && span_y.n == 32;
  const int token0 = __shfl_sync(0xffffffffu, static_cast<int>(token), 0);
  if (e.R && chunks > 0) fetch(0);
  if (!ready()) return false;
  if (chunks == 0) read();
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    const int n = n0 + c * kCols;
#pragma unroll 1
    for (int half = 0; half < kCols / 32; ++half) {
      float v[32];
      tmem_ld32(acc + c * kCols + half * 32, reinterpret_cast<uint32_t(&)[32]>(v));
      tmem_wait_ld();
      if (half == kCols / 32 - 1 && c == chunks - 1) read();
      if (e.vec_cols && in_full(c)) {
        finish_cols(e, frame, n + half * 32, v);
      } else {
        float t[32];  // its address is taken: v stays in registers
#pragma unroll
        for (int i = 0; i < 32; ++i) t[i] = v[i];
        finish_cols_each(e, frame, n + half * 32, t);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = t[i];
      }
      if (half == 0) {
        if (e.R) await_rows();
        else stage_free();
      }
#pragma unroll
      for (int q = 0; q < (OUT32 ? 8 : 4); ++q) {
        // the residual's piece of this lane's row makes way for the result's
        uint4& piece = stage_at(stage, lane, half * 4 + q);
        if (OUT32) {
          float* x = v + 4 * q;
          if (e.R) {
            const uint4 r = piece;
            x[0] += __uint_as_float(r.x);
            x[1] += __uint_as_float(r.y);
            x[2] += __uint_as_float(r.z);
            x[3] += __uint_as_float(r.w);
          }
          piece = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                             __float_as_uint(x[3]));
        } else {
          float* x = v + 8 * (q & 3);
          if (e.R) {
            const uint4 r = piece;
            add2(r.x, e.out_dtype, x[0], x[1]);
            add2(r.y, e.out_dtype, x[2], x[3]);
            add2(r.z, e.out_dtype, x[4], x[5]);
            add2(r.w, e.out_dtype, x[6], x[7]);
          }
          piece = e.out_dtype == RF_FP16
                      ? make_uint4(pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]),
                                   pack_f16x2(x[4], x[5]), pack_f16x2(x[6], x[7]))
                      : make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                   pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
        }
      }
    }
    if (!whole(c)) {
      store_elems<kBytes>(stage, Y + c * 128, span_y.at, e.n_out - n);
    } else if (bulk) {
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        tma_store_2d(tmY, smem_u32(stage), n, token0);
        bulk_commit();
      }
    } else {
      store_rows(stage, Y + c * 128, span_y, y_bytes);
    }
    if (e.R && c + 1 < chunks) fetch(c + 1);
  }
  return true;
}

struct LinearParams {
  RowMap rows;
  Epilogue epi;
  FastDiv by_N;  // tokens per frame, for the gate's row (without a list rows.N is all tokens)
  int kblocks, n_tiles, fp16;
  int32_t* status;
  // split_kernel
  int tile_tokens, cluster, stages;
  int tile_rows;  // rows of a tile of split_kernel, or of a CTA's half of a pair's
};

__device__ __forceinline__ void flag_error(const LinearParams& p, int where) {
  if (p.status) atomicOr(p.status, RF_ERR_DEVICE_TIMEOUT | (1 << (8 + where)));
}

// Token and frame of row r (r < rows of the launch); token -1 in a frame's padding.
__device__ __forceinline__ int row_token(const LinearParams& p, int r, int& frame) {
  const int a = p.rows.by_Np.div(r), q = r - a * p.rows.Np;
  const int f = p.rows.frame(a);
  const int token = f * p.rows.N + q;
  const bool valid = q < p.rows.N;
  frame = valid ? p.by_N.div(token) : 0;  // the padding behind the last frame is in none
  return valid ? token : -1;
}

// The maps of X: boxes of a whole tile, of kBoxRows rows and of rows.unit rows.
struct RowMaps {
  const CUtensorMap *whole, *many, *unit;
};
// Issue the copies of one k block of a tile's rows (one thread of each of the `of` warps they are dealt
// to; a whole tile's box is the last one's).  The barrier's one arrival carries the bytes of all of
// them and holds its phase open: copies of other warps, and of a pair's second CTA, may land before
// it, and count below zero until then.  So the arrival is never parted from the count of bytes.
template <bool PAIR, int CAP>
__device__ __forceinline__ void load_rows(const RowBoxes& x, const BoxList<CAP>& list,
                                          const RowMaps& maps, uint32_t dst, uint32_t bar, int k0,
                                          int who, int of) {
  auto load = [&](const CUtensorMap* m, int row, int tok) {
    if (PAIR) tma_load_2d_pair(dst + row * 128, m, bar, k0, tok);
    else tma_load_2d(dst + row * 128, m, bar, k0, tok);
  };
  if (x.n_many + x.n_unit == 0) {
    if (who == of - 1) load(maps.whole, 0, x.tok);
    return;
  }
  Deal mine{who, of};
#pragma unroll 1
  while (mine.more(x.n_many)) {
    const int i = mine.take();
    load(maps.many, list.row[i], list.tok[i]);
  }
#pragma unroll 1
  while (mine.more(x.n_many + x.n_unit)) {
    const int i = CAP - 1 - (mine.take() - x.n_many);
    load(maps.unit, list.row[i], list.tok[i]);
  }
}

// ---------------------------------------------------------------------------------------
// Many rows: pairs of CTAs
// ---------------------------------------------------------------------------------------
// A pair's tile is 256 tokens x kBN columns: each CTA holds 128 token rows of X, half of the tile's
// rows of W, and the accumulators of its 128 rows; the tensor cores of both read both halves of W.
// That is what the pair is for: a CTA alone on 128 x 256 would have to bring 48 KB into shared
// memory per 64 columns of K, in a pair it brings 32 KB.
// Two accumulators in tensor memory: the epilogue of a tile runs during the products of the next.
constexpr int kPairThreads = 384;  // warps 0, 3 TMA, 1 MMA (first CTA), 2 tensor memory, 4-11 epilogue
constexpr int kEpiWarps = 8;
constexpr int kBN = 256;

struct PairCfg {
  static constexpr int kABytes = 128 * 128, kBBytes = kBN / 2 * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = 196608 / kStageBytes;
  static constexpr int kBarFull = 0, kBarEmpty = kStages, kBarAccFull = 2 * kStages,
                       kBarAccEmpty = kBarAccFull + 2, kBars = kBarAccEmpty + 2;
  static constexpr int kOffStage = kStages * kStageBytes;  // rows of results, per epilogue warp
  static constexpr int kOffBar = kOffStage + kEpiWarps * kTurnBytes;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kOffList = kOffMisc + 16;
  static constexpr int kSmem = kOffList + 2 * static_cast<int>(sizeof(BoxList<128>)) + 1024;
  static constexpr uint32_t kTmemCols = 2 * kBN;
};

// Tiles in groups of eight rows of tiles, column by column within a group, so that the pairs at
// work share rows of X and of W in L2.
constexpr int kGroupM = 8;
__device__ __forceinline__ void tile_at(int t, int m_tiles, int n_tiles, int& m, int& n) {
  const int per_group = kGroupM * n_tiles;
  const int g = t / per_group, i = t - g * per_group;
  const int width = min(kGroupM, m_tiles - g * kGroupM);
  n = i / width;
  m = g * kGroupM + (i - n * width);
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmMany,
                const __grid_constant__ CUtensorMap tmUnit, const __grid_constant__ CUtensorMap tmW,
                const __grid_constant__ CUtensorMap tmY, const LinearParams p) {
  using C = PairCfg;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw);
  const uint32_t bar0 = sbase + C::kOffBar;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar(C::kBarFull + s), 1);
      mbar_init(bar(C::kBarEmpty + s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar(C::kBarAccFull + b), 1);
      mbar_init(bar(C::kBarAccEmpty + b), 2 * kEpiWarps);
    }
    *abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmW);
  }
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();  // the other CTA's barriers are initialised, its tensor memory allocated
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)

  const int R = p.rows.frames() * p.rows.Np;
  const int half = p.tile_rows;  // rows of a CTA's half of a tile
  const int m_tiles = (R + 2 * half - 1) / (2 * half);
  const int tiles = m_tiles * p.n_tiles;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0 || warp == 3) {
    // two warps: the boxes of a tile across frames are seven or more for each 64 columns of K, and
    // one warp does not issue them in the 512 cycles that the products take
    const bool lead = elect_one();
    const int who = warp == 3;
    BoxList<128>& list = reinterpret_cast<BoxList<128>*>(smem + C::kOffList)[who];
    int it = 0;
    bool ok = true;
    for (int t = pair; ok && t < tiles; t += pairs) {
      int m, n;
      tile_at(t, m_tiles, p.n_tiles, m, n);
      const RowBoxes x = list_boxes(p.rows, R, (2 * m + rank) * half, half, 128, list);
      const int w0 = n * kBN + rank * (kBN / 2);
      // of both CTAs, the other one's rows included
      const int bytes = 2 * C::kBBytes +
                        (x.rows + (rank == 0 ? boxed_rows(p.rows, R, (2 * m + 1) * half, half, 128)
                                             : 0)) * 128;
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const int s = it % C::kStages;
        if (!warp_wait<true>(bar(C::kBarEmpty + s), ((it / C::kStages) & 1) ^ 1, abort)) {
          if (lead) flag_error(p, 0);
          ok = false;
          break;
        }
        // the first CTA's barrier counts the bytes of both
        const uint32_t full = map_to_rank(bar(C::kBarFull + s), 0);
        const uint32_t dst = sbase + s * C::kStageBytes;
        if (lead) {
          if (who == 0) {
            if (rank == 0) mbar_arrive_expect_tx(bar(C::kBarFull + s), bytes);
            tma_load_2d_pair(dst + C::kABytes, &tmW, full, kb * kBlockK, w0);
          }
          load_rows<true>(x, list, {&tmX, &tmMany, &tmUnit}, dst, full, kb * kBlockK, who, 2);
        }
        __syncwarp();
      }
    }
    // every stage that was filled has been given back (so no arrival from the other CTA is still
    // to come) before this CTA may leave; after a wait that gave up, the copies in flight get time
#pragma unroll 1
    for (int s = 0; s < C::kStages; ++s)
      if (it > s)
        mbar_drain(bar(C::kBarEmpty + s), ((it - 1 - s) / C::kStages) & 1, kDrainLimitNs);
  } else if (warp == 1) {
    if (rank == 0) {
      const bool lead = elect_one();
      const uint32_t idesc = idesc_f16(p.fp16, 256, kBN, 0);
      int it = 0, n_acc = 0;
      bool ok = true;
      for (int t = pair; ok && t < tiles; t += pairs, ++n_acc) {
        const int b = n_acc & 1;
        if (!warp_wait<true>(bar(C::kBarAccEmpty + b), ((n_acc >> 1) & 1) ^ 1, abort)) {
          if (lead) flag_error(p, 1);
          break;
        }
        tc_fence_after();
        const uint32_t acc = tmem + b * kBN;
        for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
          const int s = it % C::kStages;
          if (!warp_wait<true>(bar(C::kBarFull + s), (it / C::kStages) & 1, abort)) {
            if (lead) flag_error(p, 2);
            ok = false;
            break;
          }
          tc_fence_after();
          if (lead) {
            const uint32_t sA = sbase + s * C::kStageBytes;
            const uint64_t dA = smem_desc_sw128(sA, 16, 1024);
            const uint64_t dB = smem_desc_sw128(sA + C::kABytes, 16, 1024);
#pragma unroll
            for (int k = 0; k < kBlockK / 16; ++k)
              tc_mma_ss_pair(acc, dA + k * 2, dB + k * 2, idesc, (kb | k) != 0);
            tc_commit_pair(bar(C::kBarEmpty + s));
            if (kb == p.kblocks - 1) tc_commit_pair(bar(C::kBarAccFull + b));
          }
          __syncwarp();
        }
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, part = (warp - 4) >> 2;  // lanes of tensor memory; half of kBN
    const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
    uint4* stage = reinterpret_cast<uint4*>(smem + C::kOffStage + (warp - 4) * kTurnBytes);
    int n_acc = 0;
    for (int t = pair; t < tiles; t += pairs, ++n_acc) {
      int m, n;
      tile_at(t, m_tiles, p.n_tiles, m, n);
      const int b = n_acc & 1;
      const int row = quarter * 32 + lane, r = (2 * m + rank) * half + row;
      int frame = 0;
      const int token = row < half && r < R ? row_token(p, r, frame) : -1;
      auto ready = [&]() -> bool {
        const bool ok = warp_wait<true>(bar(C::kBarAccFull + b), (n_acc >> 1) & 1, abort);
        if (!ok && lane == 0) flag_error(p, 3);
        tc_fence_after();
        return ok;
      };
      auto read = [&]() {  // the accumulator may be written again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(bar(C::kBarAccEmpty + b), 0));
      };
      const uint32_t acc = tmem + lane_base + b * kBN + part * (kBN / 2);
      const int n0 = n * kBN + part * (kBN / 2);
      if (!(p.epi.out_dtype == RF_FP32
                ? finish_tile<true>(p.epi, &tmY, stage, acc, n0, kBN / 2, token, frame, ready, read)
                : finish_tile<false>(p.epi, &tmY, stage, acc, n0, kBN / 2, token, frame, ready, read)))
        break;
    }
    if (lane == 0) bulk_wait_all();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_arrive();  // nothing of the other CTA's refers to this CTA's memory any more
  cluster_wait();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, C::kTmemCols);
  }
}

// ---------------------------------------------------------------------------------------
// Few rows: W as the M side, K split over a cluster
// ---------------------------------------------------------------------------------------
// A tile is 128 columns of the result (rows of W: the tensor core's M side) x tile_tokens tokens
// (its N side, 16 to 256), so that one token costs a sixteenth of a tile and not all of it.  The
// CTAs of a cluster take equal ranges of K; each leaves its sums in shared memory, and each
// finishes its share of the tile's tokens from all of them, in the order of the ranges.
constexpr int kSplitThreads = 256;  // warp 0 TMA, 1 MMA, 2 tensor memory, 4-7 read the accumulator
constexpr int kSplitMaxStages = 12;
constexpr int kSplitRing = 212992;  // bytes for stages; the sums of a split take their place
constexpr int kSplitBarFull = 0, kSplitBarEmpty = kSplitMaxStages,
              kSplitBarAcc = 2 * kSplitMaxStages, kSplitBars = kSplitBarAcc + 1;
constexpr int kSplitOffBar = kSplitRing, kSplitOffMisc = kSplitOffBar + kSplitBars * 8,
              kSplitOffBoxes = kSplitOffMisc + 16,
              kSplitOffTok = kSplitOffBoxes + 16, kSplitOffList = kSplitOffTok + 256 * 8,
              kSplitSmem = kSplitOffList + sizeof(BoxList<256>) + 1024;

// Results of a CTA's share of a tile's tokens from the sums of all CTAs: a warp has kTok tokens at
// a time, a lane four columns of each, with the loads of all of them in flight.  VEC: neighbouring
// columns, moved as vectors; otherwise every 32nd, so that a warp's accesses are of consecutive
// elements either way.
template <bool VEC>
__device__ __forceinline__ void finish_tokens(const Epilogue& e, const int2* tokens, uint32_t sums,
                                              int n0, int BT, int rows, int rank, int C) {
  constexpr int kTok = 4, kApart = VEC ? 1 : 32;
  const int lane = threadIdx.x & 31, col = VEC ? 4 * lane : lane, out = n0 + col;
  if (out >= e.n_out) return;
  float bias[4] = {};
  if (e.bias)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (out + i * kApart < e.n_out) bias[i] = load_elem(e.bias, out + i * kApart, e.in_dtype);
  const int step = kSplitThreads / 32 * C;  // between a warp's tokens
#pragma unroll 1
  for (int j0 = kSplitThreads / 32 * rank + (threadIdx.x >> 5); j0 < rows; j0 += kTok * step) {
    int2 t[kTok];
    float v[kTok * 4];
#pragma unroll
    for (int u = 0; u < kTok; ++u) {
      const int j = j0 + u * step;
      t[u] = j < BT ? tokens[j] : make_int2(-1, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * u + i] = bias[i];
    }
    const uint32_t at = sums + (j0 * 128 + col) * 4;
#pragma unroll 2
    for (int c = 0; c < C; ++c) {
      const uint32_t base = C > 1 ? map_to_rank(at, c) : at;
#pragma unroll
      for (int u = 0; u < kTok; ++u)
        if (t[u].x >= 0) {
          const uint32_t from = base + u * step * 512;
          if (VEC) {
            const float4 x = ld_cluster_f4(from);
            v[4 * u] += x.x;
            v[4 * u + 1] += x.y;
            v[4 * u + 2] += x.z;
            v[4 * u + 3] += x.w;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * u + i] += ld_cluster_f(from + 128 * i);
          }
        }
    }
    activate(e.act, v);
#pragma unroll
    for (int u = 0; u < kTok; ++u)
      if (t[u].x >= 0) finish4<VEC>(e, t[u].x, t[u].y, out, v + 4 * u);
  }
}

__global__ void __launch_bounds__(kSplitThreads, 1)
    split_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmMany,
                 const __grid_constant__ CUtensorMap tmUnit, const __grid_constant__ CUtensorMap tmW,
                 const LinearParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw);
  const uint32_t bar0 = sbase + kSplitOffBar;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kSplitOffMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(smem + kSplitOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int BT = p.tile_tokens, C = p.cluster;
  const int rank = C > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int tile = blockIdx.x / C;
  const int m = tile / p.n_tiles, n = tile - m * p.n_tiles;
  const int stage_bytes = 16384 + BT * 128;
  const uint32_t tmem_cols = BT < 32 ? 32 : BT;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(bar(kSplitBarFull + s), 1);
      mbar_init(bar(kSplitBarEmpty + s), 1);
    }
    mbar_init(bar(kSplitBarAcc), 1);
    *abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmW);
  }
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const int R = p.rows.frames() * p.rows.Np;
  const int r0 = m * p.tile_rows, rows = min(p.tile_rows, R - r0);
  if (r0 >= R) return;  // the whole cluster
  BoxList<256>& list = *reinterpret_cast<BoxList<256>*>(smem + kSplitOffList);
  RowBoxes* boxes = reinterpret_cast<RowBoxes*>(smem + kSplitOffBoxes);
  if (warp == 2) {
    tmem_alloc(smem_u32(tmem_slot), tmem_cols);
    tmem_relinquish();
  } else if (warp == 3) {
    const RowBoxes x = list_boxes(p.rows, R, r0, p.tile_rows, BT, list);
    if (lane == 0) *boxes = x;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int kb0 = p.kblocks * rank / C, kb1 = p.kblocks * (rank + 1) / C;

  const RowBoxes x = *boxes;
  // the boxes of a tile across frames are dealt to all warps but the MMA warp: one warp would take
  // a hundred cycles for each (33 frames of one token, 1536 -> 6144: 29 us, this way 16); a warp
  // without a box stays out, as nothing would keep the ring from passing it
  const int loaders = loading_warps(x.n_many + x.n_unit, kSplitThreads / 32 - 1);
  const int who = warp == 0 ? 0 : warp - 1;
  if (warp != 1 && who < loaders) {
    const bool lead = elect_one();
    int it = 0;
#pragma unroll 1
    for (int kb = kb0; kb < kb1; ++kb, ++it) {
      const int s = it % p.stages;
      if (!warp_wait<false>(bar(kSplitBarEmpty + s), ((it / p.stages) & 1) ^ 1, abort)) {
        if (lead) flag_error(p, 0);
        break;
      }
      const uint32_t dst = sbase + s * stage_bytes;
      if (lead) {
        if (who == 0) {
          mbar_arrive_expect_tx(bar(kSplitBarFull + s), 16384 + x.rows * 128);
          tma_load_2d(dst, &tmW, bar(kSplitBarFull + s), kb * kBlockK, n * 128);
        }
        load_rows<false>(x, list, {&tmX, &tmMany, &tmUnit}, dst + 16384,
                         bar(kSplitBarFull + s), kb * kBlockK, who, loaders);
      }
      __syncwarp();
    }
    if (who == 0)
#pragma unroll 1
      for (int s = 0; s < p.stages; ++s)  // every copy has landed
        if (it > s) mbar_drain(bar(kSplitBarFull + s), ((it - 1 - s) / p.stages) & 1, kDrainLimitNs);
  } else if (warp == 1) {
    const bool lead = elect_one();
    const uint32_t idesc = idesc_f16(p.fp16, 128, BT, 0);
    int it = 0;
    for (int kb = kb0; kb < kb1; ++kb, ++it) {
      const int s = it % p.stages;
      if (!warp_wait<false>(bar(kSplitBarFull + s), (it / p.stages) & 1, abort)) {
        if (lead) flag_error(p, 1);
        break;
      }
      tc_fence_after();
      if (lead) {
        const uint32_t sA = sbase + s * stage_bytes;
        const uint64_t dA = smem_desc_sw128(sA, 16, 1024), dB = smem_desc_sw128(sA + 16384, 16, 1024);
#pragma unroll
        for (int k = 0; k < kBlockK / 16; ++k)
          tc_mma_ss(tmem, dA + k * 2, dB + k * 2, idesc, (it | k) != 0);
        tc_commit(bar(kSplitBarEmpty + s));
      }
      __syncwarp();
    }
    // all MMAs issued are done (also after a wait that gave up: tensor memory is freed below)
    if (lead) tc_commit(bar(kSplitBarAcc));
    __syncwarp();
    mbar_drain(bar(kSplitBarAcc), 0, kDrainLimitNs);
  }
  float* sums = reinterpret_cast<float*>(smem);  // [BT][128]
  int2* tokens = reinterpret_cast<int2*>(smem + kSplitOffTok);  // {token, frame}
  if (warp >= 4) {
    const int quarter = warp & 3;
#pragma unroll 1
    for (int j = threadIdx.x - 128; j < BT; j += 128) {
      int2 t = make_int2(-1, 0);
      if (j < rows) t.x = row_token(p, r0 + j, t.y);
      tokens[j] = t;
    }
    const bool ok = warp_wait<false>(bar(kSplitBarAcc), 0, abort);
    if (!ok && lane == 0) flag_error(p, 2);
    tc_fence_after();
#pragma unroll 1
    for (int c = 0; ok && c < BT; c += 32) {
      uint32_t v[32];
      tmem_ld32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + c, v);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (c + i < BT) sums[(c + i) * 128 + quarter * 32 + lane] = __uint_as_float(v[i]);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (C > 1) {
    cluster_arrive();
    cluster_wait();
  }
  if (p.epi.vec) finish_tokens<true>(p.epi, tokens, sbase, n * 128, BT, rows, rank, C);
  else finish_tokens<false>(p.epi, tokens, sbase, n * 128, BT, rows, rank, C);
  __syncwarp();
  if (C > 1) {
    cluster_arrive();  // every CTA has read the others' sums
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, tmem_cols);
  }
}

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------
template <typename K>
rf_status set_smem(K kernel, int bytes, const DeviceInfo& di, std::atomic<bool> (&done)[64]) {
  if (bytes > di.max_smem_optin) return fail(RF_ERR_UNSUPPORTED, "rf_linear: shared memory");
  if (!done[di.device]) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             bytes))
      return fail(RF_ERR_CUDA, "cudaFuncSetAttribute(rf_linear)", e);
    done[di.device] = true;
  }
  return RF_OK;
}

rf_status map_2d(CUtensorMap* m, int dtype, const void* base, int cols, int64_t rows,
                 int64_t row_stride, int box_rows) {
  const uint64_t dims[2] = {static_cast<uint64_t>(cols), static_cast<uint64_t>(rows)};
  const uint64_t strides[1] = {static_cast<uint64_t>(row_stride) * 2};
  const uint32_t box[2] = {kBlockK, static_cast<uint32_t>(box_rows)};
  return make_tensor_map(m, dtype, base, 2, dims, strides, box);
}

// Tokens per tile and CTAs per cluster of a split launch: the pair with the least to do for the
// busiest SM, in cycles.  Per 64 columns of K a CTA loads its tile of W and of X at about 50 bytes
// per cycle (its products take 2 cycles per token, less); start and end cost about 5000, a
// cluster's start and its two barriers 750 per CTA, and each four tokens of a warp one round trip
// per CTA of the cluster, 700 cycles and 150 for every further CTA.  Clusters of 4 and 8 do not
// fill the GPCs: 36 and 15 of them run together. (333 rows 1000 -> 777: 10.8 us in tiles of 16
// tokens, 14.0 in tiles of 256 and clusters of eight.)
struct SplitPlan {
  int tokens, cluster;
};
SplitPlan split_plan(int64_t rows, int unit, int64_t n128, int kblocks, int sms) {
  SplitPlan best{256, 1};
  double least = 0;
  for (int bt = 16; bt <= 256; bt *= 2) {
    for (int c = 1; c <= 8 && c <= kblocks; c *= 2) {
      const int tile = tile_rows(unit, bt);
      const int64_t ctas = (rows + tile - 1) / tile * n128 * c;
      const int64_t at_once = c == 8 ? sms * 120 / 152 : c == 4 ? sms * 144 / 152 : sms;
      const int64_t rounds = (ctas + at_once - 1) / at_once;
      const int join = (bt + 32 * c - 1) / (32 * c);  // groups of four tokens of a warp
      const double one = 5000.0 + (kblocks + c - 1) / c * ((16384.0 + 128.0 * bt) / 50) +
                         join * (700.0 + 150.0 * (c - 1)) + (c > 1 ? 750 * c : 0);
      const double cost = static_cast<double>(rounds) * one;
      if (least == 0 || cost < least) {
        least = cost;
        best = {bt, c};
      }
    }
    if (tile_rows(unit, bt) >= rows) break;
  }
  return best;
}

struct Maps {
  CUtensorMap x, many, unit, w, y;
};
// The maps of a launch with tiles of `tile` rows of X; w_rows rows of W per box.  Boxes of part of
// a tile are made where a tile can lie across frames.
rf_status make_maps(Maps* t, const LinearParams& p, const void* d_X, int64_t x_stride,
                    const void* d_W, int64_t w_stride, int d_in, int tile, int w_rows) {
  const int dt = p.epi.in_dtype;
  if (rf_status st = map_2d(&t->x, dt, d_X, d_in, p.rows.T, x_stride, tile)) return st;
  if (rf_status st = map_2d(&t->w, dt, d_W, d_in, p.epi.n_out, w_stride, w_rows)) return st;
  t->many = t->unit = t->x;
  if (p.rows.F == 1) return RF_OK;
  if (p.rows.unit > 1 && p.rows.Np >= kBoxRows)
    if (rf_status st = map_2d(&t->many, dt, d_X, d_in, p.rows.T, x_stride, kBoxRows)) return st;
  return map_2d(&t->unit, dt, d_X, d_in, p.rows.T, x_stride, p.rows.unit);
}

rf_status launch_pair(const Maps& t, const LinearParams& p, int64_t tiles, const DeviceInfo& di,
                      cudaStream_t s) {
  static std::atomic<bool> done[64] = {};
  if (rf_status st = set_smem(pair_kernel, PairCfg::kSmem, di, done)) return st;
  // pairs that run together: where a GPC has an odd number of free SMs it is fewer than half of
  // them, and a pair that waits for the others to finish would double the time
  static std::atomic<int> resident[64] = {};
  int most = resident[di.device].load(std::memory_order_relaxed);
  if (most == 0) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(di.sm_count / 2 * 2));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = PairCfg::kSmem;
    if (cudaError_t e = cudaOccupancyMaxActiveClusters(&most, pair_kernel, &cfg))
      return fail(RF_ERR_CUDA, "cudaOccupancyMaxActiveClusters(rf_linear)", e);
    if (most < 1) return fail(RF_ERR_UNSUPPORTED, "rf_linear: no room for a pair of CTAs");
    resident[di.device].store(most, std::memory_order_relaxed);
  }
  const int64_t pairs = std::min<int64_t>(tiles, most);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = PairCfg::kSmem;
  cfg.stream = s;
  return launch_early(cfg, 1, "rf_linear pair_kernel launch", pair_kernel, t.x, t.many, t.unit, t.w,
                      t.y, p);
}

rf_status launch_split(const Maps& t, const LinearParams& p, int64_t tiles, const DeviceInfo& di,
                       cudaStream_t s) {
  static std::atomic<bool> done[64] = {};
  if (rf_status st = set_smem(split_kernel, kSplitSmem, di, done)) return st;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * p.cluster));
  cfg.blockDim = dim3(kSplitThreads);
  cfg.dynamicSmemBytes = kSplitSmem;
  cfg.stream = s;
  return launch_early(cfg, p.cluster, "rf_linear split_kernel launch", split_kernel, t.x, t.many,
                      t.unit, t.w, p);
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" rf_status rf_linear(void* d_Y, int64_t y_row_stride, int out_dtype, const void* d_X,
                               int64_t x_row_stride, const void* d_W, int64_t w_row_stride,
                               int dtype, int F, int N, int d_in, int d_out, const void* d_bias,
                               int act, const float* d_gate, int64_t gate_frame_stride,
                               const void* d_R, int64_t r_row_stride, const int32_t* d_active,
                               const int32_t* d_counts, int32_t* d_status, rf_stream_t stream) {
  if (!d_Y || !d_X || !d_W) return fail(RF_ERR_INVALID_ARG, "rf_linear: null pointer");
  if (dtype != RF_BF16 && dtype != RF_FP16) return fail(RF_ERR_UNSUPPORTED, "rf_linear: dtype");
  if (out_dtype != dtype && out_dtype != RF_FP32)
    return fail(RF_ERR_UNSUPPORTED, "rf_linear: output in the inputs' type or fp32");
  if (F < 1 || N < 1 || d_in < 1 || d_out < 1)
    return fail(RF_ERR_INVALID_ARG, "rf_linear: sizes >= 1");
  if (act < RF_ACT_NONE || act > RF_ACT_SILU) return fail(RF_ERR_INVALID_ARG, "rf_linear: act");
  if (x_row_stride < d_in || w_row_stride < d_in || y_row_stride < d_out ||
      (d_R && r_row_stride < d_out) || (d_gate && gate_frame_stride != 0 && gate_frame_stride < d_out))
    return fail(RF_ERR_INVALID_ARG, "rf_linear: row stride below the row's length");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "rf_linear: active list and counts come together");
  if (d_R == d_Y && r_row_stride != y_row_stride && static_cast<int64_t>(F) * N > 1)
    return fail(RF_ERR_INVALID_ARG, "rf_linear: in place with two strides");
  // (a row by itself has no stride that matters: the tensor map gets one on a boundary)
  if (static_cast<int64_t>(F) * N == 1) x_row_stride = (x_row_stride + 7) / 8 * 8;
  if (d_out == 1) w_row_stride = (w_row_stride + 7) / 8 * 8;
  if (!aligned16(d_X) || !aligned16(d_W) || x_row_stride % 8 || w_row_stride % 8)
    return fail(RF_ERR_MISALIGNED, "rf_linear: X and W rows on 16-byte boundaries");
  const int es_out = dtype_bytes(out_dtype);
  if (reinterpret_cast<uintptr_t>(d_Y) % es_out || reinterpret_cast<uintptr_t>(d_R) % es_out ||
      reinterpret_cast<uintptr_t>(d_bias) % 2 || reinterpret_cast<uintptr_t>(d_gate) % 4)
    return fail(RF_ERR_MISALIGNED, "rf_linear: pointer not on its elements' boundary");
  // without a list the tokens are one frame, with nothing between them
  const int64_t T = static_cast<int64_t>(F) * N;
  const int64_t Fr = d_active ? F : 1, Nr = d_active ? N : T;
  const int unit = row_unit(Nr);
  const int64_t Np = (Nr + unit - 1) / unit * unit;
  if (T > 0x7FFFFFFF - 65536 || Fr * Np > 0x7FFFFFFF - 65536 || d_out > 0x7FFFFFFF - 65536 ||
      d_in > 0x7FFFFFFF - 65536)
    return fail(RF_ERR_INVALID_ARG, "rf_linear: too many tokens or columns");
  DeviceInfo di;
  if (rf_status st = current_device_info(&di)) return st;
  if (di.cc_major != 10 || di.cc_minor != 3) return fail(RF_ERR_UNSUPPORTED, "needs sm_103");

  LinearParams p{};
  p.rows = {d_active, d_counts, static_cast<int>(Fr), static_cast<int>(Nr), static_cast<int>(Np), unit,
            static_cast<int>(T), FastDiv(static_cast<uint32_t>(Np))};
  Epilogue& e = p.epi;
  e.Y = d_Y;
  e.R = d_R;
  e.bias = d_bias;
  e.gate = d_gate;
  e.y_stride = y_row_stride;
  e.r_stride = r_row_stride;
  e.gate_stride = gate_frame_stride;
  e.act = act;
  e.in_dtype = dtype;
  e.out_dtype = out_dtype;
  e.n_out = d_out;
  e.vec_cols = aligned16(d_bias) && (!d_gate || (aligned16(d_gate) && gate_frame_stride % 4 == 0));
  e.vec = e.vec_cols && aligned16(d_Y) && y_row_stride * es_out % 16 == 0 &&
          (!d_R || (aligned16(d_R) && r_row_stride * es_out % 16 == 0));
  p.by_N = FastDiv(static_cast<uint32_t>(N));
  p.kblocks = (d_in + kBlockK - 1) / kBlockK;
  p.fp16 = dtype == RF_FP16;
  p.status = d_status;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);

  const int64_t rows = Fr * Np;  // at most: the active count is known on the device only
  const int64_t n256 = (d_out + 255) / 256, n128 = (d_out + 127) / 128;
  const int half = tile_rows(unit, 128);
  const int64_t pair_tiles = (rows + 2 * half - 1) / (2 * half) * n256;
  // Pairs of CTAs once their tiles occupy half of the 76 pairs (us, pair against split):
  //   tiles 30: 3600 rows 5120 ->  512 34.5 / 26.3     40:  512 rows 5120 -> 5120 35.9 / 45.2
  //         32: 1024 rows 1024 -> 2048 17.8 / 16.7     42: 1560 rows 1536 -> 1536 19.7 / 27.7
  //         32: 2048 rows  256 -> 1024 14.5 / 13.0     48:  384 rows 1536 -> 6144 19.8 / 18.8
  //         36:  256 rows 1536 -> 9216 20.0 / 18.2     48:  512 rows 1536 -> 6144 19.9 / 27.3
  // Up to 256 rows it is one row of tiles, and the bytes of W: for the split, whatever the width.
  Maps t;
  if (rows > 256 && pair_tiles >= di.sm_count / 4) {
    p.n_tiles = static_cast<int>(n256);
    p.tile_rows = half;
    if (rf_status st = make_maps(&t, p, d_X, x_row_stride, d_W, w_row_stride, d_in, 128, 128)) return st;
    t.y = t.x;
    if (e.vec) {  // 128 bytes of 32 rows
      const uint64_t dims[2] = {static_cast<uint64_t>(d_out), static_cast<uint64_t>(T)};
      const uint64_t strides[1] = {static_cast<uint64_t>(y_row_stride) * es_out};
      const uint32_t box[2] = {128u / es_out, 32};
      if (rf_status st = make_tensor_map(&t.y, out_dtype, d_Y, 2, dims, strides, box)) return st;
    }
    return launch_pair(t, p, pair_tiles, di, s);
  }
  const SplitPlan plan = split_plan(rows, unit, n128, p.kblocks, di.sm_count);
  const int BT = plan.tokens;
  p.tile_rows = tile_rows(unit, BT);
  const int64_t tiles = (rows + p.tile_rows - 1) / p.tile_rows * n128;
  p.n_tiles = static_cast<int>(n128);
  p.tile_tokens = BT;
  p.cluster = plan.cluster;
  p.stages = std::min(kSplitMaxStages, kSplitRing / (16384 + BT * 128));
  if (rf_status st = make_maps(&t, p, d_X, x_row_stride, d_W, w_row_stride, d_in, BT, 128)) return st;
  return launch_split(t, p, tiles, di, s);
}
