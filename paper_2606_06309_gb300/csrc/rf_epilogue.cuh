// rf_epilogue.cuh -- sums of products on their way out (scales, bias, activation, gate, residual) and the rows of a
// tile on their way in, for rf_linear and rf_linear_i8.  Both use all of it, but for finish_tile and what it
// calls: those are rf_linear's, and rf_linear_i8's pairs have a form of their own.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "rf_act.cuh"
#include "rf_deal.h"
#include "rf_ops.h"
#include "rf_rows.cuh"
#include "rf_stage.cuh"
#include "rf_tc_ptx.cuh"

namespace rf {

constexpr uint64_t kDrainLimitNs = 200000000ull;  // 0.2 s for what is in flight at teardown

// ---------------------------------------------------------------------------------------
// Epilogue
// ---------------------------------------------------------------------------------------
struct Epilogue {
  void* Y;
  const void* R;        // or null; elements of Y's type
  const void* bias;     // or null; elements of in_dtype
  const float* gate;    // or null
  int64_t y_stride, r_stride, gate_stride;  // elements; gate_stride 0: one row for all frames
  const float *x_scale, *w_scale;  // SCALED: of each token and each column, on the sums
  int act, in_dtype, out_dtype;
  int n_out;
  int vec;              // Y and R rows, bias and gate can be moved in 16-byte vectors
  int vec_cols;         // bias, gate and w_scale alone
};

// A token's scale as two factors, one for before the column's and one for after it: a sum below 2^31 times the
// first stays below 2^95, so that nothing overflows but a product of all three that does.  The second is 1 for all
// but rows of numbers above 2^70.
constexpr float kLargeScale = 0x1p64f;
__device__ __forceinline__ float scale_first(float xs) { return fabsf(xs) > kLargeScale ? 1.f : xs; }
__device__ __forceinline__ float scale_then(float xs) { return fabsf(xs) > kLargeScale ? xs : 1.f; }

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

// Results of a CTA's share of a tile's tokens from the sums of all CTAs: a warp has kTok tokens at
// a time, a lane four columns of each, with the loads of all of them in flight.  VEC: neighbouring
// columns, moved as vectors; otherwise every 32nd, so that a warp's accesses are of consecutive
// elements either way.
template <bool VEC, bool SCALED, int THREADS>
__device__ __forceinline__ void finish_tokens(const Epilogue& e, const int2* tokens, uint32_t sums,
                                              int n0, int BT, int rows, int rank, int C) {
  constexpr int kTok = 4, kApart = VEC ? 1 : 32;
  const int lane = threadIdx.x & 31, col = VEC ? 4 * lane : lane, out = n0 + col;
  if (out >= e.n_out) return;
  float bias[4] = {}, ws[4];
  if (SCALED)
#pragma unroll
    for (int i = 0; i < 4; ++i) ws[i] = out + i * kApart < e.n_out ? e.w_scale[out + i * kApart] : 0.f;
  if (e.bias)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (out + i * kApart < e.n_out) bias[i] = load_elem(e.bias, out + i * kApart, e.in_dtype);
  const int step = THREADS / 32 * C;  // between a warp's tokens
#pragma unroll 1
  for (int j0 = THREADS / 32 * rank + (threadIdx.x >> 5); j0 < rows; j0 += kTok * step) {
    int2 t[kTok];
    float v[kTok * 4];
#pragma unroll
    for (int u = 0; u < kTok; ++u) {
      const int j = j0 + u * step;
      t[u] = j < BT ? tokens[j] : make_int2(-1, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * u + i] = SCALED ? 0.f : bias[i];
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
    if (SCALED)
#pragma unroll
      for (int u = 0; u < kTok; ++u) {
        const float xs = t[u].x >= 0 ? e.x_scale[t[u].x] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * u + i] = v[4 * u + i] * scale_first(xs) * ws[i] * scale_then(xs) + bias[i];
      }
    activate(e.act, v);
#pragma unroll
    for (int u = 0; u < kTok; ++u)
      if (t[u].x >= 0) finish4<VEC>(e, t[u].x, t[u].y, out, v + 4 * u);
  }
}

}  // namespace rf
