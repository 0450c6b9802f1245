// rf_linear_i8.cu -- matrix product of 8-bit integers with a scale per token and per column, bias,
// activation, gate and residual, over the active frames.
//
//     Y[t, n] = R[t, n] + g[n] * act(s[t] u[n] sum_k X[t, k] W[n, k] + b[n])     t: tokens of active frames
//
// The tensor cores of sm_103a have no product of 8-bit integers (tcgen05's kind::i8 is refused for this
// target).  A byte is exact in fp16, a product of two in 15 bits, so digits are expanded to fp16 on
// their way to the tensor cores and summed in fp32: exactly while sums stay below 2^24.  Memory and L2
// see bytes only.
//
// Three kernels:
//   pair8_kernel  many rows: a pair of CTAs on 256 tokens x 192 columns (cta_group::2)
//   split8_kernel few rows: 128 columns of W against 16 to 256 tokens, K split over a cluster
//   dot8_kernel   up to eight rows: whole-number sums (dp4a), no tensor core
//
// Measured (device time, calls one after another):
//   75,600 rows 5120 -> 5120: 2.13 to 2.18 ms, 1.85 PFLOP/s while the clock holds, of the tensor cores' 2.4 at
//     that clock: the expanding warps' instructions (two thirds of the issue slots) and the hand-overs; with
//     residual 2.30 to 2.41.  (rf_linear of 16-bit rows: 1.87 to 1.96, with residual and gate 2.2 to 2.5.)
//   6,240 of 20,280 rows 1536 -> 6144, bias and tanh-GELU: 113 to 136 us.  As one frame without activation 92 to
//     98: eleven rounds of the 76 pairs, some 16,500 cycles a tile, of which 24 steps at the rate of long rows are
//     11,200; what the others go to is not known.  (rf_linear: 82 and 65 to 73.)
//   1 row 1536 -> 9216: 3.3 us, of which W's 14 MB take 2.1.
//   333 rows 1000 -> 777: 12 us: launch, tensor memory, and digits that come in three dependent steps
//     (global memory, registers, shared memory).
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "rf_epilogue.cuh"
#include "rf_vec.cuh"

namespace rf {
namespace {

struct I8Params {
  LinearParams lin;  // kblocks: of 64 digits
  const int8_t *X, *W;
  int64_t x_stride, w_stride;
  int K, bn;  // bn: columns of a pair's tile
  FastDiv by_group;  // kGroupM rows of tiles
};

// Four bytes to four fp16, exactly: with the sign bit turned over a byte is the digit + 128; behind
// 0x64 it is the fp16 number 1024 + that.
__device__ __forceinline__ void expand4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  const __half2 off = __half2half2(__ushort_as_half(0x6480));  // 1152
  const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off);
  const __half2 y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void expand16(const uint4& v, uint32_t* to) {
  expand4(v.x, to[0], to[1]);
  expand4(v.y, to[2], to[3]);
  expand4(v.z, to[4], to[5]);
  expand4(v.w, to[6], to[7]);
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Eight rows of 64 digits, a warp's: lane -> row of the eight and 16 digits of it.
struct Unit {
  int row, c;
  __device__ __forceinline__ explicit Unit(int lane) : row(lane >> 2), c(lane & 3) {}
  // 16 expanded digits into a tile of rows of 64 fp16, 128-byte swizzle, at the eight rows' address.  Eight
  // lanes that store together have an even row's even pieces and the next row's, which are odd ones.
  __device__ __forceinline__ void put(uint32_t eight_rows, const uint32_t* v) const {
    const uint32_t at = eight_rows + row * 128 + (((2 * c) ^ row) << 4);
    sts128(at, make_uint4(v[0], v[1], v[2], v[3]));
    sts128(at ^ 16, make_uint4(v[4], v[5], v[6], v[7]));
  }
};

// ---------------------------------------------------------------------------------------
// Epilogue of a tile
// ---------------------------------------------------------------------------------------
// The columns' scales, biases and gates of a tile in shared memory, in 32 bits, fetched while the accumulator
// is still being summed: from global memory as they were needed, two round trips for each 32 columns
// held the rows up, 8000 of 13,500 cycles for 192 columns.
constexpr int kTileCols = 192;
struct TileCols {
  float scale[kTileCols], bias[kTileCols], gate[kTileCols];
};
// Column `at` of those from n0 on, one per thread; gate_row: of all of the tile's rows, or null.
__device__ __forceinline__ void fetch_col(const Epilogue& e, TileCols& c, int n0, int at, const float* gate_row) {
  const int n = n0 + at;
  const bool on = n < e.n_out;
  const float scale = on ? e.w_scale[n] : 0.f, gate = gate_row && on ? gate_row[n] : 0.f;
  const float bias = e.bias && on ? load_elem(e.bias, n, e.in_dtype) : 0.f;
  c.scale[at] = scale;
  c.bias[at] = bias;
  c.gate[at] = gate;
}
__device__ __forceinline__ void each4(const float* from, float (&v)[32], uint64_t (*op)(uint64_t, uint64_t)) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const float4 s = *reinterpret_cast<const float4*>(from + i);
    f2_unpack(op(f2_pack(v[i], v[i + 1]), f2_pack(s.x, s.y)), v[i], v[i + 1]);
    f2_unpack(op(f2_pack(v[i + 2], v[i + 3]), f2_pack(s.z, s.w)), v[i + 2], v[i + 3]);
  }
}
// 32 columns from column `at` of the tile, n of the result: scales, bias, activation, gate.
__device__ __forceinline__ void finish_scaled(const Epilogue& e, const TileCols& c, int at, int frame, int n,
                                              float xs, bool one_gate, float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) f2_unpack(fmul2(f2_pack(v[i], v[i + 1]), f2_both(scale_first(xs))), v[i], v[i + 1]);
  each4(c.scale + at, v, fmul2);
  if (fabsf(xs) > kLargeScale)
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= xs;
  if (e.bias) each4(c.bias + at, v, fadd2);
  activate(e.act, v);
  if (!e.gate) return;
  if (one_gate) {
    each4(c.gate + at, v, fmul2);
  } else {
    const float* g = e.gate + frame * e.gate_stride + n;
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (n + i < e.n_out) v[i] *= g[i];
  }
}

// As rf_linear's finish_tile, with scales, and other registers and waits: a warp's 32 rows of an accumulator (tensor memory columns from `acc`; a row per
// lane, its token or -1), columns n0 .. n0 + cols - 1 of the result, the tile's from `col` on, 128 bytes of them at a time through the
// warp's stage.  ready() is called when the accumulator is wanted, read() when it has been read; false from
// ready() ends it.
template <bool OUT32, typename Ready, typename Read>
__device__ __forceinline__ bool finish_tile8(const Epilogue& e, const CUtensorMap* tmY, uint4* stage,
                                             const TileCols& tc, bool one_gate, uint32_t acc, int n0, int col,
                                             int cols, int64_t token, int frame, Ready&& ready, Read&& read) {
  constexpr int kCols = OUT32 ? 32 : 64, kBytes = OUT32 ? 4 : 2, kHalves = kCols / 32;
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
  auto whole = [&](int c) { return e.vec && n0 + (c + 1) * kCols <= e.n_out; };
  auto fetch = [&](int c) {  // the residual's rows, ahead of their use
    stage_free();
    if (whole(c)) fetch_rows(stage, R + c * 128, span_r, r_bytes);
    else if (on_words<kBytes>(R, span_r, r_bytes))
      fetch_words<kBytes>(stage, R + c * 128, span_r, r_bytes, e.n_out - n0 - c * kCols);
    else fetch_elems<kBytes>(stage, R + c * 128, span_r.at, e.n_out - n0 - c * kCols);
  };
  // 32 consecutive tokens leave through TMA, in the background
  const bool bulk = span_y.regular && span_y.n == 32;
  const int token0 = __shfl_sync(0xffffffffu, static_cast<int>(token), 0);
  if (e.R && chunks > 0) fetch(0);
  const float xs = token >= 0 ? e.x_scale[token] : 0.f;
  if (!ready()) return false;
  const int pieces = chunks * kHalves;
  if (pieces == 0) {
    read();
    return true;
  }
  // piece i of 32 columns, v its sums
  auto piece = [&](int i, int half, float (&v)[32]) {
    const int c = i / kHalves;
    finish_scaled(e, tc, col + i * 32, frame, n0 + i * 32, xs, one_gate, v);
    if (half == 0) {
      if (e.R) await_rows();
      else stage_free();
    }
#pragma unroll
    for (int q = 0; q < (OUT32 ? 8 : 4); ++q) {
      // the residual's piece of this lane's row makes way for the result's
      uint4& at = stage_at(stage, lane, half * 4 + q);
      if (OUT32) {
        float* x = v + 4 * q;
        if (e.R) {
          const uint4 r = at;
          x[0] += __uint_as_float(r.x);
          x[1] += __uint_as_float(r.y);
          x[2] += __uint_as_float(r.z);
          x[3] += __uint_as_float(r.w);
        }
        at = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                        __float_as_uint(x[3]));
      } else {
        float* x = v + 8 * (q & 3);
        if (e.R) {
          const uint4 r = at;
          add2(r.x, e.out_dtype, x[0], x[1]);
          add2(r.y, e.out_dtype, x[2], x[3]);
          add2(r.z, e.out_dtype, x[4], x[5]);
          add2(r.w, e.out_dtype, x[6], x[7]);
        }
        at = e.out_dtype == RF_FP16
                 ? make_uint4(pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]), pack_f16x2(x[4], x[5]),
                              pack_f16x2(x[6], x[7]))
                 : make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                              pack_bf16x2(x[6], x[7]));
      }
    }
    if (half != kHalves - 1) return;
    if (!whole(c)) {
      if (span_y.regular) store_words<kBytes>(stage, Y + c * 128, span_y, y_bytes, e.n_out - n0 - c * kCols);
      else store_elems<kBytes>(stage, Y + c * 128, span_y.at, e.n_out - n0 - c * kCols);
    } else if (bulk) {
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        tma_store_2d(tmY, smem_u32(stage), n0 + c * kCols, token0);
        bulk_commit();
      }
    } else {
      store_rows(stage, Y + c * 128, span_y, y_bytes);
    }
    if (e.R && c + 1 < chunks) fetch(c + 1);
  };
#pragma unroll 1
  for (int i = 0; i < pieces; i += kHalves) {
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
      float v[32];
      tmem_ld32(acc + (i + half) * 32, reinterpret_cast<uint32_t(&)[32]>(v));
      tmem_wait_ld();
      if (i + half == pieces - 1) read();
      piece(i + half, half, v);
    }
  }
  return true;
}

// tile_at without divisions: every warp of a pair asks for every tile.
__device__ __forceinline__ void tile_at8(const I8Params& q, int t, int m_tiles, int& m, int& n) {
  const int g = q.by_group.div(t), i = t - g * static_cast<int>(q.by_group.d);
  const int width = min(kGroupM, m_tiles - g * kGroupM);
  n = width == kGroupM ? i / kGroupM : i / width;
  m = g * kGroupM + (i - n * width);
}

// ---------------------------------------------------------------------------------------
// Many rows: pairs of CTAs
// ---------------------------------------------------------------------------------------
// Digits come by TMA, 128 columns of K at a time.  One warpgroup expands the CTA's 128 rows of X into
// tensor memory, as the product's A side (a row is a lane: no shared memory, whose bandwidth is the
// scarce thing here), another its half of the tile's rows of W into shared memory.  Per 64 columns
// of K the CTA's shared memory then moves 12 + 8 KB of digits twice (in, and to the registers) and W's 12 KB
// of fp16 twice: 416 cycles' worth at 128 bytes each, beside the 384 of the products.
// Tensor memory: two accumulators of 192 columns, four stages of A of 32.
constexpr int kThreads8 = 896;  // warps 0, 3 TMA, 1 MMA (first CTA), 2 tensor memory, 4-11 epilogue, 12-27 digits
constexpr int kEpi8 = 8, kConv8 = 8;  // two sets of four for X and four for W, each with every other step
constexpr int kBN8 = kTileCols;

struct Pair8 {
  static constexpr int kABytes = 128 * 128, kBBytes = kBN8 / 2 * 128;
  static constexpr int kDigits = kABytes + kBBytes, kStages = 5;  // stages of 128 digits
  static constexpr int kHalfBytes = kBN8 / 2 * 128, kWide = 2;  // of 64 columns in fp16; stages of two
  static constexpr int kBarFull = 0, kBarEmpty = kStages, kBarIn = 2 * kStages, kBarOut = kBarIn + kWide,
                       kBarAccFull = kBarOut + kWide, kBarAccEmpty = kBarAccFull + 2,
                       kBarCols = kBarAccEmpty + 2, kBars = kBarCols + 2;
  static constexpr int kOffHalf = kStages * kDigits;
  static constexpr int kOffStage = kOffHalf + 2 * kWide * kHalfBytes;
  static constexpr int kOffBar = kOffStage + kEpi8 * kTurnBytes;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kOffCols = kOffMisc + 16;
  static constexpr int kOffList = kOffCols + 2 * static_cast<int>(sizeof(TileCols));
  static constexpr int kSmem = kOffList + 2 * static_cast<int>(sizeof(BoxList<128>)) + 1024;
  static constexpr uint32_t kTmemCols = 512, kTmemA = 2 * kBN8;
};
// Registers: 896 threads are launched with 72 each; the warpgroups' shares add up to that.
constexpr int kRegsCtl = 40, kRegsEpi = 104, kRegsConv = 64;
static_assert(kRegsCtl + 2 * kRegsEpi + 4 * kRegsConv <= 7 * 72, "registers");

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads8, 1)
    pair8_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmMany,
                 const __grid_constant__ CUtensorMap tmUnit, const __grid_constant__ CUtensorMap tmW,
                 const __grid_constant__ CUtensorMap tmY, const __grid_constant__ I8Params q) {
  using C = Pair8;
  const LinearParams& p = q.lin;
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
      mbar_init(bar(C::kBarEmpty + s), kConv8);
    }
    for (int s = 0; s < C::kWide; ++s) {
      mbar_init(bar(C::kBarIn + s), 2 * kConv8);
      mbar_init(bar(C::kBarOut + s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar(C::kBarAccFull + b), 1);
      mbar_init(bar(C::kBarAccEmpty + b), 2 * kEpi8);
      mbar_init(bar(C::kBarCols + b), kEpi8);
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
  const int steps = (p.kblocks + 1) / 2;  // of 128 digits
  const int w_rows = q.bn / 2;            // of W in a CTA

  if (warp < 4) {
    reg_dealloc<kRegsCtl>();
    if (warp == 0 || warp == 3) {  // two warps, as a tile across frames has many boxes
      const bool lead = elect_one();
      const int who = warp == 3;
      BoxList<128>& list = reinterpret_cast<BoxList<128>*>(smem + C::kOffList)[who];
      int it = 0, s = 0, turn = 1;
      bool ok = true;
      for (int t = pair; ok && t < tiles; t += pairs) {
        int m, n;
        tile_at8(q, t, m_tiles, m, n);
        const RowBoxes x = list_boxes(p.rows, R, (2 * m + rank) * half, half, 128, list);
        const int w0 = n * q.bn + rank * w_rows;
#pragma unroll 1
        for (int kb = 0; kb < steps; ++kb, ++it) {
          const uint32_t dst = sbase + s * C::kDigits, full = bar(C::kBarFull + s);
          if (!ready_wait<false>(bar(C::kBarEmpty + s), turn, abort)) {
            if (lead) flag_error(p, 0);
            ok = false;
            break;
          }
          if (lead) {
            if (who == 0) {
              mbar_arrive_expect_tx(full, (w_rows + x.rows) * 128);
              tma_load_2d(dst + C::kABytes, &tmW, full, kb * 128, w0);
              tma_load_2d(dst + C::kABytes + C::kBBytes / 2, &tmW, full, kb * 128 + 64, w0);
            }
            load_rows<false>(x, list, {&tmX, &tmMany, &tmUnit}, dst, full, kb * 128, who, 2);
          }
          __syncwarp();
          if (++s == C::kStages) {
            s = 0;
            turn ^= 1;
          }
        }
      }
      // every copy has landed
      if (who == 0)
#pragma unroll 1
        for (int i = 0; i < C::kStages; ++i)
          if (it > i) mbar_drain_inline(bar(C::kBarFull + i), ((it - 1 - i) / C::kStages) & 1, kDrainLimitNs);
    } else if (warp == 1 && rank == 0) {
      const bool lead = elect_one();
      const uint32_t idesc = idesc_f16(1, 256, q.bn, 0);
      const uint64_t dB0 = smem_desc_sw128(sbase + C::kOffHalf, 16, 1024);
      int it = 0, n_acc = 0;
      bool ok = true;
      for (int t = pair; ok && t < tiles; t += pairs, ++n_acc) {
        const int b = n_acc & 1;
        if (!warp_wait<true>(bar(C::kBarAccEmpty + b), ((n_acc >> 1) & 1) ^ 1, abort)) {
          if (lead) flag_error(p, 1);
          break;
        }
        tc_fence_after();
        const uint32_t acc = tmem + b * kBN8;
#pragma unroll 1
        for (int kb = 0; kb < steps; ++kb, ++it) {
          const int s = it & 1;
          if (!ready_wait<true>(bar(C::kBarIn + s), (it >> 1) & 1, abort)) {
            if (lead) flag_error(p, 2);
            ok = false;
            break;
          }
          tc_fence_after();
          if (lead) {
            const uint32_t a = tmem + C::kTmemA + s * 64;
            const uint64_t dB = dB0 + s * (2 * C::kHalfBytes / 16);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma_ts_pair(acc, a + k * 8, dB + k * 2, idesc, (kb | k) != 0);
            if (2 * kb + 1 < p.kblocks)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                tc_mma_ts_pair(acc, a + 32 + k * 8, dB + C::kHalfBytes / 16 + k * 2, idesc, 1);
            tc_commit_pair(bar(C::kBarOut + s));
            if (kb == steps - 1) tc_commit_pair(bar(C::kBarAccFull + b));
          }
          __syncwarp();
        }
      }
    }
  } else if (warp < 12) {
    reg_alloc<kRegsEpi>();
    const int quarter = warp & 3, part = (warp - 4) >> 2;  // lanes of tensor memory; half of the columns
    const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
    uint4* stage = reinterpret_cast<uint4*>(smem + C::kOffStage + (warp - 4) * kTurnBytes);
    TileCols* tile_cols = reinterpret_cast<TileCols*>(smem + C::kOffCols);
    // columns of the first half, whole pieces of 128 bytes; where that is two of three, the halves take it in turn
    const int piece = p.epi.out_dtype == RF_FP32 ? 32 : 64;
    const int first = ((q.bn + piece - 1) / piece + 1) / 2 * piece;
    int n_acc = 0;
    for (int t = pair; t < tiles; t += pairs, ++n_acc) {
      int m, n;
      tile_at8(q, t, m_tiles, m, n);
      const int b = n_acc & 1, side = part ^ b;
      const int col = side ? first : 0, cols = side ? max(q.bn - first, 0) : min(first, q.bn);
      const int r0 = (2 * m + rank) * half, row = quarter * 32 + lane, r = r0 + row;
      // (the buffer's last use is over: its readers have waited for the other one's columns since)
      TileCols& tc = tile_cols[b];
      const float* gate = p.epi.gate;
      bool one_gate = p.epi.gate_stride == 0;
      if (gate && !one_gate) {  // the tile's rows are of one frame?
        // (without a list the rows are the tokens, and those that pad them are of no frame)
        const RowsFrame rf = p.rows.active ? rows_frame(r0, half, R, p.rows.by_Np)
                                           : rows_frame(r0, half, p.rows.T, p.by_N);
        one_gate = rf.one;
        if (one_gate) gate += p.rows.frame(rf.a) * p.epi.gate_stride;
      }
      if (threadIdx.x - 128 < kTileCols) fetch_col(p.epi, tc, n * q.bn, threadIdx.x - 128, one_gate ? gate : nullptr);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kBarCols + b));
      int frame = 0;
      const int token = row < half && r < R ? row_token(p, r, frame) : -1;
      auto ready = [&]() -> bool {
        const bool ok = ready_wait<false>(bar(C::kBarCols + b), (n_acc >> 1) & 1, abort) &&
                        warp_wait<true>(bar(C::kBarAccFull + b), (n_acc >> 1) & 1, abort);
        if (!ok && lane == 0) flag_error(p, 3);
        tc_fence_after();
        return ok;
      };
      auto read = [&]() {  // the accumulator may be written again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(bar(C::kBarAccEmpty + b), 0));
      };
      const uint32_t acc = tmem + lane_base + b * kBN8 + col;
      const int n0 = n * q.bn + col;
      if (!(p.epi.out_dtype == RF_FP32
                ? finish_tile8<true>(p.epi, &tmY, stage, tc, one_gate, acc, n0, col, cols, token, frame, ready, read)
                : finish_tile8<false>(p.epi, &tmY, stage, tc, one_gate, acc, n0, col, cols, token, frame, ready, read)))
        break;
    }
    if (lane == 0) bulk_wait_all();
  } else {
    reg_dealloc<kRegsConv>();
    // These warps' instructions bound the kernel: one flat loop over the steps of all tiles, with little
    // around the loads, the expansion and the stores.  A set has one of the two stages to itself, and the
    // time of the other one's products for what cannot be done before its own are over.
    const int quarter = warp & 3, set = warp >= 20;
    const int total = pair < tiles ? ((tiles - 1 - pair) / pairs + 1) * steps : 0;
    const uint32_t in = map_to_rank(bar(C::kBarIn + set), 0);
    int it = set;
    bool ok = true;
    // get: half h of a stage's digits (past K zeros, which nothing reads); put: expanded into half h of the
    // products' stage; seal: before they may read it.
    auto convert = [&](auto&& get, auto&& put, auto&& seal) {
      uint4 d[4];
      int s = set, turn = 0;
      auto fetch = [&]() {
        ok = ready_wait<false>(bar(C::kBarFull + s), turn, abort);
        if (ok) get(sbase + s * C::kDigits, 0, d);
      };
      if (it < total) fetch();
#pragma unroll 1
      for (; ok && it < total; it += 2) {
        uint32_t v[32];
#pragma unroll
        for (int c = 0; c < 4; ++c) expand16(d[c], v + 8 * c);
        get(sbase + s * C::kDigits, 1, d);
        ok = ready_wait<true>(bar(C::kBarOut + set), ((it >> 1) & 1) ^ 1, abort);
        if (!ok) break;
        put(0, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) expand16(d[c], v + 8 * c);
        put(1, v);
        seal();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_shared(in);
          mbar_arrive(bar(C::kBarEmpty + s));
        }
        s += 2;
        if (s >= C::kStages) {
          s -= C::kStages;
          turn ^= 1;
        }
        if (it + 2 < total) fetch();
      }
    };
    if ((warp & 4) != 0) {  // X: a lane's row of 128 digits, into that lane of tensor memory
      const uint32_t row = quarter * 32 + lane;
      uint32_t at[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) at[c] = row * 128 + ((c ^ (row & 7)) << 4);
      const uint32_t to = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + C::kTmemA + set * 64;
      convert(
          [&](uint32_t from, int h, uint4 (&d)[4]) {
#pragma unroll
            for (int c = 0; c < 4; ++c) d[c] = lds128(from + at[4 * h + c]);
          },
          [&](int h, uint32_t (&v)[32]) {
            tc_fence_after();  // the products that read this stage are done
            tmem_st32(to + h * 32, v);
          },
          [&]() {
            tmem_wait_st();
            tc_fence_before();
          });
    } else {  // W: every fourth group of eight rows
      const Unit unit(lane);
      const uint32_t at = C::kABytes + quarter * 512 + lane * 16;
      const uint32_t to = sbase + C::kOffHalf + set * 2 * C::kHalfBytes + quarter * 1024;
      const int groups = (w_rows - quarter * 8 + 31) / 32;
      convert(
          [&](uint32_t from, int h, uint4 (&d)[4]) {
#pragma unroll
            for (int i = 0; i < 3; ++i)
              if (i < groups) d[i] = lds128(from + at + h * (C::kBBytes / 2) + i * 2048);
          },
          [&](int h, uint32_t (&v)[32]) {
#pragma unroll
            for (int i = 0; i < 3; ++i)
              if (i < groups) unit.put(to + h * C::kHalfBytes + i * 4096, v + 8 * i);
          },
          [&]() { fence_proxy_async(); });
    }
    if (!ok && lane == 0) flag_error(p, 4);
    // the products have read the stage, so no arrival on this CTA's barrier is still to come
    if (it > set) mbar_drain_inline(bar(C::kBarOut + set), ((it - 2) >> 1) & 1, kDrainLimitNs);
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
// As rf_linear's split kernel: 128 columns of the result (rows of W) x tile_tokens tokens, the CTAs of a
// cluster with equal ranges of K, joined through distributed shared memory in order.  All warps but
// the MMA warp load digits from global memory, some steps ahead in registers, expand them, and leave
// them in shared memory: no boxes, as a lane's row may be any token's.
constexpr int kSplitThreads8 = 288;  // warps 0-7 digits and results, 8 MMA and tensor memory
constexpr int kWork8 = 256;
constexpr int kSplitRing8 = 196608, kSplitMaxStages8 = 8;
constexpr int kS8Full = 0, kS8Empty = kSplitMaxStages8, kS8Acc = 2 * kSplitMaxStages8, kS8Bars = kS8Acc + 1;
constexpr int kS8OffBar = kSplitRing8, kS8OffMisc = kS8OffBar + kS8Bars * 8, kS8OffTok = kS8OffMisc + 24,
              kSplitSmem8 = kS8OffTok + 256 * 8 + 1024;

// 16 digits of a row from k on; zeros past K, and where there is no row.  (An ordinary load: the launch before may
// have made W or X while this grid was resident already, which .nc does not allow.)
__device__ __forceinline__ uint4 digits16(const int8_t* row, int k, int K) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (!row || k >= K) return v;
  if (k + 16 <= K) {
    asm volatile("ld.global.L1::no_allocate.L2::128B.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(row + k));
    return v;
  }
  uint32_t* w = &v.x;
#pragma unroll
  for (int i = 0; i < 15; ++i)
    if (k + i < K) w[i >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(row[k + i])) << 8 * (i & 3);
  return v;
}

// G: groups of eight rows of a warp; AHEAD: steps of 64 digits in registers.
template <int G, int AHEAD>
__global__ void __launch_bounds__(kSplitThreads8, 1) split8_kernel(const __grid_constant__ I8Params q) {
  const LinearParams& p = q.lin;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw);
  const uint32_t bar0 = sbase + kS8OffBar;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kS8OffMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(smem + kS8OffMisc + 4);
  int2* tokens = reinterpret_cast<int2*>(smem + kS8OffTok);  // {token, frame}
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int BT = p.tile_tokens, C = p.cluster;
  const int rank = C > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int tile = blockIdx.x / C;
  const int m = tile / p.n_tiles, n = tile - m * p.n_tiles;
  const int stage_bytes = (128 + BT) * 128;
  const uint32_t tmem_cols = BT < 32 ? 32 : BT;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(bar(kS8Full + s), kWork8 / 32);
      mbar_init(bar(kS8Empty + s), 1);
    }
    mbar_init(bar(kS8Acc), 1);
    *abort = 0;
    fence_mbar_init();
  }
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const int R = p.rows.frames() * p.rows.Np;
  const int r0 = m * p.tile_rows, rows = min(p.tile_rows, R - r0);
  if (r0 >= R) return;  // the whole cluster
  if (warp == 8) {
    tmem_alloc(smem_u32(tmem_slot), tmem_cols);
    tmem_relinquish();
  } else {
    for (int j = threadIdx.x; j < BT; j += kWork8) {
      int2 t = make_int2(-1, 0);
      if (j < rows) t.x = row_token(p, r0 + j, t.y);
      tokens[j] = t;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int kb0 = p.kblocks * rank / C, kb1 = p.kblocks * (rank + 1) / C;

  if (warp < 8) {
    const Unit unit(lane);
    const int8_t* row[G];
    bool has[G];  // of this warp
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int r = (warp + 8 * g) * 8 + unit.row;
      row[g] = nullptr;
      has[g] = (warp + 8 * g) * 8 < 128 + BT;
      if (r < 128) {
        if (n * 128 + r < p.epi.n_out) row[g] = q.W + (n * 128 + r) * q.w_stride;
      } else if (r < 128 + BT) {
        const int token = tokens[r - 128].x;
        if (token >= 0) row[g] = q.X + token * q.x_stride;
      }
    }
    uint4 v[AHEAD][G];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (kb0 + a < kb1) v[a][g] = digits16(row[g], (kb0 + a) * 64 + unit.c * 16, q.K);
    bool ok = true;
#pragma unroll 1
    for (int kb = kb0; ok && kb < kb1; kb += AHEAD) {
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        if (kb + a >= kb1) break;
        const int it = kb + a - kb0, s = it % p.stages;
        if (!warp_wait<false>(bar(kS8Empty + s), ((it / p.stages) & 1) ^ 1, abort)) {
          if (lane == 0) flag_error(p, 0);
          ok = false;
          break;
        }
        const uint32_t dst = sbase + s * stage_bytes;
#pragma unroll
        for (int g = 0; g < G; ++g)
          if (has[g]) {
            uint32_t w[8];
            expand16(v[a][g], w);
            unit.put(dst + (warp + 8 * g) * 1024, w);
          }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kS8Full + s));
#pragma unroll
        for (int g = 0; g < G; ++g)
          if (kb + a + AHEAD < kb1) v[a][g] = digits16(row[g], (kb + a + AHEAD) * 64 + unit.c * 16, q.K);
      }
    }
  } else {
    const bool lead = elect_one();
    const uint32_t idesc = idesc_f16(1, 128, BT, 0);
    int it = 0;
    for (int kb = kb0; kb < kb1; ++kb, ++it) {
      const int s = it % p.stages;
      if (!warp_wait<false>(bar(kS8Full + s), (it / p.stages) & 1, abort)) {
        if (lead) flag_error(p, 1);
        break;
      }
      tc_fence_after();
      if (lead) {
        const uint32_t sA = sbase + s * stage_bytes;
        const uint64_t dA = smem_desc_sw128(sA, 16, 1024), dB = smem_desc_sw128(sA + 16384, 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k) tc_mma_ss(tmem, dA + k * 2, dB + k * 2, idesc, (it | k) != 0);
        tc_commit(bar(kS8Empty + s));
      }
      __syncwarp();
    }
    // all MMAs issued are done (also after a wait that gave up: tensor memory is freed below)
    if (lead) tc_commit(bar(kS8Acc));
    __syncwarp();
    mbar_drain(bar(kS8Acc), 0, kDrainLimitNs);
  }
  float* sums = reinterpret_cast<float*>(smem);  // [BT][128]
  if (warp < 8) {
    const bool ok = warp_wait<false>(bar(kS8Acc), 0, abort);
    if (!ok && lane == 0) flag_error(p, 2);
    tc_fence_after();
    const int quarter = warp & 3;
#pragma unroll 1
    for (int c = (warp >> 2) * 32; ok && c < BT; c += 64) {
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
  if (warp < 8) {
    if (p.epi.vec) finish_tokens<true, true, kWork8>(p.epi, tokens, sbase, n * 128, BT, rows, rank, C);
    else finish_tokens<false, true, kWork8>(p.epi, tokens, sbase, n * 128, BT, rows, rank, C);
  }
  __syncwarp();
  if (C > 1) {
    cluster_arrive();  // every CTA has read the others' sums
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, tmem_cols);
  }
}

// ---------------------------------------------------------------------------------------
// Up to eight rows
// ---------------------------------------------------------------------------------------
// A warp takes kCols columns: each lane 16 digits of W's rows at a time against the same digits of the
// ROWS tokens (from L1), four products per instruction, sums in whole numbers, joined over the lanes.
constexpr int kDotThreads = 128;
template <int ROWS, int COLS>
__global__ void __launch_bounds__(kDotThreads) dot8_kernel(const __grid_constant__ I8Params q) {
  const LinearParams& p = q.lin;
  const Epilogue& e = p.epi;
  const int lane = threadIdx.x & 31;
  const int n0 = (blockIdx.x * (kDotThreads / 32) + (threadIdx.x >> 5)) * COLS;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  if (n0 >= e.n_out) return;
  const int8_t *w[COLS], *x[ROWS];
  int token[ROWS], frame[ROWS];
  const int R = p.rows.frames() * p.rows.Np;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    token[r] = -1;
    if (r < R) token[r] = row_token(p, r, frame[r]);
    x[r] = token[r] >= 0 ? q.X + token[r] * q.x_stride : nullptr;
  }
#pragma unroll
  for (int c = 0; c < COLS; ++c) w[c] = n0 + c < e.n_out ? q.W + (n0 + c) * q.w_stride : nullptr;
  int sum[ROWS][COLS] = {};
#pragma unroll 2
  for (int k = lane * 16; k < q.K; k += 512) {
    uint4 a[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) a[c] = digits16(w[c], k, q.K);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      uint4 b = make_uint4(0, 0, 0, 0);
      if (x[r] && k + 16 <= q.K) b = *reinterpret_cast<const uint4*>(x[r] + k);
      else b = digits16(x[r], k, q.K);
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        int s = sum[r][c];
        s = __dp4a(static_cast<int>(a[c].x), static_cast<int>(b.x), s);
        s = __dp4a(static_cast<int>(a[c].y), static_cast<int>(b.y), s);
        s = __dp4a(static_cast<int>(a[c].z), static_cast<int>(b.z), s);
        sum[r][c] = __dp4a(static_cast<int>(a[c].w), static_cast<int>(b.w), s);
      }
    }
  }
  int mine = 0;  // lane r * COLS + c has that sum
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      const int s = __reduce_add_sync(0xffffffffu, sum[r][c]);
      if (lane == r * COLS + c) mine = s;
    }
  const int c = lane % COLS, n = n0 + c;
  int t = -1, f = 0;
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    if (lane / COLS == r) {
      t = token[r];
      f = frame[r];
    }
  if (t < 0 || n >= e.n_out) return;
  const float xs = e.x_scale[t];
  float v[1] = {static_cast<float>(mine) * scale_first(xs) * e.w_scale[n] * scale_then(xs)};
  if (e.bias) v[0] += load_elem(e.bias, n, e.in_dtype);
  activate(e.act, v);
  if (e.gate) v[0] *= e.gate[f * e.gate_stride + n];
  if (e.R) v[0] += load_elem(e.R, t * e.r_stride + n, e.out_dtype);
  store_elem(e.Y, t * e.y_stride + n, e.out_dtype, v[0]);
}

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------
template <typename K>
rf_status set_smem(K kernel, int bytes, const DeviceInfo& di, std::atomic<bool> (&done)[64]) {
  if (bytes > di.max_smem_optin) return fail(RF_ERR_UNSUPPORTED, "rf_linear_i8: shared memory");
  if (!done[di.device]) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes))
      return fail(RF_ERR_CUDA, "cudaFuncSetAttribute(rf_linear_i8)", e);
    done[di.device] = true;
  }
  return RF_OK;
}

rf_status map_digits(CUtensorMap* m, const void* base, int cols, int64_t rows, int64_t stride, int box_rows,
                     int box_cols = 128) {
  const uint64_t dims[2] = {static_cast<uint64_t>(cols), static_cast<uint64_t>(rows)};
  const uint64_t strides[1] = {static_cast<uint64_t>(stride)};
  const uint32_t box[2] = {static_cast<uint32_t>(box_cols), static_cast<uint32_t>(box_rows)};
  return make_tensor_map(m, kInt8, base, 2, dims, strides, box);
}

rf_status launch_pair(I8Params& q, int64_t rows, const DeviceInfo& di, cudaStream_t s) {
  LinearParams& p = q.lin;
  const Epilogue& e = p.epi;
  p.n_tiles = (e.n_out + kBN8 - 1) / kBN8;
  q.by_group = FastDiv(static_cast<uint32_t>(kGroupM * p.n_tiles));
  q.bn = p.n_tiles > 1 ? kBN8 : (e.n_out + 31) / 32 * 32;
  const int64_t tiles = (rows + 2 * p.tile_rows - 1) / (2 * p.tile_rows) * p.n_tiles;
  CUtensorMap x, many, unit, w, y;
  if (rf_status st = map_digits(&x, q.X, q.K, p.rows.T, q.x_stride, 128)) return st;
  if (rf_status st = map_digits(&w, q.W, q.K, e.n_out, q.w_stride, q.bn / 2, 64)) return st;
  many = unit = y = x;
  if (p.rows.F > 1) {  // a tile can lie across frames
    if (p.rows.unit > 1 && p.rows.Np >= kBoxRows)
      if (rf_status st = map_digits(&many, q.X, q.K, p.rows.T, q.x_stride, kBoxRows)) return st;
    if (rf_status st = map_digits(&unit, q.X, q.K, p.rows.T, q.x_stride, p.rows.unit)) return st;
  }
  if (e.vec) {  // 128 bytes of 32 rows
    const int es = dtype_bytes(e.out_dtype);
    const uint64_t dims[2] = {static_cast<uint64_t>(e.n_out), static_cast<uint64_t>(p.rows.T)};
    const uint64_t strides[1] = {static_cast<uint64_t>(e.y_stride) * es};
    const uint32_t box[2] = {128u / es, 32};
    if (rf_status st = make_tensor_map(&y, e.out_dtype, e.Y, 2, dims, strides, box)) return st;
  }
  static std::atomic<bool> done[64] = {};
  if (rf_status st = set_smem(pair8_kernel, Pair8::kSmem, di, done)) return st;
  static std::atomic<int> resident[64] = {};  // pairs that run together
  int most = resident[di.device].load(std::memory_order_relaxed);
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(kThreads8);
  cfg.dynamicSmemBytes = Pair8::kSmem;
  if (most == 0) {
    cfg.gridDim = dim3(static_cast<unsigned>(di.sm_count / 2 * 2));
    if (cudaError_t err = cudaOccupancyMaxActiveClusters(&most, pair8_kernel, &cfg))
      return fail(RF_ERR_CUDA, "cudaOccupancyMaxActiveClusters(rf_linear_i8)", err);
    if (most < 1) return fail(RF_ERR_UNSUPPORTED, "rf_linear_i8: no room for a pair of CTAs");
    resident[di.device].store(most, std::memory_order_relaxed);
  }
  cfg.gridDim = dim3(static_cast<unsigned>(2 * std::min<int64_t>(tiles, most)));
  cfg.stream = s;
  return launch_early(cfg, 1, "rf_linear_i8 pair8_kernel launch", pair8_kernel, x, many, unit, w, y, q);
}

// Tokens per tile and CTAs per cluster of a split launch: the pair with the least to do for the busiest
// SM, in cycles, as rf_linear's plan; a step of 64 digits takes the warps about a cycle for each four
// of the 64 x (128 + tokens).  It ranks the plans of one product, and is no measure of their time where W is
// long: 16 rows 5120 -> 13824 take 54.9 us, over three times what it says.
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
      const double one = 5000.0 + (kblocks + c - 1) / c * ((128.0 + bt) * 64 / 30) +
                         join * (700.0 + 150.0 * (c - 1)) + (c > 1 ? 500 * c : 0);
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

template <int G, int AHEAD>
rf_status run_split(const I8Params& q, int64_t tiles, const DeviceInfo& di, cudaStream_t s) {
  static std::atomic<bool> done[64] = {};
  if (rf_status st = set_smem(split8_kernel<G, AHEAD>, kSplitSmem8, di, done)) return st;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * q.lin.cluster));
  cfg.blockDim = dim3(kSplitThreads8);
  cfg.dynamicSmemBytes = kSplitSmem8;
  cfg.stream = s;
  return launch_early(cfg, q.lin.cluster, "rf_linear_i8 split8_kernel launch", split8_kernel<G, AHEAD>, q);
}
rf_status launch_split(I8Params& q, int64_t rows, const DeviceInfo& di, cudaStream_t s) {
  LinearParams& p = q.lin;
  const int64_t n128 = (p.epi.n_out + 127) / 128;
  const SplitPlan plan = split_plan(rows, p.rows.unit, n128, p.kblocks, di.sm_count);
  p.tile_tokens = plan.tokens;
  p.cluster = plan.cluster;
  p.tile_rows = tile_rows(p.rows.unit, plan.tokens);
  p.n_tiles = static_cast<int>(n128);
  p.stages = std::min(kSplitMaxStages8, kSplitRing8 / ((128 + plan.tokens) * 128));
  const int64_t tiles = (rows + p.tile_rows - 1) / p.tile_rows * n128;
  if (plan.tokens <= 64) return run_split<3, 4>(q, tiles, di, s);
  if (plan.tokens == 128) return run_split<4, 3>(q, tiles, di, s);
  return run_split<6, 2>(q, tiles, di, s);
}

template <int ROWS, int COLS>
rf_status run_dot(const I8Params& q, cudaStream_t s) {
  constexpr int per_block = kDotThreads / 32 * COLS;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((q.lin.epi.n_out + per_block - 1) / per_block));
  cfg.blockDim = dim3(kDotThreads);
  cfg.stream = s;
  return launch_early(cfg, 1, "rf_linear_i8 dot8_kernel launch", dot8_kernel<ROWS, COLS>, q);
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" rf_status rf_linear_i8(void* d_Y, int64_t y_row_stride, int dtype, const int8_t* d_X,
                                  int64_t x_row_stride, const float* d_x_scale, const int8_t* d_W,
                                  int64_t w_row_stride, const float* d_w_scale, int F, int N, int d_in,
                                  int d_out, const void* d_bias, int act, const float* d_gate,
                                  int64_t gate_frame_stride, const void* d_R, int64_t r_row_stride,
                                  const int32_t* d_active, const int32_t* d_counts, int32_t* d_status,
                                  rf_stream_t stream) {
  if (!d_Y || !d_X || !d_W || !d_x_scale || !d_w_scale)
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: null pointer");
  if (!dtype_bytes(dtype)) return fail(RF_ERR_UNSUPPORTED, "rf_linear_i8: dtype");
  if (F < 1 || N < 1 || d_in < 1 || d_out < 1)
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: sizes >= 1");
  if (d_in >= 1 << 17) return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: d_in above 131071");
  if (act < RF_ACT_NONE || act > RF_ACT_SILU) return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: act");
  if (x_row_stride < d_in || w_row_stride < d_in || y_row_stride < d_out ||
      (d_R && r_row_stride < d_out) || (d_gate && gate_frame_stride != 0 && gate_frame_stride < d_out))
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: row stride below the row's length");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: active list and counts come together");
  if (d_R == d_Y && r_row_stride != y_row_stride && static_cast<int64_t>(F) * N > 1)
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: in place with two strides");
  // (a row by itself has no stride that matters)
  if (static_cast<int64_t>(F) * N == 1) x_row_stride = (x_row_stride + 15) / 16 * 16;
  if (d_out == 1) w_row_stride = (w_row_stride + 15) / 16 * 16;
  if (!aligned16(d_X) || !aligned16(d_W) || x_row_stride % 16 || w_row_stride % 16)
    return fail(RF_ERR_MISALIGNED, "rf_linear_i8: X and W rows on 16-byte boundaries");
  const int es = dtype_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(d_Y) % es || reinterpret_cast<uintptr_t>(d_R) % es ||
      reinterpret_cast<uintptr_t>(d_bias) % es || reinterpret_cast<uintptr_t>(d_gate) % 4 ||
      reinterpret_cast<uintptr_t>(d_x_scale) % 4 || reinterpret_cast<uintptr_t>(d_w_scale) % 4)
    return fail(RF_ERR_MISALIGNED, "rf_linear_i8: pointer not on its elements' boundary");
  // without a list the tokens are one frame, with nothing between them
  const int64_t T = static_cast<int64_t>(F) * N;
  const int64_t Fr = d_active ? F : 1, Nr = d_active ? N : T;
  const int unit = row_unit(Nr);
  const int64_t Np = (Nr + unit - 1) / unit * unit;
  if (T > 0x7FFFFFFF - 65536 || Fr * Np > 0x7FFFFFFF - 65536 || d_out > 0x7FFFFFFF - 65536)
    return fail(RF_ERR_INVALID_ARG, "rf_linear_i8: too many tokens or columns");
  DeviceInfo di;
  if (rf_status st = current_device_info(&di)) return st;
  if (di.cc_major != 10 || di.cc_minor != 3) return fail(RF_ERR_UNSUPPORTED, "needs sm_103");

  I8Params q{};
  q.X = d_X;
  q.W = d_W;
  q.x_stride = x_row_stride;
  q.w_stride = w_row_stride;
  q.K = d_in;
  LinearParams& p = q.lin;
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
  e.x_scale = d_x_scale;
  e.w_scale = d_w_scale;
  e.act = act;
  e.in_dtype = e.out_dtype = dtype;
  e.n_out = d_out;
  e.vec_cols = aligned16(d_bias) && aligned16(d_w_scale) &&
               (!d_gate || (aligned16(d_gate) && gate_frame_stride % 4 == 0));
  e.vec = e.vec_cols && aligned16(d_Y) && y_row_stride * es % 16 == 0 &&
          (!d_R || (aligned16(d_R) && r_row_stride * es % 16 == 0));
  p.by_N = FastDiv(static_cast<uint32_t>(N));
  p.kblocks = (d_in + 63) / 64;
  p.status = d_status;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);

  const int64_t rows = Fr * Np;  // at most: the active count is known on the device only
  p.tile_rows = tile_rows(unit, 128);
  const int64_t pair_tiles = (rows + 2 * p.tile_rows - 1) / (2 * p.tile_rows) * ((d_out + kBN8 - 1) / kBN8);
  // Pairs of CTAs once their tiles occupy a third of the 76 pairs (us, pair against split; K -> columns):
  //   tiles 15:  600 rows  320 ->  960  9.3 /  7.4    27:  128 rows 5120 ->  5120 27.0 / 31.0
  //         16:  256 rows 1536 -> 3000 15.9 / 14.5    40:  300 rows 1000 ->  3840 12.3 / 15.3
  //         16:  512 rows 1536 -> 1536 13.9 / 14.6    48: 2048 rows  256 ->  1024  9.4 / 10.8
  //         24: 1024 rows  128 -> 1024  8.7 /  6.8    64: 4096 rows   64 ->   640  9.3 / 12.5
  // A row of tiles costs the same whatever its rows, so for few of them it has to be longer, and K too:
  //         48:   64 rows 1536 -> 9216 14.5 / 12.5    72:   16 rows 1536 -> 13824 14.9 / 15.6
  //         72:   32 rows  320 -> 13824 10.5 / 7.3    72:   16 rows 5120 -> 13824 27.8 / 54.9
  // (Between those, 100 rows 1536 -> 9216 take 14.3 / 15.0 and go the longer way.)
  // Up to four rows it is W's bytes: dot products (4 rows 5120 -> 13824 12.3; 8 rows 32.6, pairs 29.0; 5 rows
  // 1536 -> 1536 7.1).
  const bool pair = rows > 256 ? pair_tiles >= 25
                               : pair_tiles >= (rows >= 128 ? 25 : 64) && p.kblocks >= 16;
  if (rows == 1) return run_dot<1, 2>(q, s);
  if (rows <= 4) return run_dot<4, 4>(q, s);
  if (pair) return launch_pair(q, rows, di, s);
  if (rows <= 8) return run_dot<8, 4>(q, s);
  return launch_split(q, rows, di, s);
}
