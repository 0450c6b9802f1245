// rf_norm.cu -- group norm over the active frames, channels last, with its activation, rows of 8 bits
// behind it, and its gradients.
//
//   frame f, group g: m = mean of x, r = 1 / sqrt(var + eps) over N tokens and C / G channels
//   y = act(z),  z = (x - m) r w[c] + b[c]
//   gradients: dz = dy act'(z), xh = (x - m) r;  dw = sum dz xh,  db = sum dz  (active frames' tokens)
//              dx = r (w dz - mean(w dz) - xh mean(w dz xh))     (means over the frame's group)
//   8 bits: as rf_quantize_rows of y
//
// Three launches, each of which may begin while the one before it ends:
//   sums   every block has a piece, some rows of a frame and a tile of channels, and leaves its groups' moments
//          (for the gradients, sums) in the workspace
//   join   a few blocks join these, in one order: (mean, 1 / deviation) or the means, and dW, db
//   rows   every block makes the rows of a piece; the pieces in turned order, so that what the sums read last
//          still is in L2
// (In one cooperative launch, over waves of units that stay in L2, a wave cost 10 to 14 us whatever its size: a
// grid barrier behind the rows' stores, and the joining in every block.  75,600 rows of 5120 took 533 us.)
// Where frames fit a block per tile, one launch (whole_kernel).
//
// Measured (device, fp16 and bf16): 75,600 rows of 5120 with SiLU 364 to 369 us: two reads and a write, 2.3 GB, would be 6.3 TB/s; 4 of 13
// frames of 1560 rows of 1536 17.5 us; one image of 399,360 x 128 with SiLU 58 us, two reads and a write, which would be 5.3 TB/s;
// gradients of 75,600 rows of 1536 225 us, 1.16 GB in five passes: the activation's slope and the products, twice each, at 60%
// of the issue slots.  Bound by HBM where rows are many, by three launches of 5 us in all where they are few.
// (How much of the second read comes from L2 is not measured: under the profiler each launch begins with cold caches.)
//
// The moments of a thread's rows are (mean, sum of squares about it), four (of single elements, sixteen) rows at a time, joined pairwise
// (Chan, Golub and LeVeque, "Updating formulae and a pairwise algorithm for computing sample variances",
// 1979): no difference of large sums, whatever the channels' distance from zero.  Sums are joined in one
// order: the same bits every time.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "rf_act.cuh"
#include "rf_ops.h"
#include "rf_quant.cuh"
#include "rf_vec.cuh"

namespace rf {
namespace {

constexpr int kThreads = 256;   // of a block
constexpr int kTileVecs = 128;              // vectors of a tile at most (of single elements: kThreads)
constexpr int kMaxC = 65536;                // channels

enum Mode { kRows, kDigits, kGrad };
// (152 SMs, sm_103a's: the workspace's size goes by these, and is asked for where there may be no device.)
constexpr int slots_of(int mode) { return (mode == kGrad ? 2 : 3) * 152; }
constexpr int blocks_of(int mode) { return mode == kGrad ? 2 : 3; }  // of an SM

struct NormParams {
  const int32_t* active;  // or null: every frame
  const int32_t* counts;
  const void *X, *dY, *weight, *bias;     // weight, bias: or null
  void* Y;                                // or dX
  int64_t x_stride, y_stride, dy_stride;  // elements
  float* stats;                           // [F][G][2], or null
  float2* part;                           // workspace
  float* scale;                           // of rows of 8 bits
  float *dW, *db;
  int F, N, C, G, cpg;
  int tiles, tx, ty;  // a block: ty rows x tx vectors of a tile
  int tile_groups;    // groups of a tile at most
  int seg;            // neighbouring channels of a thread that are always of one group: 1, 2, 4 or 8
  int group_segs;     // of a group in a tile at most
  FastDiv by_cpg, by_tx, by_ty, by_segs;
  int w_vec;          // weight and bias take vectors
  int cut;            // tiles cut groups
  int chunks, chunk_rows;  // pieces of a frame's rows
  int64_t blocks;     // kDigits: the last launch's
  int join_groups;    // of a joining block
  int wide;           // kGrad: blocks for dW and db
  float2* done;       // [F][G]: what the groups' rows need
  float2* channels;   // kGrad: [pieces of rows][C] sums
  FastDiv by_pieces, by_tiles;  // by_pieces: a frame's
  int act, w32;
  float eps;
  int team, segs, ring;  // kDigits: threads of a row; its parts that a team's registers hold; rows come ahead
  int whole;          // rows of results on vectors' boundaries

  __device__ __forceinline__ int frames() const { return active ? min(max(counts[0], 0), F) : F; }
  __device__ __forceinline__ int frame(int a) const { return active ? active[a] : a; }
};

template <typename T>
__device__ __forceinline__ float weight_at(const NormParams& p, const void* w, int c, float none) {
  return !w ? none : p.w32 ? static_cast<const float*>(w)[c] : to_f(static_cast<const T*>(w)[c]);
}
// Pairs of floats of the thread's channels: f(e) for the e-th.
template <int E, typename F>
__device__ __forceinline__ void each_pair(uint64_t (&to)[kPairs<E>], F&& f) {
#pragma unroll
  for (int i = 0; i < kPairs<E>; ++i) to[i] = f2_pack(f(2 * i), E == 1 ? 0.f : f(E == 1 ? 0 : 2 * i + 1));
}
// Sums over the block: thread t has a part of the sum of item t % items (items: a power of two up to kThreads),
// and gets the whole of it, added in one order.  scratch: kThreads floats, not touched by the last call before
// this one.
__device__ __forceinline__ float items_sum(float v, int items, float* scratch) {
  for (int o = 16; o >= items; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  scratch[threadIdx.x] = v;
  __syncthreads();
  const int stride = max(items, 32);
  v = 0.f;
  for (int i = threadIdx.x & (items - 1); i < kThreads; i += stride) v += scratch[i];
  return v;
}
// f(item, first part, apart, there) for `n` items, a power of two of them at a time, whose parts are dealt to threads.
template <typename F>
__device__ __forceinline__ void each_item(int n, F&& f) {
  int items = 1;
  while (items < n && items < kThreads) items *= 2;
  for (int i0 = 0; i0 < n; i0 += items) {
    const int i = i0 + (threadIdx.x & (items - 1));
    f(min(i, n - 1), items, static_cast<int>(threadIdx.x) / items, kThreads / items, i < n);
  }
}

// A block's piece: rows [r0, r1) of active frame a, channels [c0, c1), and the thread's of these.
struct Piece {
  int a, chunk, tile, r0, r1, c0, c1, tx, ty, col;
  bool mine;  // this thread has channels
  __device__ __forceinline__ Piece(const NormParams& p, int E, int i) {
    a = p.by_pieces.div(i);
    i -= a * static_cast<int>(p.by_pieces.d);
    chunk = p.by_tiles.div(i);
    tile = i - chunk * p.tiles;
    r0 = chunk * p.chunk_rows;
    r1 = min(r0 + p.chunk_rows, p.N);
    c0 = tile * p.tx * E;
    c1 = min(c0 + p.tx * E, p.C);
    ty = p.by_tx.div(static_cast<int>(threadIdx.x));
    tx = threadIdx.x - ty * p.tx;
    col = c0 + tx * E;
    mine = ty < p.ty && col < c1;
  }
  // the sums of a piece's groups
  static __device__ __forceinline__ float2* part(const NormParams& p, int a, int chunk, int tile) {
    return p.part + ((static_cast<int64_t>(a) * p.chunks + chunk) * p.tiles + tile) * p.tile_groups;
  }
  __device__ __forceinline__ int first_group(const NormParams& p) const { return p.by_cpg.div(c0); }
  __device__ __forceinline__ int groups(const NormParams& p) const { return p.by_cpg.div(c1 - 1) - p.by_cpg.div(c0) + 1; }
};

// A thread's rows of a piece, of ARRAYS matrices, U rows at a time.  They come to a ring of the thread's own in
// shared memory, U * kAhead rows ahead of their use.
// Vectors of less than 16 bytes are loaded as they are wanted.
template <int E>
constexpr int kRowsAtOnce = E == 1 ? 16 : 4;  // of a thread, in registers
template <int E>
constexpr int kGradRows = E == 1 ? 8 : 2;
template <typename T, int E, int ARRAYS, int U, int kAhead>
struct Rows {
  static constexpr bool kRing = sizeof(T) * E == 16;
  static constexpr int kSlots = U * kAhead;  // rows
  const T* from[ARRAYS];
  int64_t step[ARRAYS];
  int n, next;  // rows in all, and asked for
  uint32_t ring;  // this thread's first slot

  __device__ __forceinline__ void prime(const NormParams& p, const Piece& b) {
    n = b.mine && b.r0 + b.ty < b.r1 ? (b.r1 - b.r0 - b.ty + p.ty - 1) / p.ty : 0;
    next = 0;
    if (n > 0) {
      const int64_t row = static_cast<int64_t>(p.frame(b.a)) * p.N + b.r0 + b.ty;
      from[0] = static_cast<const T*>(p.X) + row * p.x_stride + b.col;
      step[0] = p.x_stride * p.ty;
      if (ARRAYS == 2) {
        from[ARRAYS - 1] = static_cast<const T*>(p.dY) + row * p.dy_stride + b.col;
        step[ARRAYS - 1] = p.dy_stride * p.ty;
      }
    }
    if (kRing)
#pragma unroll
      for (int g = 0; g < kAhead; ++g) ask();
  }
  __device__ __forceinline__ void ask() {  // for the next U rows
#pragma unroll
    for (int u = 0; u < U; ++u, ++next)
      if (next < n)
#pragma unroll
        for (int a = 0; a < ARRAYS; ++a) {
          const uint32_t to = ring + ((next & (kSlots - 1)) * ARRAYS + a) * (blockDim.x * 16);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from[a]) : "memory");
          from[a] += step[a];
        }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // f(first row, rows there are, v[array][row], whether that is U) for all rows
  template <typename F>
  __device__ __forceinline__ void each(F&& f) {
#pragma unroll 1
    for (int j = 0; j < n; j += U) {
      Vec<T, E> v[ARRAYS][U];
      take(j, v);
      if (j + U <= n) f(j, U, v, std::true_type());
      else f(j, n - j, v, std::false_type());
      if (kRing) ask();  // (into the slots whose values have been used)
    }
  }
  __device__ __forceinline__ void take(int j, Vec<T, E> (&v)[ARRAYS][U]) {
    if (kRing) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u < n)
#pragma unroll
          for (int a = 0; a < ARRAYS; ++a) {
            uint32_t* w = reinterpret_cast<uint32_t*>(&v[a][u]);
            const uint32_t at = ring + (((j + u) & (kSlots - 1)) * ARRAYS + a) * (blockDim.x * 16);
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
          }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u < n)
#pragma unroll
          for (int a = 0; a < ARRAYS; ++a) {
            v[a][u] = *reinterpret_cast<const Vec<T, E>*>(from[a]);
            from[a] += step[a];
          }
    }
  }
};

// ---------------------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------------------
// Moments of the thread's channels, into shared memory.
template <typename T, int E, typename Stream>
__device__ __forceinline__ void moments(const NormParams& p, const Piece& b, Stream& in, float2* sm) {
  constexpr int P = kPairs<E>;
  uint64_t mean[P] = {}, m2[P] = {};  // pairs of floats
  in.each([&](int n, int nb, const auto& v, auto full) {
    constexpr bool kFull = decltype(full)::value;
    constexpr int U = kRowsAtOnce<E>;
    const float share = static_cast<float>(nb) / static_cast<float>(n + nb);
    const uint64_t share2 = f2_both(share), cross2 = f2_both(share * n);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      uint64_t x[U], s = 0, q = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (kFull || u < nb) {
          x[u] = pair_of(v[0][u], i);
          s = fadd2(s, x[u]);
        }
      if (kFull) {
        s = fmul2(s, f2_both(1.f / U));
      } else {  // (exact where all are equal)
        float lo, hi;
        f2_unpack(s, lo, hi);
        s = f2_pack(lo / nb, hi / nb);
      }
      const uint64_t off = f2_neg(s);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (kFull || u < nb) {
          const uint64_t d = fadd2(x[u], off);
          q = ffma2(d, d, q);
        }
      const uint64_t d = fadd2(s, f2_neg(mean[i]));
      mean[i] = ffma2(d, share2, mean[i]);
      m2[i] = fadd2(m2[i], ffma2(fmul2(d, d), cross2, q));
    }
  });
  if (!b.mine) return;
  // neighbouring channels of one group become one (all have the same number of rows)
  float m[E], q[E];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    float a[2], c[2];
    f2_unpack(mean[i], a[0], a[1]);
    f2_unpack(m2[i], c[0], c[1]);
#pragma unroll
    for (int k = 0; k < (E == 1 ? 1 : 2); ++k) {
      m[2 * i + k] = a[k];
      q[2 * i + k] = c[k];
    }
  }
  float half = 0.5f * in.n;  // rows of each of two over 2
#pragma unroll
  for (int w = 1; w < E; w *= 2, half *= 2.f) {
    if (p.seg <= w) break;
#pragma unroll
    for (int e = 0; e < E; e += 2 * w) {
      const float d = m[e] - m[e + w];
      m[e] = fmaf(-0.5f, d, m[e]);
      q[e] = fmaf(d * d, half, q[e] + q[e + w]);
    }
  }
  const int each = E / p.seg;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e % p.seg == 0) sm[(b.ty * p.tx + b.tx) * each + e / p.seg] = make_float2(m[e], q[e]);
}
// The piece's groups, each from `parts` entries of the threads (entry k: row of threads k / segs, and one of the
// group's segments): f(group, items, first entry, step, there, get), get(k) -> rows of that thread, place in sm.
template <typename F>
__device__ __forceinline__ void each_group(const NormParams& p, const Piece& b, int E, F&& f) {
  const int g0 = b.first_group(p), rows = b.r1 - b.r0, ny = min(p.ty, rows);
  const int more = p.by_ty.div(rows), odd = rows - more * p.ty, each = E / p.seg, pitch = p.tx * each;
  each_item(b.groups(p), [&](int i, int items, int first, int step, bool there) {
    const int lo = max((g0 + i) * p.cpg, b.c0), hi = min((g0 + i + 1) * p.cpg, b.c1);
    const int n = (hi - lo) / p.seg, at = (lo - b.c0) / p.seg;
    f(i, lo, hi, items, there, [&](auto&& use) {
      for (int k = first; k < ny * p.group_segs; k += step) {
        const int y = p.by_segs.div(k), x = k - y * p.group_segs;
        if (x < n) use(y * pitch + at + x, static_cast<float>(more + (y < odd)));
      }
    });
  });
}
__device__ __forceinline__ void group_moments(const NormParams& p, const Piece& b, int E, const float2* sm,
                                              float* scratch) {
  __syncthreads();
  float2* part = Piece::part(p, b.a, b.chunk, b.tile);
  each_group(p, b, E, [&](int i, int lo, int hi, int items, bool there, auto&& each) {
      // sums of distances from one of the means: short numbers
      const float near = sm[(lo - b.c0) / p.seg].x, width = static_cast<float>(p.seg);
      float s = 0.f, q = 0.f;
      each([&](int at, float n) { s = fmaf(sm[at].x - near, n, s); });
      const float m = near + items_sum(s, items, scratch) * width /
                                 (static_cast<float>(b.r1 - b.r0) * (hi - lo));
      each([&](int at, float n) {
        const float d = sm[at].x - m;
        q += fmaf(d * d, n * width, sm[at].y);
      });
      q = items_sum(q, items, scratch + kThreads);
      if (there && static_cast<int>(threadIdx.x) < items) part[i] = make_float2(m, q);
      __syncthreads();  // sm and scratch may be written again
    });
}

// The partial sums of group g of frame a: f(sums, elements), of the pieces of rows from `l` on, every step-th.  The
// first of them stay in registers, so that the moments' second round waits for memory no more.
struct Parts {
  static constexpr int kKept = 8;
  const NormParams& p;
  int E, a, g, t0, t1, l, step;
  float2 kept[kKept];
  __device__ __forceinline__ Parts(const NormParams& p_, int E_, int a_, int g_, int l_, int step_)
      : p(p_), E(E_), a(a_), g(g_), l(l_), step(step_) {
    t0 = g * p.cpg / (p.tx * E);
    t1 = (g * p.cpg + p.cpg - 1) / (p.tx * E);
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (l + k * step < p.chunks) kept[k] = at(t0, l + k * step);
  }
  __device__ __forceinline__ float2 at(int t, int c) const {
    return Piece::part(p, a, c, t)[g - p.by_cpg.div(t * p.tx * E)];
  }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int cut = p.tx * E, last = p.N - (p.chunks - 1) * p.chunk_rows;  // rows of the last piece
    for (int t = t0; t <= t1; ++t) {
      const float cols = static_cast<float>(min(g * p.cpg + p.cpg, (t + 1) * cut) - max(g * p.cpg, t * cut));
      const float n = cols * p.chunk_rows, n_last = cols * last;
      int c = l;
      if (t == t0) {
#pragma unroll
        for (int k = 0; k < kKept; ++k, c += step)
          if (c < p.chunks) f(kept[k], c == p.chunks - 1 ? n_last : n);
      }
#pragma unroll 8
      for (; c < p.chunks; c += step) f(at(t, c), c == p.chunks - 1 ? n_last : n);
    }
  }
};

// ---------------------------------------------------------------------------------------
// Gradients: what a thread's channels have
// ---------------------------------------------------------------------------------------
// The thread's channels' weights or biases.
template <typename T, int E>
__device__ __forceinline__ void weights(const NormParams& p, const void* w, int col, float none, uint64_t (&to)[kPairs<E>]) {
  if (w && p.w_vec && E > 1) {
    if (p.w32) {
      Vec<float, E> f;
#pragma unroll
      for (int i = 0; i < E / 4; ++i)
        reinterpret_cast<float4*>(&f)[i] = reinterpret_cast<const float4*>(static_cast<const float*>(w) + col)[i];
      each_pair<E>(to, [&](int e) { return f.e[e]; });
    } else {
      const Vec<T, E> f = *reinterpret_cast<const Vec<T, E>*>(static_cast<const T*>(w) + col);
#pragma unroll
      for (int i = 0; i < kPairs<E>; ++i) to[i] = pair_of(f, i);
    }
  } else {
    each_pair<E>(to, [&](int e) { return weight_at<T>(p, w, col + e, none); });
  }
}
template <typename T, int E>
struct Channels {
  static constexpr int P = kPairs<E>;
  uint64_t m[P], r[P], w[P], o[P];  // -mean, 1 / deviation, weight, bias
  __device__ __forceinline__ Channels(const NormParams& p, const Piece& b) {
    const float2* st = reinterpret_cast<const float2*>(p.stats) + static_cast<int64_t>(p.frame(b.a)) * p.G;
    each_pair<E>(m, [&](int e) { return -st[p.by_cpg.div(b.col + e)].x; });
    each_pair<E>(r, [&](int e) { return st[p.by_cpg.div(b.col + e)].y; });
    weights<T, E>(p, p.weight, b.col, 1.f, w);
    weights<T, E>(p, p.bias, b.col, 0.f, o);
  }
  // a row's xh, and dz in place of dy
  __device__ __forceinline__ void at(int act, const Vec<T, E>& x, const Vec<T, E>& dy, uint64_t (&xh)[P],
                                     uint64_t (&dz)[P]) const {
    float z[2 * P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      xh[i] = fmul2(fadd2(pair_of(x, i), m[i]), r[i]);
      dz[i] = pair_of(dy, i);
      f2_unpack(ffma2(xh[i], w[i], o[i]), z[2 * i], z[2 * i + 1]);
    }
    if (act == RF_ACT_NONE) return;
    act_slopes(act, z);
#pragma unroll
    for (int i = 0; i < P; ++i) dz[i] = fmul2(dz[i], f2_pack(z[2 * i], z[2 * i + 1]));
  }
};

// Sums of dz and dz xh of the thread's channels, into `total`, and with the weight into sm.
template <typename T, int E, typename Stream>
__device__ __forceinline__ void gradient_sums(const NormParams& p, const Piece& b, Stream& in, float2* sm,
                                              float2* total) {
  if (!b.mine) return;
  constexpr int P = kPairs<E>;
  const Channels<T, E> ch(p, b);
  uint64_t s0[P] = {}, s1[P] = {};
  in.each([&](int, int nb, const auto& v, auto full) {
#pragma unroll
    for (int u = 0; u < kGradRows<E>; ++u)
      if (decltype(full)::value || u < nb) {
        uint64_t xh[P], dz[P];
        ch.at(p.act, v[0][u], v[1][u], xh, dz);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          s0[i] = fadd2(s0[i], dz[i]);
          s1[i] = ffma2(dz[i], xh[i], s1[i]);
        }
      }
  });
  float g0[E], g1[E];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    float a[2], c[2], w[2];
    f2_unpack(s0[i], a[0], a[1]);
    f2_unpack(s1[i], c[0], c[1]);
    f2_unpack(ch.w[i], w[0], w[1]);
#pragma unroll
    for (int k = 0; k < (E == 1 ? 1 : 2); ++k) {
      const int at = (b.ty * p.tx + b.tx) * E + 2 * i + k;
      total[at] = make_float2(a[k], c[k]);
      g0[2 * i + k] = w[k] * a[k];
      g1[2 * i + k] = w[k] * c[k];
    }
  }
  const int each = E / p.seg;
#pragma unroll
  for (int e = 0; e < E; ++e) {  // neighbouring channels of one group become one
    if (e % p.seg) continue;
    float2 t = make_float2(g0[e], g1[e]);
#pragma unroll
    for (int k = 1; k < E; ++k)
      if (k < p.seg && e + k < E) {
        t.x += g0[e + k];
        t.y += g1[e + k];
      }
    sm[(b.ty * p.tx + b.tx) * each + e / p.seg] = t;
  }
}
// Of the piece's groups, from there.
__device__ __forceinline__ void group_gradients(const NormParams& p, const Piece& b, int E, const float2* sm,
                                                float* scratch) {
  __syncthreads();
  float2* part = Piece::part(p, b.a, b.chunk, b.tile);
  each_group(p, b, E, [&](int i, int, int, int items, bool there, auto&& each) {
      float s0 = 0.f, s1 = 0.f;
      each([&](int at, float) {
        const float2 t = sm[at];
        s0 += t.x;
        s1 += t.y;
      });
      s0 = items_sum(s0, items, scratch);
      s1 = items_sum(s1, items, scratch + kThreads);
      if (there && static_cast<int>(threadIdx.x) < items) part[i] = make_float2(s0, s1);
      __syncthreads();  // sm and scratch may be written again
    });
}

// ---------------------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------------------
// join_groups groups of a frame: (mean, 1 / deviation), or the gradients' two means.
template <int MODE>
__global__ void __launch_bounds__(kThreads) join_kernel(const __grid_constant__ NormParams p, int E) {
  __shared__ float2 sm[kThreads];
  float* scratch = reinterpret_cast<float*>(sm);
  cudaGridDependencySynchronize();
  const int A = p.frames();
  const int per_frame = (p.G + p.join_groups - 1) / p.join_groups, a = blockIdx.x / per_frame;
  if (a >= A) return;
  const int g0 = (blockIdx.x - a * per_frame) * p.join_groups, ng = min(p.join_groups, p.G - g0);
  const int64_t frame = p.frame(a);
  each_item(ng, [&](int i, int items, int first, int step, bool there) {
    const Parts parts(p, E, a, g0 + i, first, step);
    const float all = static_cast<float>(p.N) * p.cpg;
    float s0 = 0.f, s1 = 0.f;
    if (MODE == kGrad) {
      parts.each([&](float2 u, float) {
        s0 += u.x;
        s1 += u.y;
      });
      s0 = items_sum(s0, items, scratch) / all;
      s1 = items_sum(s1, items, scratch + kThreads) / all;
    } else {
      const float near = parts.at(parts.t0, 0).x;
      parts.each([&](float2 u, float n) { s0 = fmaf(u.x - near, n, s0); });
      s0 = near + items_sum(s0, items, scratch) / all;
      parts.each([&](float2 u, float n) {
        const float d = u.x - s0;
        s1 += fmaf(d * d, n, u.y);
      });
      s1 = 1.f / sqrtf(items_sum(s1, items, scratch + kThreads) / all + p.eps);
    }
    if (there && static_cast<int>(threadIdx.x) < items) {
      p.done[static_cast<int64_t>(a) * p.G + g0 + i] = make_float2(s0, s1);
      if (MODE != kGrad && p.stats) reinterpret_cast<float2*>(p.stats)[frame * p.G + g0 + i] = make_float2(s0, s1);
    }
    __syncthreads();
  });
}

// A thread's rows of the result.
template <typename T, int E>
struct Out {
  T* to;
  int64_t step;
  __device__ __forceinline__ Out(const NormParams& p, const Piece& b)
      : to(static_cast<T*>(p.Y) + (static_cast<int64_t>(p.frame(b.a)) * p.N + b.r0 + b.ty) * p.y_stride + b.col),
        step(p.y_stride * p.ty) {}
  __device__ __forceinline__ void put(const NormParams& p, const Vec<T, E>& v) {
    if (p.whole) {
      store_stream(to, v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) to[e] = v.e[e];
    }
    to += step;
  }
};
template <typename T, int E, typename Stream>
__device__ __forceinline__ void rows(const NormParams& p, const Piece& b, Stream& in) {
  constexpr int P = kPairs<E>;
  const float2* sm = p.done + static_cast<int64_t>(b.a) * p.G;
  uint64_t m[P], w[P], o[P];
  each_pair<E>(m, [&](int e) { return -sm[p.by_cpg.div(b.col + e)].x; });
  each_pair<E>(o, [&](int e) { return sm[p.by_cpg.div(b.col + e)].y; });
  weights<T, E>(p, p.weight, b.col, 1.f, w);
#pragma unroll
  for (int i = 0; i < P; ++i) w[i] = fmul2(w[i], o[i]);
  weights<T, E>(p, p.bias, b.col, 0.f, o);
  Out<T, E> out(p, b);
  in.each([&](int, int nb, const auto& v, auto full) {
#pragma unroll
    for (int u = 0; u < kRowsAtOnce<E>; ++u)
      if (decltype(full)::value || u < nb) {
        Vec<T, E> r;
        float y[2 * P];
#pragma unroll
        for (int i = 0; i < P; ++i)
          f2_unpack(ffma2(fadd2(pair_of(v[0][u], i), m[i]), w[i], o[i]), y[2 * i], y[2 * i + 1]);
        activate(p.act, y);
#pragma unroll
        for (int i = 0; i < P; ++i) set_pair(r, i, y[2 * i], y[2 * i + 1]);
        out.put(p, r);
      }
  });
}

template <typename T, int E, typename Stream>
__device__ __forceinline__ void gradient_rows(const NormParams& p, const Piece& b, Stream& in) {
  constexpr int P = kPairs<E>;
  const Channels<T, E> ch(p, b);
  const float2* sm = p.done + static_cast<int64_t>(b.a) * p.G;
  uint64_t m0[P], m1[P];
  each_pair<E>(m0, [&](int e) { return -sm[p.by_cpg.div(b.col + e)].x; });
  each_pair<E>(m1, [&](int e) { return -sm[p.by_cpg.div(b.col + e)].y; });
  Out<T, E> out(p, b);
  in.each([&](int, int nb, const auto& v, auto full) {
#pragma unroll
    for (int u = 0; u < kGradRows<E>; ++u)
      if (decltype(full)::value || u < nb) {
        Vec<T, E> r;
        uint64_t xh[P], dz[P];
        ch.at(p.act, v[0][u], v[1][u], xh, dz);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          float lo, hi;
          f2_unpack(fmul2(ch.r[i], ffma2(xh[i], m1[i], ffma2(ch.w[i], dz[i], m0[i]))), lo, hi);
          set_pair(r, i, lo, hi);
        }
        out.put(p, r);
      }
  });
}

// Rows of 8 bits: a block has rows of a frame, each with all of its channels: a row is a team's, 4 to 256 threads
// with up to kDigitVecs vectors each, which stay in registers in 32 bits until the row's largest value is known
// (of longer rows they are made twice).  The next row comes to shared memory meanwhile, a thread's vectors to its own
// slots; the channels' factors are there for all rows of the block.  The blocks are dealt to the frames that are
// active (3 of 15 x 1766 rows of 1824: 54 -> 30 us; 75,600 of 1536 203 -> 189).  What bounds it are instructions, 32 an
// element, at two thirds of the issue slots.  With the sums, bf16: 75,600 rows of 1536 with SiLU 189 us, 12,480 of 2048
// 52, 7 x 1003 of 960 23, 11,907 of 752 with tanh-GELU 26.  (Eight vectors of a thread, the blocks dealt to all frames:
// 195, 52, 25, 27, and 550 rows of 96 11.4 instead of 10.6; rows of a block in step, a thread per vector: 250, 57, 28, 31.)
template <int E>
constexpr int kDigitVecs = E == 1 ? 16 : 4;
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, 2) digits_kernel(const __grid_constant__ NormParams p) {
  constexpr int V = kDigitVecs<E>, P = kPairs<E>, Q = E == 1 ? 1 : E / 4;
  constexpr bool kVec = sizeof(T) * E == 16;
  extern __shared__ __align__(16) uint8_t smem[];  // each vector's -mean, factor, bias; the ring
  __shared__ uint32_t top[2][kThreads / 32];
  const int nv = p.C / E, team = p.team, lane = threadIdx.x & (team - 1);
  const int who = static_cast<int>(threadIdx.x) / team, teams = kThreads / team;
  // all blocks over the frames that are active
  const int frames = p.frames();
  const int blocks = max(1, min(static_cast<int>(gridDim.x) / max(frames, 1), (p.N + teams - 1) / teams));
  const int a = static_cast<int>(blockIdx.x) / blocks, mine = blockIdx.x - a * blocks;
  if (a >= frames) {
    cudaGridDependencySynchronize();
    return;
  }
  const int r0 = static_cast<int>(static_cast<int64_t>(p.N) * mine / blocks);
  const int n = static_cast<int>(static_cast<int64_t>(p.N) * (mine + 1) / blocks) - r0;
  const int64_t row0 = static_cast<int64_t>(p.frame(a)) * p.N + r0;
  const T* const x0 = static_cast<const T*>(p.X) + row0 * p.x_stride;
  const bool ring = kVec && p.ring;
  // a vector's factors in shared memory, in 16 bytes: an odd number, so that neighbours' lie in other banks
  const int step = E == 8 && ring ? 7 : 3 * Q;
  const uint32_t slots = smem_u32(smem) + step * nv * 16 + threadIdx.x * 16;
  auto ask = [&](int i) {
    if (i < n) {
      const T* x = x0 + i * p.x_stride;
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k * team + lane < nv)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slots + k * (kThreads * 16)),
                       "l"(x + (k * team + lane) * E) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (ring) ask(who);
  cudaGridDependencySynchronize();
  {
    float* to = reinterpret_cast<float*>(smem);
    const float2* sm = p.done + static_cast<int64_t>(a) * p.G;
    auto put = [&](int f, int v, const uint64_t (&k)[P]) {
      if constexpr (E == 1) {
        float none;
        f2_unpack(k[0], to[f * nv + v], none);
      } else {
#pragma unroll
        for (int h = 0; h < Q; ++h)
          reinterpret_cast<ulonglong2*>(to)[v * step + f * Q + h] = make_ulonglong2(k[2 * h], k[2 * h + 1]);
      }
    };
    for (int v = threadIdx.x; v < nv; v += kThreads) {
      uint64_t r[P], k[P];
      each_pair<E>(k, [&](int e) { return -sm[p.by_cpg.div(v * E + e)].x; });
      put(0, v, k);
      each_pair<E>(r, [&](int e) { return sm[p.by_cpg.div(v * E + e)].y; });
      weights<T, E>(p, p.weight, v * E, 1.f, k);
#pragma unroll
      for (int i = 0; i < P; ++i) k[i] = fmul2(k[i], r[i]);
      put(1, v, k);
      weights<T, E>(p, p.bias, v * E, 0.f, k);
      put(2, v, k);
    }
  }
  __syncthreads();
  auto factor = [&](int f, int v, int h, uint64_t (&k)[2]) {
    if constexpr (E == 1) {
      k[0] = f2_pack(reinterpret_cast<const float*>(smem)[f * nv + v], 0.f);
    } else {
      const ulonglong2 t = reinterpret_cast<const ulonglong2*>(smem)[v * step + f * Q + h];
      k[0] = t.x;
      k[1] = t.y;
    }
  };
  float y[V][2 * P], most;
  auto value = [&](int k, int v, const Vec<T, E>& x) {
#pragma unroll
    for (int h = 0; h < Q; ++h) {
      uint64_t m[2], w[2], o[2];
      factor(0, v, h, m);
      factor(1, v, h, w);
      factor(2, v, h, o);
#pragma unroll
      for (int j = 0; j < (E == 1 ? 1 : 2); ++j)
        f2_unpack(ffma2(fadd2(pair_of(x, 2 * h + j), m[j]), w[j], o[j]), y[k][4 * h + 2 * j], y[k][4 * h + 2 * j + 1]);
    }
    if constexpr (E == 1) y[k][1] = 0.f;
    activate(p.act, reinterpret_cast<float(&)[E]>(y[k]));
#pragma unroll
    for (int j = 0; j < P; ++j) most = largest(most, y[k][2 * j], y[k][2 * j + 1]);
  };
  // the seg-th of the thread's vectors of row i, into y
  auto make = [&](int i, int seg) {
    if (ring) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int v = k * team + lane;
        if (i >= n || v >= nv) continue;
        Vec<T, E> x;
        uint32_t* w = reinterpret_cast<uint32_t*>(&x);
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(slots + k * (kThreads * 16)) : "memory");
        value(k, v, x);
      }
      ask(i + teams);
    } else if (i < n) {
      constexpr int U = kVec ? 1 : 8;  // (longer rows than the ring takes: one at a time)
      const T* from = x0 + i * p.x_stride;
#pragma unroll
      for (int k0 = 0; k0 < V; k0 += U) {
        Vec<T, E> x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int v = (seg * V + k0 + k) * team + lane;
          if (v < nv) x[k] = *reinterpret_cast<const Vec<T, E>*>(from + v * E);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int v = (seg * V + k0 + k) * team + lane;
          if (v < nv) value(k0 + k, v, x[k]);
        }
      }
    }
  };
  int turn = 0;
#pragma unroll 1
  for (int at = 0, i = who; at < n; at += teams, i += teams, turn ^= 1) {
    most = 0.f;
#pragma unroll 1
    for (int seg = 0; seg < p.segs; ++seg) make(i, seg);
    uint32_t bits = __float_as_uint(most);
    if (team >= 32) {
      bits = __reduce_max_sync(0xffffffffu, bits);
      if (team > 32) {
        const int warp = threadIdx.x >> 5, first = who * (team / 32);
        if ((threadIdx.x & 31) == 0) top[turn][warp] = bits;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + who), "r"(team) : "memory");
        for (int w = 0; w < team / 32; ++w) bits = max(bits, top[turn][first + w]);
      }
    } else {
      for (int o = team / 2; o; o >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
    }
    if (i >= n) continue;
    const RowScale rs(bits);
    if (lane == 0) p.scale[row0 + i] = rs.scale;
    int8_t* to = static_cast<int8_t*>(p.Y) + (row0 + i) * p.y_stride;
#pragma unroll 1
    for (int seg = 0; seg < p.segs; ++seg) {
      if (p.segs > 1) make(i, seg);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int v = (seg * V + k) * team + lane;
        if (v >= nv) continue;
        const Vec<int8_t, E> d = rs.template digits<false>(reinterpret_cast<const float(&)[E]>(y[k]));
        if (p.whole) {
          *reinterpret_cast<Vec<int8_t, E>*>(to + v * E) = d;
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) to[v * E + e] = d.e[e];
        }
      }
    }
  }
}

// Shared memory: the ring, the threads' sums and, of the gradients, once more without the weight; scratch.
template <typename T, int E, int MODE>
struct Layout {
  static constexpr int kArrays = MODE == kGrad ? 2 : 1, kU = MODE == kGrad ? kGradRows<E> : kRowsAtOnce<E>;
  using In = Rows<T, E, kArrays, kU, MODE == kGrad ? 4 : 2>;
  static constexpr int kRing = In::kRing ? In::kSlots * kArrays * kThreads * 16 : 0;
  static int64_t sums_bytes(const NormParams& p) {
    return kRing + 8ll * (p.ty * p.tx * E * (MODE == kGrad ? 2 : 1) + kThreads);
  }
};

// The groups of a frame's only piece of rows, from what this block's threads have left.
template <int MODE>
__device__ __forceinline__ void finish_groups(const NormParams& p, const Piece& b) {
  const float2* part = Piece::part(p, b.a, 0, b.tile);
  const int64_t g0 = static_cast<int64_t>(b.tile) * p.tile_groups;
  const float all = static_cast<float>(p.N) * p.cpg;
  for (int i = threadIdx.x; i < b.groups(p); i += kThreads) {
    float2 t = part[i];
    t = MODE == kGrad ? make_float2(t.x / all, t.y / all) : make_float2(t.x, 1.f / sqrtf(t.y / all + p.eps));
    p.done[static_cast<int64_t>(b.a) * p.G + g0 + i] = t;
    if (MODE != kGrad && p.stats) reinterpret_cast<float2*>(p.stats)[static_cast<int64_t>(p.frame(b.a)) * p.G + g0 + i] = t;
  }
}
// The piece's sums of each channel.
__device__ __forceinline__ void channel_parts(const NormParams& p, const Piece& b, int E, const float2* total) {
  float2* to = p.channels + (static_cast<int64_t>(b.a) * p.chunks + b.chunk) * p.C + b.c0;
  const int pitch = p.tx * E, ny = min(p.ty, b.r1 - b.r0);
  for (int c = threadIdx.x; c < b.c1 - b.c0; c += kThreads) {
    float2 t = total[c];
    for (int y = 1; y < ny; ++y) {
      t.x += total[y * pitch + c].x;
      t.y += total[y * pitch + c].y;
    }
    to[c] = t;
  }
}

template <typename T, int E, int MODE>
__global__ void __launch_bounds__(kThreads, blocks_of(MODE)) sums_kernel(const __grid_constant__ NormParams p) {
  using L = Layout<T, E, MODE>;
  extern __shared__ __align__(16) uint8_t smem[];
  float* scratch = reinterpret_cast<float*>(smem + L::kRing);
  float2 *sm = reinterpret_cast<float2*>(scratch + 2 * kThreads), *total = sm + p.ty * p.tx * E;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const Piece b(p, E, blockIdx.x);
  if (b.a >= p.frames()) return;
  typename L::In in;
  in.ring = smem_u32(smem) + threadIdx.x * 16;
  in.prime(p, b);
  if (MODE == kGrad) {
    gradient_sums<T, E>(p, b, in, sm, total);
    group_gradients(p, b, E, sm, scratch);
    channel_parts(p, b, E, total);
  } else {
    moments<T, E>(p, b, in, sm);
    group_moments(p, b, E, sm, scratch);
    if (MODE == kDigits && p.chunks == 1 && !p.cut) finish_groups<MODE>(p, b);
  }
}

// Frames of one piece per tile: sums, joining and rows in one block.
template <typename T, int E, int MODE>
__global__ void __launch_bounds__(kThreads, blocks_of(MODE)) whole_kernel(const __grid_constant__ NormParams p) {
  using L = Layout<T, E, MODE>;
  extern __shared__ __align__(16) uint8_t smem[];
  float* scratch = reinterpret_cast<float*>(smem + L::kRing);
  float2 *sm = reinterpret_cast<float2*>(scratch + 2 * kThreads), *total = sm + p.ty * p.tx * E;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  const Piece b(p, E, blockIdx.x);
  if (b.a >= p.frames()) return;
  typename L::In in;
  in.ring = smem_u32(smem) + threadIdx.x * 16;
  in.prime(p, b);
  if (MODE == kGrad) {
    gradient_sums<T, E>(p, b, in, sm, total);
    in.prime(p, b);  // the rows again, from L2
    group_gradients(p, b, E, sm, scratch);
    channel_parts(p, b, E, total);
  } else {
    moments<T, E>(p, b, in, sm);
    in.prime(p, b);
    group_moments(p, b, E, sm, scratch);
  }
  finish_groups<MODE>(p, b);
  __syncthreads();
  if (!b.mine) return;
  if (MODE == kGrad) gradient_rows<T, E>(p, b, in);
  else rows<T, E>(p, b, in);
}

// dW and db of 32 channels, over the pieces of rows of all frames.
__device__ __forceinline__ void channel_sums(const NormParams& p, int c0, float2* sm) {
  const int c = c0 + (threadIdx.x & 31), warp = threadIdx.x >> 5, n = p.frames() * p.chunks;
  float2 t = make_float2(0.f, 0.f);
  if (c < p.C)
#pragma unroll 8
    for (int i = warp; i < n; i += kThreads / 32) {
      const float2 u = p.channels[static_cast<int64_t>(i) * p.C + c];
      t.x += u.x;
      t.y += u.y;
    }
  sm[threadIdx.x] = t;
  __syncthreads();
  if (warp == 0 && c < p.C) {
    for (int w = 1; w < kThreads / 32; ++w) {
      t.x += sm[w * 32 + threadIdx.x].x;
      t.y += sm[w * 32 + threadIdx.x].y;
    }
    if (p.db) p.db[c] = t.x;
    if (p.dW) p.dW[c] = t.y;
  }
}

__global__ void __launch_bounds__(kThreads) channels_kernel(const __grid_constant__ NormParams p) {
  __shared__ float2 sm[kThreads];
  cudaGridDependencySynchronize();
  channel_sums(p, blockIdx.x * 32, sm);
}

template <typename T, int E, int MODE>
__global__ void __launch_bounds__(kThreads, blocks_of(MODE)) rows_kernel(const __grid_constant__ NormParams p) {
  using L = Layout<T, E, MODE>;
  extern __shared__ __align__(16) uint8_t smem[];
  // (the launches before this one have waited for what makes x, dy and the lists, so these may be read at once)
  const int n = p.frames() * static_cast<int>(p.by_pieces.d);
  const int i = n - 1 - (static_cast<int>(blockIdx.x) - p.wide);
  typename L::In in;
  if (MODE == kGrad && static_cast<int>(blockIdx.x) < p.wide) {  // beside the rows, whose means do not wait for these
    cudaGridDependencySynchronize();
    channel_sums(p, blockIdx.x * 32, reinterpret_cast<float2*>(smem));
    return;
  }
  if (i >= 0) {
    in.ring = smem_u32(smem) + threadIdx.x * 16;
    in.prime(p, Piece(p, E, i));
  }
  cudaGridDependencySynchronize();
  if (i < 0) return;
  const Piece b(p, E, i);
  if (!b.mine) return;
  if (MODE == kGrad) gradient_rows<T, E>(p, b, in);
  else rows<T, E>(p, b, in);
}

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------
// Tiles of whole groups where there are any of up to kTileVecs vectors, and 16 or more: of those the ones that leave
// the fewest threads idle.  Pieces of up to 32 rows of a thread, and as many as run at once (`slots`) when a third
// of up to 24 frames is active: how many are is known on the device only.  One or two frames have up to 64.
void shape(NormParams& p, int E, int slots) {
  const int nv = p.C / E, most = E == 1 ? kThreads : kTileVecs;
  p.tiles = (nv + most - 1) / most;
  p.tx = (nv + p.tiles - 1) / p.tiles;
  p.tiles = (nv + p.tx - 1) / p.tx;
  p.cut = 1;
  double best = 0;
  for (int t = p.tiles; t <= std::min(p.G, std::max(p.tiles, nv / 16)); ++t) {
    const int groups = (p.G + t - 1) / t, c = groups * p.cpg, tx = c / E;
    if ((p.G + groups - 1) / groups != t || c % E || tx > most) continue;
    // threads at work, on average over the tiles; a twentieth more is worth another tile
    const double used = static_cast<double>(kThreads / tx * tx) * p.G / (static_cast<double>(t) * groups);
    if (used > 1.05 * best) {
      best = used;
      p.tx = tx;
      p.tiles = t;
      p.cut = 0;
    }
  }
  p.ty = std::max(1, std::min({kThreads / p.tx, p.N, 32}));
  p.tile_groups = p.cut ? (p.tx * E - 1) / p.cpg + 2 : p.tx * E / p.cpg;
  const int64_t each = static_cast<int64_t>((p.N + p.ty - 1) / p.ty);  // rows of a thread in a frame
  const int64_t likely = p.F <= 2 ? p.F : std::min((p.F + 2) / 3, 8);
  const int64_t rows = std::min<int64_t>(p.F <= 2 ? 64 : 32, std::max<int64_t>(4, (each * p.tiles * likely + slots - 1) / slots));
  // (frames that a block goes through in the time of two launches are pieces by themselves)
  p.chunk_rows = static_cast<int>(each <= 32 ? p.N : std::min<int64_t>(p.N, rows * p.ty));
  p.chunks = (p.N + p.chunk_rows - 1) / p.chunk_rows;
}

// What all calls take: tokens, and pieces with their number in a launch's grid.
bool too_many_tokens(int F, int N) { return static_cast<int64_t>(F) * N > 0x7FFFFFFF - 65536; }
bool too_many_pieces(const NormParams& p) {
  return static_cast<int64_t>(p.F) * p.chunks * p.tiles > 0x7FFFFFFF - 65536;
}

// Workspace for any alignment: the pieces' sums, for the gradients all channels' too, and the joined ones.
// -1 where rows of all alignments have too many pieces.
int64_t norm_bytes(int F, int N, int C, int G, bool grad) {
  int64_t most = -1;
  for (int E : {1, 4, 8}) {
    if (C % E) continue;
    NormParams p{};
    p.F = F;
    p.N = N;
    p.C = C;
    p.G = G;
    p.cpg = C / G;
    shape(p, E, slots_of(grad ? kGrad : kRows));
    if (too_many_pieces(p)) continue;
    const int64_t pieces = static_cast<int64_t>(F) * p.chunks;
    most = std::max(most, 8 * (pieces * (static_cast<int64_t>(p.tiles) * p.tile_groups + (grad ? C : 0)) + static_cast<int64_t>(F) * G));
  }
  return most;
}

template <typename K, typename... A>
rf_status run(K kernel, int64_t grid, int64_t smem, const DeviceInfo& di, cudaStream_t st, const char* what,
              std::atomic<bool> (&done)[64], const A&... args) {
  if (smem + 1024 > 48 * 1024 && !done[di.device]) {  // (with what a kernel declares)
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, di.max_smem_optin - 1024))
      return fail(RF_ERR_CUDA, "cudaFuncSetAttribute(rf_group_norm)", e);
    done[di.device] = true;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cfg.stream = st;
  return launch_early(cfg, 1, what, kernel, args...);
}

template <typename T, int E, int MODE>
rf_status launch(NormParams& p, const DeviceInfo& di, cudaStream_t st, const char* what) {
  using L = Layout<T, E, MODE>;
  shape(p, E, slots_of(MODE));
  if (too_many_pieces(p)) return fail(RF_ERR_INVALID_ARG, "rf_group_norm: too many frames");
  p.by_cpg = FastDiv(static_cast<uint32_t>(p.cpg));
  p.by_tx = FastDiv(static_cast<uint32_t>(p.tx));
  p.by_ty = FastDiv(static_cast<uint32_t>(p.ty));
  p.by_tiles = FastDiv(static_cast<uint32_t>(p.tiles));
  p.by_pieces = FastDiv(static_cast<uint32_t>(p.chunks * p.tiles));
  for (p.seg = 1; p.seg < E && p.cpg % (2 * p.seg) == 0;) p.seg *= 2;
  p.group_segs = std::min(p.cpg, p.tx * E) / p.seg;
  p.by_segs = FastDiv(static_cast<uint32_t>(p.group_segs));
  p.w_vec = aligned16(p.weight) && aligned16(p.bias);
  const int64_t pieces = static_cast<int64_t>(p.F) * p.chunks * p.tiles;
  p.done = p.part + pieces * p.tile_groups;
  p.channels = p.done + static_cast<int64_t>(p.F) * p.G;
  static std::atomic<bool> done[3][64] = {};
  int64_t smem8 = 0;
  if (MODE == kDigits) {
    p.whole = reinterpret_cast<uintptr_t>(p.Y) % E == 0 && p.y_stride % E == 0;
    // the smallest team whose registers hold a row, a larger one where there are few rows
    const int nv = p.C / E;
    const int64_t rows = static_cast<int64_t>(p.F) * p.N;
    p.team = 4;
    while (p.team < kThreads && p.team * kDigitVecs<E> < nv) p.team *= 2;
    while (p.team < kThreads && 2 * p.team <= nv && rows * p.team < 152 * 2 * kThreads) p.team *= 2;
    p.segs = (nv + p.team * kDigitVecs<E> - 1) / (p.team * kDigitVecs<E>);
    smem8 = p.C * (E == 8 ? 14ll : 12ll) + kDigitVecs<E> * kThreads * 16;
    p.ring = sizeof(T) * E == 16 && p.segs == 1 && smem8 + 1024 <= di.max_smem_optin;
    if (!p.ring) smem8 = p.C * 12ll;
    if (smem8 + 1024 > di.max_smem_optin)  // (before the first launch: a call that is refused writes nothing)
      return fail(RF_ERR_UNSUPPORTED, "rf_group_norm: too many channels for rows of 8 bits");
    // whole waves of blocks, with 64 rows of a block and up where every frame is active
    p.blocks = std::max<int64_t>(p.F, 2 * 152 * std::max<int64_t>(1, rows / (2 * 152 * 64)));
  } else {
    p.whole = reinterpret_cast<uintptr_t>(p.Y) % (sizeof(T) * E) == 0 && p.y_stride % E == 0;
  }
  p.wide = MODE == kGrad && (p.dW || p.db) ? (p.C + 31) / 32 : 0;
  if constexpr (MODE != kDigits)
    if (p.chunks == 1 && !p.cut) {
      static std::atomic<bool> whole[2][64] = {};
      const rf_status e = run(whole_kernel<T, E, MODE>, pieces, L::sums_bytes(p), di, st, what, whole[0], p);
      return e || !p.wide ? e : run(channels_kernel, p.wide, 0, di, st, what, whole[1], p);
    }
  if (rf_status e = run(sums_kernel<T, E, MODE>, pieces, L::sums_bytes(p), di, st, what, done[0], p)) return e;
  if (MODE != kDigits || p.chunks > 1 || p.cut) {
    // a thread of a joining block has about eight pieces' sums of its group
    for (p.join_groups = 1; p.join_groups < std::min(32, p.G) && 2 * p.join_groups * p.chunks <= 8 * kThreads;)
      p.join_groups *= 2;
    const int64_t joins = static_cast<int64_t>(p.F) * ((p.G + p.join_groups - 1) / p.join_groups);
    if (rf_status e = run(join_kernel<MODE == kGrad ? kGrad : kRows>, joins, 0, di, st, what, done[1], p, E)) return e;
  }
  if constexpr (MODE == kDigits)
    return run(digits_kernel<T, E>, p.blocks, smem8, di, st, what, done[2], p);
  else
    return run(rows_kernel<T, E, MODE>, pieces + p.wide, std::max<int64_t>(L::kRing, kThreads * 8), di, st, what, done[2], p);
}

// By type and alignment: vectors of 16 bytes, or element by element.
template <int MODE>
rf_status launch_by_type(int dtype, bool vec, NormParams& p, const DeviceInfo& di, cudaStream_t s, const char* what) {
  if (dtype == RF_FP32)
    return vec ? launch<float, 4, MODE>(p, di, s, what) : launch<float, 1, MODE>(p, di, s, what);
  if (dtype == RF_FP16)
    return vec ? launch<__half, 8, MODE>(p, di, s, what) : launch<__half, 1, MODE>(p, di, s, what);
  return vec ? launch<__nv_bfloat16, 8, MODE>(p, di, s, what) : launch<__nv_bfloat16, 1, MODE>(p, di, s, what);
}

bool on_vectors(const void* p, int64_t row_bytes) { return aligned16(p) && row_bytes % 16 == 0; }

rf_status device(DeviceInfo* di) {
  if (rf_status st = current_device_info(di)) return st;
  if (di->cc_major != 10 || di->cc_minor != 3) return fail(RF_ERR_UNSUPPORTED, "needs sm_103");
  return RF_OK;
}
// What both directions of the norm take.
rf_status check_norm(const char* fn, int dtype, int F, int N, int C, int G, int w_dtype, int act,
                     const void* d_weight, const void* d_bias, const int32_t* d_active,
                     const int32_t* d_counts, const void* d_workspace, int64_t bytes, bool grad) {
  if (!dtype_bytes(dtype)) return fail(RF_ERR_UNSUPPORTED, fn);
  if (F < 1 || N < 1 || C < 1) return fail(RF_ERR_INVALID_ARG, fn);
  if (too_many_tokens(F, N)) return fail(RF_ERR_INVALID_ARG, "group norm: too many tokens");
  if (C > kMaxC) return fail(RF_ERR_INVALID_ARG, "group norm: more than 65536 channels");
  if (G < 1 || C % G) return fail(RF_ERR_INVALID_ARG, "group norm: channels are not whole groups");
  if (w_dtype != dtype && w_dtype != RF_FP32)
    return fail(RF_ERR_UNSUPPORTED, "group norm: weight and bias in the input's type or fp32");
  if (act < RF_ACT_NONE || act > RF_ACT_SILU) return fail(RF_ERR_INVALID_ARG, "group norm: act");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "group norm: active list and counts come together");
  if (reinterpret_cast<uintptr_t>(d_workspace) % 8 ||
      reinterpret_cast<uintptr_t>(d_weight) % dtype_bytes(w_dtype) ||
      reinterpret_cast<uintptr_t>(d_bias) % dtype_bytes(w_dtype))
    return fail(RF_ERR_MISALIGNED, "group norm: pointer not on its elements' boundary");
  const int64_t need = norm_bytes(F, N, C, G, grad);
  if (need < 0) return fail(RF_ERR_INVALID_ARG, "group norm: too many frames");
  if (bytes < need)
    return fail(RF_ERR_INVALID_ARG, "group norm: workspace below rf_group_norm_workspace_bytes");
  return RF_OK;
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" int64_t rf_group_norm_workspace_bytes(int F, int N, int C, int G, int dtype) {
  if (F < 1 || N < 1 || C < 1 || G < 1 || C % G || C > kMaxC || !dtype_bytes(dtype) || too_many_tokens(F, N))
    return -1;
  return norm_bytes(F, N, C, G, true);
}

extern "C" rf_status rf_group_norm(void* d_Y, int64_t y_row_stride, float* d_scale, const void* d_X,
                                   int64_t x_row_stride, int dtype, int F, int N, int C, int G,
                                   const void* d_weight, const void* d_bias, int w_dtype, float eps,
                                   int act, float* d_stats, void* d_workspace, int64_t workspace_bytes,
                                   const int32_t* d_active, const int32_t* d_counts,
                                   rf_stream_t stream) {
  if (!d_Y || !d_X || !d_workspace) return fail(RF_ERR_INVALID_ARG, "rf_group_norm: null pointer");
  if (rf_status st = check_norm("rf_group_norm: dtype or sizes", dtype, F, N, C, G, w_dtype, act,
                                d_weight, d_bias, d_active, d_counts, d_workspace, workspace_bytes, false))
    return st;
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(RF_ERR_INVALID_ARG, "rf_group_norm: eps >= 0");
  if (x_row_stride < C || y_row_stride < C)
    return fail(RF_ERR_INVALID_ARG, "rf_group_norm: row stride below the row's length");
  if (d_Y == d_X && (d_scale || (x_row_stride != y_row_stride && static_cast<int64_t>(F) * N > 1)))
    return fail(RF_ERR_INVALID_ARG, "rf_group_norm: in place with two strides or types");
  const int es = dtype_bytes(dtype), eo = d_scale ? 1 : es;
  if (reinterpret_cast<uintptr_t>(d_X) % es || reinterpret_cast<uintptr_t>(d_Y) % eo ||
      reinterpret_cast<uintptr_t>(d_scale) % 4 || reinterpret_cast<uintptr_t>(d_stats) % 8)
    return fail(RF_ERR_MISALIGNED, "rf_group_norm: pointer not on its elements' boundary");
  DeviceInfo di;
  if (rf_status st = device(&di)) return st;
  NormParams p{};
  p.N = N;
  p.C = C;
  p.G = G;
  p.cpg = C / G;
  p.active = d_active;
  p.counts = d_counts;
  p.F = F;
  p.X = d_X;
  p.Y = d_Y;
  p.weight = d_weight;
  p.bias = d_bias;
  p.w32 = w_dtype == RF_FP32;
  p.x_stride = x_row_stride;
  p.y_stride = y_row_stride;
  p.stats = d_stats;
  p.part = static_cast<float2*>(d_workspace);
  p.scale = d_scale;
  p.act = act;
  p.eps = eps;
  const bool vec = static_cast<int64_t>(C) * es % 16 == 0 && on_vectors(d_X, x_row_stride * es);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return d_scale ? launch_by_type<kDigits>(dtype, vec, p, di, s, "rf_group_norm launch")
                 : launch_by_type<kRows>(dtype, vec, p, di, s, "rf_group_norm launch");
}

extern "C" rf_status rf_group_norm_bwd(void* d_dX, int64_t dx_row_stride, float* d_dW, float* d_db,
                                       const void* d_dY, int64_t dy_row_stride, const void* d_X,
                                       int64_t x_row_stride, const float* d_stats, int dtype, int F,
                                       int N, int C, int G, const void* d_weight, const void* d_bias,
                                       int w_dtype, int act, void* d_workspace,
                                       int64_t workspace_bytes, const int32_t* d_active,
                                       const int32_t* d_counts, rf_stream_t stream) {
  if (!d_dX || !d_dY || !d_X || !d_stats || !d_workspace)
    return fail(RF_ERR_INVALID_ARG, "rf_group_norm_bwd: null pointer");
  if (rf_status st = check_norm("rf_group_norm_bwd: dtype or sizes", dtype, F, N, C, G, w_dtype, act,
                                d_weight, d_bias, d_active, d_counts, d_workspace, workspace_bytes, true))
    return st;
  if (x_row_stride < C || dx_row_stride < C || dy_row_stride < C)
    return fail(RF_ERR_INVALID_ARG, "rf_group_norm_bwd: row stride below the row's length");
  if (static_cast<int64_t>(F) * N > 1 && ((d_dX == d_X && dx_row_stride != x_row_stride) ||
                                          (d_dX == d_dY && dx_row_stride != dy_row_stride)))
    return fail(RF_ERR_INVALID_ARG, "rf_group_norm_bwd: in place with two strides");
  const int es = dtype_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(d_X) % es || reinterpret_cast<uintptr_t>(d_dX) % es ||
      reinterpret_cast<uintptr_t>(d_dY) % es || reinterpret_cast<uintptr_t>(d_stats) % 8 ||
      reinterpret_cast<uintptr_t>(d_dW) % 4 || reinterpret_cast<uintptr_t>(d_db) % 4)
    return fail(RF_ERR_MISALIGNED, "rf_group_norm_bwd: pointer not on its elements' boundary");
  DeviceInfo di;
  if (rf_status st = device(&di)) return st;
  NormParams p{};
  p.N = N;
  p.C = C;
  p.G = G;
  p.cpg = C / G;
  p.active = d_active;
  p.counts = d_counts;
  p.F = F;
  p.X = d_X;
  p.dY = d_dY;
  p.Y = d_dX;
  p.weight = d_weight;
  p.bias = d_bias;
  p.w32 = w_dtype == RF_FP32;
  p.x_stride = x_row_stride;
  p.dy_stride = dy_row_stride;
  p.y_stride = dx_row_stride;
  p.stats = const_cast<float*>(d_stats);
  p.part = static_cast<float2*>(d_workspace);
  p.dW = d_dW;
  p.db = d_db;
  p.act = act;
  const bool vec = static_cast<int64_t>(C) * es % 16 == 0 && on_vectors(d_X, x_row_stride * es) &&
                   on_vectors(d_dX, dx_row_stride * es) && on_vectors(d_dY, dy_row_stride * es);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return launch_by_type<kGrad>(dtype, vec, p, di, s, "rf_group_norm_bwd launch");
}
