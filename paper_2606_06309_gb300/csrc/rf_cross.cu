// rf_cross.cu -- attention of the active frames' tokens to an encoder's states (tcgen05 / TMEM /
// TMA).
//
//     O[t, h] = sum_j p_j v_j,   p = softmax_j(scale q_{t,h} . k_j)   h: query head, key head h / g
//
// over the keys j of the token's frame: all L states, or the frame's own range of them, without the
// masked ones.  A row that sees no key gets O = 0 and LSE = -inf.
//
// One CTA per SM, 384 threads, in the roles of the step core's attention: warp 0 brings query tiles
// and K/V tiles of 128 keys by TMA, warps 1 and 2 issue the products of query tile A and B (S = Q
// K^T, O += P V, P over S in tensor memory), warpgroups 1 and 2 hold the running maximum and sum of
// their tile's rows in registers, fp32, and rescale O only when a row's maximum grows by more than
// 2^8.  Encoder states are few: an item (a pair of query tiles over one frame's keys) is often only
// four K/V tiles long, so the next item's queries and keys are loaded, and its first product
// issued, while the softmax warps still write the last one's rows.
//
// What masked keys hold must not matter, and 0 * NaN is NaN in a product: their scores are replaced
// by -inf before anything is computed with them, and warp 3 sets their rows of V to zero in shared
// memory before P V reads them (launches with ranges or a mask; past the last state TMA fills in
// zeros by itself).  What a mask leaves out at the ends is not visited; where it leaves few states
// between, and all rows see the same, only those are brought: K and V row by row (TMA gather, four
// rows an instruction, K by warp 0, V by warp 3), so that an item is as long as what is seen.
//
// Query rows.  Without ranges the active tokens are one list of rows (a frame padded to a multiple
// of 8, so that a tile across frames is gathered in boxes of 8 rows); with ranges a tile stays in
// its frame.  Where a frame's tokens times the query heads of a key head fit a tile, they are its
// rows together (`packed`): K and V are then read once for all of these heads, which is what a
// launch of few rows costs.
//
// Few items: the K/V tiles of an item are dealt to a cluster of up to 8 CTAs.  Each leaves its
// unnormalised rows, maxima and sums in its shared memory, and each joins a share of the columns
// from all of them, in the order of the ranges.
//
// Measured (device time, calls one after another):
//   75,600 tokens, 40 heads of 128, 512 states: 541 us, 1.47 PFLOP/s on one set of inputs (609 us with
//     inputs that change from call to call, when the power limit lowers the clock).  An item of 4 K/V
//     tiles takes 13,200 cycles: 9,200 in its steps, of which the products are 8,200, and 4,000 from
//     the last product to the next item's first P.
//   6,240 of 20,280 tokens, 12 heads, 512 states: 20.1 us: 300 items, two for nearly every SM, and the
//     launch's start and end.
//   16 sequences of one token, 12 heads, 32,000 states in 16 ranges: 44.5 us, 4.4 TB/s of K and V: the
//     longest sequence's tiles on the SMs that share it.
//   20 of 33 frames of 1003 tokens, 24 heads on 6 of 64, windows of 1500 states with masked ones: 68 us.
//     Items of two or three K/V tiles: half of the time is the change from item to item.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "rf_ops.h"
#include "rf_rows.cuh"
#include "rf_stage.cuh"
#include "rf_tc_ptx.cuh"

namespace rf {
namespace {

// Which keys a launch may leave out: none, some (ranges), or, under a mask without ranges, some
// that are the same for all rows (they may be gathered).
constexpr int kAllKeys = 0, kSomeKeys = 1, kSameKeys = 2;
constexpr int kBM = 128, kBN = 128;  // rows of a query tile, keys of a K/V tile
constexpr int kThreads = 384;        // three warpgroups
// Registers after setmaxnreg: 128 * 104 + 256 * 200 = 64512 = 384 * 168, what the launch holds.
constexpr int kRegsLaunch = 168, kRegsControl = 104, kRegsSoftmax = 200;
static_assert(128 * kRegsControl + 256 * kRegsSoftmax <= kThreads * kRegsLaunch, "register split");
constexpr uint32_t kTmemCols = 512;  // S_A, S_B at 0, 128; O_A, O_B at 256, 384
constexpr uint64_t kDrainLimitNs = 200000000ull;  // 0.2 s for what is in flight at teardown
constexpr float kRescaleLog2 = 8.0f;
// P goes to the tile's MMA warp in two parts of 64 keys, and the two MMA warps take turns, over
// hardware named barriers.  Those have no time limit: who waits on one is always released, by the
// arrivals of the normal path or, after a bounded wait elsewhere gave up, by release_mma.
constexpr int kPThreads = 128 + 32;
__device__ __forceinline__ int p_barrier(int X, int part) { return 1 + 2 * X + part; }
__device__ __forceinline__ int turn_barrier(int X) { return 5 + X; }

struct CrossParams {
  uint16_t* O;
  float* lse;
  const int2* kv_range;     // [F] or null
  const uint8_t* key_mask;  // [L] or null
  int32_t* status;
  RowMap rows;
  int64_t o_row_stride;
  int L, g;            // g: query heads per key head
  int units;           // heads an item is of: query heads, or key heads where packed
  int packed;          // rows of a tile are (frame, token, query head of the key head)
  int frame_rows;      // packed: rows of a frame, N * g
  int tile_frames;     // packed: frames of a tile
  int tile_rows;       // not packed: rows of a tile
  int cluster;
  float scale_log2;
  FastDiv by_g, by_frame_rows, by_units;
};

__device__ __forceinline__ void flag_error(const CrossParams& p, int where) {
  if (p.status) atomicOr(p.status, RF_ERR_DEVICE_TIMEOUT | (1 << (8 + where)));
}
__device__ __forceinline__ bool all_wait(uint32_t bar, uint32_t parity, volatile int* abort) {
  return warp_wait<false>(bar, parity, abort);
}

// The work of a launch, from the active count on the device.
constexpr int kMaxSorted = 256, kSortRounds = 8;
struct Work {
  int rows;  // of a tile
  int A, groups, tiles, pairs, items;  // groups of tiles with keys of their own (frames, or one)
  int first, step[2];  // this CTA's items: the steps to the next one, in turn
  FastDiv by_pairs;
  // Launches with ranges and a few items per CTA: the frames by falling length.  The items are
  // dealt to the CTAs from the first to the last, then from the last to the first, and so on, so
  // that who has a long one of a round has a short one of the next (16 sequences of 1000, 2000 and
  // 3000 states x 12 heads, in their own order 48 K/V tiles for the busiest CTA, this way 24: 66 us
  // -> 46; with many rounds lengths even out, and the order costs 2 us at the start).
  bool sorted;
  int lo, hi;  // no state before lo or from hi on is seen: what the mask pads at the ends is not visited
  // Masks without ranges that leave few states between: only those are brought, by their rows (TMA
  // gather), and the keys of an item are the `seen` ones, numbered from 0.
  bool gather;
  int seen;
  uint8_t order[kMaxSorted];
};
template <int D>
struct Cfg {
  static constexpr int kHalves = D / 64;           // 128-byte swizzle atoms across the head dim
  static constexpr int kTileBytes = 128 * D * 2;   // one tile of Q, K or V
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kSlots = D == 128 ? 4 : 8;  // K in even slots, V in odd ones
  static constexpr int kOffKV = 2 * kTileBytes;
  static constexpr int kOffStage = kOffKV + kSlots * kTileBytes;  // rows of results, per softmax warp
  static constexpr int kOffBar = kOffStage + 8 * kTurnBytes;
  static constexpr int kQFull = 0, kQEmpty = 2, kKVFull = 4, kKVEmpty = 4 + kSlots,
                       kVClean = 4 + 2 * kSlots, kSFull = 4 + 3 * kSlots, kODone = kSFull + 2,
                       kDrain = kODone + 2, kBars = kDrain + 2;
  static constexpr int kOffMisc = kOffBar + kBars * 8;  // tensor memory address, abort, MMA done [2]
  static constexpr int kOffList = kOffMisc + 32;        // boxes of the query tiles
  static constexpr int kOffKeys = kOffList + 2 * static_cast<int>(sizeof(BoxList<kBM>));
  static constexpr int kOffWork = kOffKeys + 2 * kBN * 4;  // kOffKeys: keys of a gathered tile of K, of V
  static constexpr int kSmem = kOffWork + static_cast<int>(sizeof(Work));
  // A split item's rows: [tile][D / 4][128] float4 over the K/V ring, {max, sum} [tile][128] over
  // the queries
  static_assert(2 * 128 * D * 4 <= kSlots * kTileBytes, "partial rows fit the ring");
};

template <int KEYS>
__device__ __forceinline__ bool gathers(const Work& w) {
  return KEYS == kSameKeys && w.gather;
}
__device__ __forceinline__ void make_work(const CrossParams& p, Work& w) {
  w.rows = p.tile_rows;
  w.A = p.rows.frames();
  w.groups = p.kv_range ? w.A : 1;
  if (p.packed)
    w.tiles = p.kv_range ? 1 : (w.A + p.tile_frames - 1) / p.tile_frames;
  else
    w.tiles = ((p.kv_range ? p.rows.N : w.A * p.rows.Np) + w.rows - 1) / w.rows;
  w.pairs = (w.tiles + 1) / 2;
  w.items = p.units * w.groups * w.pairs;
  w.lo = 0;
  w.hi = p.L;
  w.gather = false;
  w.seen = 0;
  const int ctas = gridDim.x / p.cluster;  // (or clusters)
  w.first = blockIdx.x / p.cluster;
  w.sorted = p.kv_range && w.groups > 1 && w.groups <= kMaxSorted && w.items > ctas &&
             w.items <= kSortRounds * ctas;
  w.step[0] = w.sorted ? 2 * (ctas - 1 - w.first) + 1 : ctas;
  w.step[1] = w.sorted ? 2 * w.first + 1 : ctas;
  w.by_pairs = FastDiv(max(w.pairs, 1));
}
// K/V tiles of a frame's range.
__device__ __forceinline__ int range_tiles(const CrossParams& p, const Work& w, int frame, int& begin,
                                           int& end) {
  const int2 r = p.kv_range ? p.kv_range[frame] : make_int2(0, p.L);
  begin = min(max(r.x, w.lo), w.hi);
  end = min(max(r.y, begin), w.hi);
  return (end - begin + kBN - 1) / kBN;
}
// All threads of the block: w.lo, w.hi and the number of states seen from the mask (L bytes; a word
// of 4 at a time where it lies on their boundary), and whether they are gathered.
template <int KEYS>
__device__ __forceinline__ void trim_states(const CrossParams& p, Work& w, int rank) {
  if (threadIdx.x == 0) {
    w.lo = p.L;
    w.hi = 0;
  }
  __syncthreads();
  int lo = p.L, hi = 0, seen = 0;
  if ((reinterpret_cast<uintptr_t>(p.key_mask) & 3) == 0 && p.L >= 4) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(p.key_mask);
#pragma unroll 4
    for (int i = threadIdx.x; i < p.L >> 2; i += kThreads)
      if (const uint32_t v = words[i]) {
        lo = min(lo, 4 * i + ((__ffs(v) - 1) >> 3));
        hi = max(hi, 4 * i + 4 - (__clz(v) >> 3));
        seen += __popc((((v & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | v) & 0x80808080u);
      }
    for (int k = (p.L & ~3) + threadIdx.x; k < p.L; k += kThreads)
      if (p.key_mask[k]) {
        lo = min(lo, k);
        hi = max(hi, k + 1);
        ++seen;
      }
  } else {
    for (int k = threadIdx.x; k < p.L; k += kThreads)
      if (p.key_mask[k]) {
        lo = min(lo, k);
        hi = max(hi, k + 1);
        ++seen;
      }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  seen = __reduce_add_sync(0xffffffffu, seen);
  if ((threadIdx.x & 31) == 0) {
    atomicMin(&w.lo, lo);
    atomicMax(&w.hi, hi);
    atomicAdd(&w.seen, seen);
  }
  __syncthreads();
  if (KEYS != kSameKeys || w.seen == 0) return;
  lo = w.lo;
  const int span = w.hi - lo;
  // Gathered where that leaves half of the tiles or fewer; a tile by rows takes 1.4 (head dim 64)
  // to 1.8 times (128) a whole one's time, in issuing.  Tiles, us gathered against us whole: 6240
  // tokens, 12 heads of 128, 2048 states: 4 of 16 40.0 / 78.2, 8 54.4 / 64.3, 12 72.9 / 59.6; 20
  // frames of 1003 tokens, 24 heads of 64, 1500 states: 6 of 12 189 / 252, 9 249 / 245.  The same
  // in all CTAs of a cluster.
  if ((w.seen + kBN - 1) / kBN * 2 > (span + kBN - 1) / kBN) return;
  if (p.cluster > 1) {  // a CTA's share is one of all states, with what is seen of them
    hi = lo + static_cast<int>(static_cast<int64_t>(span) * (rank + 1) / p.cluster);
    lo += static_cast<int>(static_cast<int64_t>(span) * rank / p.cluster);
    seen = 0;
    for (int k = lo + threadIdx.x; k < hi; k += kThreads) seen += p.key_mask[k] != 0;
    seen = __reduce_add_sync(0xffffffffu, seen);
    __syncthreads();  // read by all
    if (threadIdx.x == 0) {
      w.lo = lo;
      w.hi = hi;
      w.seen = 0;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) atomicAdd(&w.seen, seen);
  }
  if (threadIdx.x == 0) w.gather = true;
  __syncthreads();
}
// All threads of the block; `tiles`: room for kMaxSorted numbers.
__device__ __forceinline__ void sort_frames(const CrossParams& p, Work& w, int* tiles) {
  const int i = threadIdx.x;
  int begin, end, mine = 0, rank = 0;
  if (i < w.groups) tiles[i] = mine = range_tiles(p, w, p.rows.frame(i), begin, end);
  __syncthreads();
  if (i < w.groups) {
    for (int j = 0; j < w.groups; ++j)
      rank += tiles[j] > mine || (tiles[j] == mine && j < i);
    w.order[rank] = static_cast<uint8_t>(i);
  }
  __syncthreads();
}

// One item, or a cluster CTA's share of it: a pair of query tiles of a head over key rows
// [begin + 128 j0, ...) of the range [begin, end).
struct Item {
  int unit, group, pair;
  int begin, end, j0, j1;
};
template <int KEYS>
__device__ __forceinline__ Item get_item(const CrossParams& p, const Work& w, int i, int rank) {
  Item t;
  const int gp = w.by_pairs.div(i);
  t.pair = i - gp * w.pairs;
  const int slot = p.by_units.div(gp);
  t.unit = gp - slot * p.units;
  t.group = w.sorted ? w.order[slot] : slot;
  t.j0 = 0;
  if (gathers<KEYS>(w)) {
    t.begin = 0;
    t.end = w.seen;
    t.j1 = (w.seen + kBN - 1) / kBN;
    return t;
  }
  const int nt =  // below 2^24
      range_tiles(p, w, p.kv_range ? p.rows.frame(t.group) : 0, t.begin, t.end);
  t.j1 = nt;
  if (p.cluster > 1) {
    t.j0 = nt * rank / p.cluster;
    t.j1 = nt * (rank + 1) / p.cluster;
  }
  return t;
}

// Token and query head of a tile's row; token -1 where the row is none.
__device__ __forceinline__ int row_of(const CrossParams& p, const Work& w, const Item& t, int tile,
                                      int row, int& head) {
  head = t.unit;
  if (p.packed) {
    const int al = p.by_frame_rows.div(row), rem = row - al * p.frame_rows;
    const int a = p.kv_range ? t.group : tile * p.tile_frames + al;
    if (al >= p.tile_frames || a >= w.A) return -1;
    const int q = p.by_g.div(rem);
    head = t.unit * p.g + (rem - q * p.g);
    return p.rows.frame(a) * p.rows.N + q;
  }
  const int r = tile * w.rows + row;
  if (row >= w.rows) return -1;
  if (p.kv_range) return r < p.rows.N ? p.rows.frame(t.group) * p.rows.N + r : -1;
  if (r >= w.A * p.rows.Np) return -1;
  const int a = p.rows.by_Np.div(r), q = r - a * p.rows.Np;
  return q < p.rows.N ? p.rows.frame(a) * p.rows.N + q : -1;
}

// Whether a tile's row is one: row_of(...) >= 0, without the active list.
__device__ __forceinline__ bool is_row(const CrossParams& p, const Work& w, const Item& t, int tile,
                                       int row) {
  if (p.packed) {
    const int al = p.by_frame_rows.div(row);
    return al < p.tile_frames && (p.kv_range || tile * p.tile_frames + al < w.A);
  }
  const int r = tile * w.rows + row;
  if (p.kv_range) return r < p.rows.N;
  return row < w.rows && r < w.A * p.rows.Np && r - p.rows.by_Np.div(r) * p.rows.Np < p.rows.N;
}

// The first of the 128 consecutive tokens of one head that a tile's rows are, or -1: rows of
// several frames or heads, or fewer than 128.
__device__ __forceinline__ int whole_tile(const CrossParams& p, const Work& w, const Item& t, int tile) {
  const int r = tile * kBM;
  if (p.packed || w.rows < kBM) return -1;
  if (p.kv_range) return r + kBM <= p.rows.N ? p.rows.frame(t.group) * p.rows.N + r : -1;
  const int a = p.rows.by_Np.div(r), q = r - a * p.rows.Np;
  return a < w.A && q + kBM <= p.rows.N ? p.rows.frame(a) * p.rows.N + q : -1;
}

// Which keys of tile j a row may see: bit c of word c / 32.  Warp-collective, in two parts so that
// the mask's bytes can be on their way meanwhile: this lane's keys (bit i: key lane + 32 i), and
// all.
struct KeyBits {
  uint32_t w[4];
  __device__ __forceinline__ bool all() const {
    return (w[0] & w[1] & w[2] & w[3]) == 0xFFFFFFFFu;
  }
};
// gather: all keys of the item are seen.
__device__ __forceinline__ uint32_t own_keys(const CrossParams& p, bool gather, const Item& t,
                                             int j) {
  const int k0 = t.begin + j * kBN + (threadIdx.x & 31);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = k0 + 32 * i;
    if (k < t.end && (gather || !p.key_mask || p.key_mask[k] != 0)) m |= 1u << i;
  }
  return m;
}
__device__ __forceinline__ KeyBits all_keys(uint32_t own) {
  KeyBits b;
#pragma unroll
  for (int i = 0; i < 4; ++i) b.w[i] = __ballot_sync(0xffffffffu, (own >> i) & 1u);
  return b;
}

// ---------------------------------------------------------------------------------------
// TMA producer
// ---------------------------------------------------------------------------------------
// The states that the mask lets through, in order, 128 at a time.  Warp-collective.
struct KeyWalk {
  const uint8_t* mask;
  int hi, pos;          // pos: first of the 128 states at hand
  uint32_t own, ahead;  // this lane's of them that are still to come (bit i: pos + lane + 32 i); the next 128
  __device__ __forceinline__ uint32_t read(int k0) const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = k0 + (threadIdx.x & 31) + 32 * i;
      if (k < hi && mask[k] != 0) m |= 1u << i;
    }
    return m;
  }
  __device__ __forceinline__ void start(const CrossParams& p, const Work& w) {
    mask = p.key_mask;
    hi = w.hi;
    pos = w.lo;
    own = read(pos);
    ahead = read(pos + kBN);
  }
  // The next 128 into `keys`; behind the last one the first of the tile again.
  __device__ __forceinline__ void tile(int* keys) {
    const int lane = threadIdx.x & 31;
    const uint32_t below = (1u << lane) - 1;
    const int from = pos;
    int fill = 0;
#pragma unroll 1
    while (fill < kBN && pos < hi) {
      const KeyBits b = all_keys(own);
      uint32_t left = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((own >> i) & 1u) {
          const int at = fill + __popc(b.w[i] & below);
          if (at < kBN) keys[at] = pos + lane + 32 * i;
          else left |= 1u << i;
        }
        fill += __popc(b.w[i]);
      }
      if (fill > kBN) {
        own = left;
      } else {
        own = ahead;
        pos += kBN;
        ahead = read(pos + kBN);
      }
    }
    __syncwarp();
    const int first = fill > 0 ? keys[0] : min(from, hi - 1);
    for (int i = fill + lane; i < kBN; i += 32) keys[i] = first;
    __syncwarp();
  }
};
// Their rows of K or V (one thread).
template <int D>
__device__ __forceinline__ void gather_tile(const CUtensorMap* map, const int* keys, int hk,
                                            uint32_t dst, uint32_t bar) {
#pragma unroll 1
  for (int i = 0; i < kBN / 4; i += 8) {
    int4 r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = reinterpret_cast<const int4*>(keys)[i + k];
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int hb = 0; hb < Cfg<D>::kHalves; ++hb)
        tma_gather4(dst + hb * Cfg<D>::kHalfBytes + (i + k) * 512, map, bar, hk * D + hb * 64, r[k]);
  }
}

// The maps of Q: boxes of a tile, of kBoxRows rows, and of rows.unit rows or (packed) a frame.
struct QueryMaps {
  const CUtensorMap *whole, *many, *unit;
};
// What an item's loads need, found before they can be issued.
struct Load {
  Item t;
  RowBoxes x0, x1;
};
template <int D, int KEYS>
__device__ __forceinline__ void prepare_load(const QueryMaps& maps, const CrossParams& p,
                                             const Work& w, int i, int rank, BoxList<kBM>* list, bool lead,
                                             Load& n) {
  n.t = get_item<KEYS>(p, w, i, rank);
  if (p.packed || n.t.j0 >= n.t.j1) return;
#pragma unroll 1
  for (int X = 0; X < 2; ++X) {
    const int tile = 2 * n.t.pair + X;
    if (tile >= w.tiles) break;
    const RowBoxes x =
        p.kv_range ? RowBoxes{kBM, 0, 0, p.rows.frame(n.t.group) * p.rows.N + tile * kBM}
                   : list_boxes(p.rows, w.A * p.rows.Np, tile * w.rows, w.rows, kBM, list[X]);
    (X ? n.x1 : n.x0) = x;
    // on their way to L2 while the item before is worked on: the queries' own buffer is free only
    // when that item's last Q K^T is done
    if (lead && x.n_many + x.n_unit == 0)
#pragma unroll
      for (int hb = 0; hb < Cfg<D>::kHalves; ++hb)
        tma_prefetch_3d(maps.whole, hb * 64, n.t.unit, x.tok);
  }
}
template <int D>
__device__ __forceinline__ void load_queries(const QueryMaps& maps, const CrossParams& p,
                                             const Work& w, const Item& t, int tile,
                                             const RowBoxes& x, const BoxList<kBM>& list, uint32_t dst,
                                             uint32_t bar) {
  using C = Cfg<D>;
  auto load = [&](const CUtensorMap* m, int row, int head, int tok) {
#pragma unroll
    for (int hb = 0; hb < C::kHalves; ++hb)
      tma_load_3d(dst + hb * C::kHalfBytes + row * 128, m, bar, hb * 64, head, tok);
  };
  if (p.packed) {
    // one box per frame: its tokens, and for each the query heads of the key head
    const int a0 = p.kv_range ? t.group : tile * p.tile_frames;
    const int n = min(p.tile_frames, w.A - a0);
    mbar_arrive_expect_tx(bar, n * p.frame_rows * 128 * C::kHalves);
#pragma unroll 1
    for (int i = 0; i < n; ++i)
      load(maps.unit, i * p.frame_rows, t.unit * p.g, p.rows.frame(a0 + i) * p.rows.N);
    return;
  }
  mbar_arrive_expect_tx(bar, x.rows * 128 * C::kHalves);
  if (x.n_many + x.n_unit == 0) {
    load(maps.whole, 0, t.unit, x.tok);
    return;
  }
#pragma unroll 1
  for (int i = 0; i < x.n_many; ++i) load(maps.many, list.row[i], t.unit, list.tok[i]);
#pragma unroll 1
  for (int i = kBM - x.n_unit; i < kBM; ++i) load(maps.unit, list.row[i], t.unit, list.tok[i]);
}

// GATHER: w.gather (two copies of the loop: with a branch in it, whole tiles took 4 to 10% longer).
template <int D, int KEYS, bool GATHER>
__device__ __forceinline__ void producer(const QueryMaps& maps, const CUtensorMap* tmK,
                                         const CUtensorMap* tmV, const CUtensorMap* tmRowsK,
                                         const CrossParams& p, const Work& w, int rank,
                                         BoxList<kBM>* list, int* keys, uint32_t sQ0,
                                         uint32_t sKV0, uint32_t bar0, volatile int* abort) {
  using C = Cfg<D>;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const bool lead = elect_one();
  int q_cnt0 = 0, q_cnt1 = 0;
  int it = 0;
  bool ok = true;
  KeyWalk walk;
  Load n;
  int i = w.first, turn = 0;
  if (i < w.items) prepare_load<D, KEYS>(maps, p, w, i, rank, list, lead, n);
  while (ok && i < w.items) {
    const Item t = n.t;
    const int hk = p.packed ? t.unit : p.by_g.div(t.unit);
    // K and V of the tiles in turn.  The first keys go before the queries: their slot is free
    // earlier
    if (GATHER) walk.start(p, w);
#pragma unroll 1
    for (int n2 = 2 * t.j0; ok && n2 < 2 * t.j1; ++n2) {
      const int s = it % C::kSlots;
      if (GATHER) {
        if (n2 & 1) {  // warp 3 brings V
          ++it;
          continue;
        }
        walk.tile(keys);
      }
      ok = all_wait(bar(C::kKVEmpty + s), ((it / C::kSlots) & 1) ^ 1, abort);
      if (!ok) break;
      if (lead) {
        const CUtensorMap* m = (n2 & 1) ? tmV : tmK;
        mbar_arrive_expect_tx(bar(C::kKVFull + s), C::kTileBytes);
        if (GATHER)
          gather_tile<D>(tmRowsK, keys, hk, sKV0 + s * C::kTileBytes, bar(C::kKVFull + s));
        else
#pragma unroll
        for (int hb = 0; hb < C::kHalves; ++hb)
          tma_load_3d(sKV0 + s * C::kTileBytes + hb * C::kHalfBytes, m, bar(C::kKVFull + s),
                      hb * 64, hk, t.begin + (n2 >> 1) * kBN);
      }
      __syncwarp();
      ++it;
      if (n2 != 2 * t.j0) continue;
#pragma unroll 1
      for (int X = 0; X < 2; ++X) {
        const int tile = 2 * t.pair + X;
        if (tile >= w.tiles) break;
        ok = all_wait(bar(C::kQEmpty + X), ((X ? q_cnt1 : q_cnt0) & 1) ^ 1, abort);
        if (!ok) break;
        if (lead)
          load_queries<D>(maps, p, w, t, tile, X ? n.x1 : n.x0, list[X], sQ0 + X * C::kTileBytes,
                          bar(C::kQFull + X));
        __syncwarp();
        (X ? q_cnt1 : q_cnt0) += 1;
      }
    }
    i += w.step[turn];
    turn ^= 1;
    if (ok && i < w.items) prepare_load<D, KEYS>(maps, p, w, i, rank, list, lead, n);
  }
  if (!ok && lead) flag_error(p, 0);
  // every copy has landed
#pragma unroll 1
  for (int s = 0; s < C::kSlots; ++s)
    if (it > s) mbar_drain(bar(C::kKVFull + s), ((it - 1 - s) / C::kSlots) & 1, kDrainLimitNs);
  if (q_cnt0 > 0) mbar_drain(bar(C::kQFull), (q_cnt0 - 1) & 1, kDrainLimitNs);
  if (q_cnt1 > 0) mbar_drain(bar(C::kQFull + 1), (q_cnt1 - 1) & 1, kDrainLimitNs);
}

// ---------------------------------------------------------------------------------------
// V rows of keys that may not be seen (warp 3)
// ---------------------------------------------------------------------------------------
// Rows of a tile of V whose keys are not in `seen`.
template <int D>
__device__ __forceinline__ void clear_rows(uint8_t* tile, const KeyBits& seen) {
  const int lane = threadIdx.x & 31;
  // a row is 128 bytes in each half: the swizzle moves 16-byte pieces within them
#pragma unroll 1
  for (int r = lane; r < kBN; r += 32)
    if (!((seen.w[r >> 5] >> lane) & 1u))
#pragma unroll
      for (int hb = 0; hb < Cfg<D>::kHalves; ++hb)
#pragma unroll
        for (int q = 0; q < 8; ++q)
          *reinterpret_cast<uint4*>(tile + hb * Cfg<D>::kHalfBytes + r * 128 + q * 16) =
              make_uint4(0u, 0u, 0u, 0u);
}
// Gathered states: warp 3 brings the tiles of V, and clears what follows the last state.
template <int D, int KEYS>
__device__ __forceinline__ void gather_values(const CUtensorMap* tmRowsV, const CrossParams& p,
                                              const Work& w, int rank, int* keys, uint32_t sKV0,
                                              uint8_t* kv, uint32_t bar0, volatile int* abort) {
  using C = Cfg<D>;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const bool lead = elect_one();
  int it = 1;  // V follows K in the ring
  bool ok = true;
  KeyWalk walk;
#pragma unroll 1
  for (int i = w.first, turn = 0; ok && i < w.items; i += w.step[turn], turn ^= 1) {
    const Item t = get_item<KEYS>(p, w, i, rank);
    const int hk = p.packed ? t.unit : p.by_g.div(t.unit);
    walk.start(p, w);
#pragma unroll 1
    for (int j = t.j0; ok && j < t.j1; ++j, it += 2) {
      const int s = it % C::kSlots;
      walk.tile(keys);
      ok = all_wait(bar(C::kKVEmpty + s), ((it / C::kSlots) & 1) ^ 1, abort);
      if (!ok) break;
      if (lead) {
        mbar_arrive_expect_tx(bar(C::kKVFull + s), C::kTileBytes);
        gather_tile<D>(tmRowsV, keys, hk, sKV0 + s * C::kTileBytes, bar(C::kKVFull + s));
      }
      __syncwarp();
      if (j + 1 == t.j1 && w.seen % kBN != 0) {
        ok = all_wait(bar(C::kKVFull + s), (it / C::kSlots) & 1, abort);
        if (!ok) break;
        clear_rows<D>(kv + s * C::kTileBytes, all_keys(own_keys(p, true, t, j)));
        fence_proxy_async();
        __syncwarp();
        if (lead) mbar_arrive(bar(C::kVClean + s));
      }
    }
  }
  if (!ok && lead) flag_error(p, 1);
#pragma unroll 1
  for (int s = 1; s < C::kSlots; s += 2)  // every copy has landed
    if (it > s + 1)
      mbar_drain(bar(C::kKVFull + s), ((it - 2 - s) / C::kSlots) & 1, kDrainLimitNs);
}
template <int D, int KEYS>
__device__ __forceinline__ void cleaner(const CrossParams& p, const Work& w, int rank, uint32_t sKV0,
                                        uint8_t* kv, uint32_t bar0, volatile int* abort) {
  using C = Cfg<D>;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const int lane = threadIdx.x & 31;
  int it = 1;  // V follows K in the ring
#pragma unroll 1
  for (int i = w.first, turn = 0; i < w.items; i += w.step[turn], turn ^= 1) {
    const Item t = get_item<KEYS>(p, w, i, rank);
#pragma unroll 1
    for (int j = t.j0; j < t.j1; ++j, it += 2) {
      const KeyBits b = all_keys(own_keys(p, false, t, j));
      const int s = it % C::kSlots;
      if (!all_wait(bar(C::kKVFull + s), (it / C::kSlots) & 1, abort)) {
        if (lane == 0) flag_error(p, 1);
        return;
      }
      if (!b.all()) {
        clear_rows<D>(kv + s * C::kTileBytes, b);
        fence_proxy_async();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kVClean + s));
    }
  }
}

// ---------------------------------------------------------------------------------------
// MMA issuer of query tile X
// ---------------------------------------------------------------------------------------
template <int D, bool F16>
__device__ __forceinline__ void mma_qk(uint32_t tS, uint64_t dQ, uint64_t dK) {
  constexpr uint32_t idesc = idesc_f16(F16, kBM, kBN, 0);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const uint64_t off = ((k >> 2) * (kBM * 128) + (k & 3) * 32) >> 4;
    tc_mma_ss(tS, dQ + off, dK + off, idesc, k > 0);
  }
}
// O (+)= P V over keys [64 part, 64 part + 64) of the tile.
template <int D, bool F16>
__device__ __forceinline__ void mma_pv(uint32_t tO, uint32_t tP, uint64_t dV, int part, uint32_t acc) {
  constexpr uint32_t idesc = idesc_f16(F16, kBM, D, 1);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    tc_mma_ts(tO, tP + part * 32 + k * 8, dV + part * 512 + ((k * 2048) >> 4), idesc, acc | k | part);
}

template <int D, bool F16, int KEYS, bool GATHER>
__device__ __forceinline__ bool mma_issuer(const CrossParams& p, const Work& w, int rank, int X,
                                           uint32_t tmem, uint32_t sQ0, uint32_t sKV0,
                                           uint32_t bar0, volatile int* abort) {
  using C = Cfg<D>;
  const bool lead = elect_one();
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const uint32_t tS = tmem + X * 128, tO = tmem + 256 + X * 128;
  const uint64_t dQ = smem_desc_sw128(sQ0 + X * C::kTileBytes, 16, 1024);
  int q_cnt = 0, it = 0;    // it: ring index of the item's first tile of keys
  const bool tail = GATHER && w.seen % kBN != 0;
  uint32_t cleared = 0;     // bit s: parity of the clearings of slot s (gathered values)
  bool my_turn = X == 0;    // the first turn is tile A's
  bool ok = true;
#pragma unroll 1
  for (int i = w.first, turn = 0; ok && i < w.items; i += w.step[turn], turn ^= 1) {
    const Item t = get_item<KEYS>(p, w, i, rank);
    const int nt = t.j1 - t.j0;
    if (nt <= 0) continue;
    const bool both = 2 * t.pair + 1 < w.tiles, mine = X == 0 || both;
    if (mine) {
      ok = all_wait(bar(C::kQFull + X), q_cnt & 1, abort);
      ++q_cnt;
    }
    // step j: P V of tile j, Q K^T of tile j + 1
#pragma unroll 1
    for (int j = -1; ok && j < nt; ++j) {
      const bool first = j < 0, more = j + 1 < nt;
      const int iV = it + 2 * j + 1, iK = iV + 1;
      const int sV = iV % C::kSlots, sK = iK % C::kSlots;
      // (V cleaned, where a launch has keys that may not be seen)
      if (!first) {
        if (GATHER && tail && !more) {
          ok = all_wait(bar(C::kVClean + sV), (cleared >> sV) & 1, abort);
          cleared ^= 1u << sV;
        } else {
          ok = all_wait(bar((KEYS != kAllKeys && !GATHER ? C::kVClean : C::kKVFull) + sV),
                        (iV / C::kSlots) & 1, abort);
        }
      }
      if (ok && more) ok = all_wait(bar(C::kKVFull + sK), (iK / C::kSlots) & 1, abort);
      ok = __all_sync(0xffffffffu, ok && *abort == 0);
      if (!ok) break;
      if (!mine) {  // no such query tile: only give the slots back
        if (lead) {
          if (!first) mbar_arrive(bar(C::kKVEmpty + sV));
          if (more) mbar_arrive(bar(C::kKVEmpty + sK));
        }
        __syncwarp();
        continue;
      }
      if (both) {
        if (!my_turn) named_sync(turn_barrier(X), 64);
        my_turn = false;
      }
      if (!first) {
        const uint64_t dV = smem_desc_sw128(sKV0 + sV * C::kTileBytes, kBN * 128, 1024);
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
          named_sync(p_barrier(X, part), kPThreads);
          tc_fence_after();
          if (lead) mma_pv<D, F16>(tO, tS, dV, part, j > 0);
          __syncwarp();
        }
      } else {
        tc_fence_after();
      }
      if (lead) {
        if (more) {
          mma_qk<D, F16>(tS, dQ, smem_desc_sw128(sKV0 + sK * C::kTileBytes, 16, 1024));
          tc_commit(bar(C::kSFull + X));
          // the item's last Q K^T: the next item's queries may come
          if (j + 2 == nt) tc_commit(bar(C::kQEmpty + X));
          tc_commit(bar(C::kKVEmpty + sK));
        } else {
          tc_commit(bar(C::kODone + X));
        }
        if (!first) tc_commit(bar(C::kKVEmpty + sV));
      }
      __syncwarp();
      if (both) named_arrive(turn_barrier(X ^ 1), 64);
    }
    it += 2 * nt;
  }
  // a wait that gave up has raised the flag
  if (__all_sync(0xffffffffu, *abort == 0)) return true;
  if (lead) flag_error(p, 2);
  return false;
}

// ---------------------------------------------------------------------------------------
// Softmax and results (128 threads, thread = row of query tile X)
// ---------------------------------------------------------------------------------------
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return F16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
}
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float* o, float scale) {
  return make_uint4(pack2<F16>(o[0] * scale, o[1] * scale), pack2<F16>(o[2] * scale, o[3] * scale),
                    pack2<F16>(o[4] * scale, o[5] * scale), pack2<F16>(o[6] * scale, o[7] * scale));
}

// The running maximum (in units of log2, scaled) and sum of a row over a CTA's K/V tiles of an
// item, with P left in tensor memory for the MMA warp.  False: a wait gave up.
template <int D, bool F16, int KEYS>
__device__ __forceinline__ bool softmax_item(const CrossParams& p, const Work& w, const Item& t,
                                             int X, bool has_row, uint32_t tS, uint32_t tO,
                                             uint32_t bar_s, int& s_cnt, float& m_out,
                                             float& l_out, volatile int* abort) {
  const float sl2 = p.scale_log2;
  const bool gather = gathers<KEYS>(w);
  float m = -INFINITY, l = 0.f;
  uint32_t own = KEYS != kAllKeys ? own_keys(p, gather, t, t.j0) : 0;
#pragma unroll 1
  for (int j = t.j0; j < t.j1; ++j) {
    KeyBits bits{};
    if (KEYS != kAllKeys) {
      bits = all_keys(own);
      if (j + 1 < t.j1) own = own_keys(p, gather, t, j + 1);
    }
    if (!all_wait(bar_s, s_cnt & 1, abort)) return false;
    ++s_cnt;
    tc_fence_after();
    uint32_t s[kBN];
#pragma unroll
    for (int c = 0; c < kBN / 32; ++c)
      tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
    tmem_wait_ld();
    float* sf = reinterpret_cast<float*>(s);
    if (KEYS != kAllKeys) {
      if (!bits.all()) {
#pragma unroll
        for (int c = 0; c < kBN; ++c)
          if (!((bits.w[c >> 5] >> (c & 31)) & 1u)) sf[c] = -INFINITY;
      }
    } else if ((j + 1) * kBN > t.end) {
      const int valid = t.end - j * kBN;
#pragma unroll
      for (int c = 0; c < kBN; ++c)
        if (c >= valid) sf[c] = -INFINITY;
    }
    // row maximum over 8 independent chains
    float mx8[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) mx8[i] = fmaxf(sf[i], sf[i + 8]);
#pragma unroll
    for (int c = 16; c < kBN; c += 16)
#pragma unroll
      for (int i = 0; i < 8; ++i) mx8[i] = fmax3(mx8[i], sf[c + i], sf[c + 8 + i]);
    const float mx = fmaxf(fmaxf(fmaxf(mx8[0], mx8[1]), fmaxf(mx8[2], mx8[3])),
                           fmaxf(fmaxf(mx8[4], mx8[5]), fmaxf(mx8[6], mx8[7])));
    const float m_new = fmaxf(m, mx * sl2);
    // (what is in the tile past its rows has no say: tokens of other frames, or an earlier tile's)
    const bool rescale = __any_sync(0xffffffffu, has_row && m_new > m + kRescaleLog2);
    float fac = 1.f;
    if (rescale) {
      // a row that has seen no key yet has m = m_new = -inf: factor 1, not 2^(-inf + inf)
      fac = m == m_new ? 1.f : ex2_approx(m - m_new);
      l *= fac;
      m = m_new;
    }
    // O was last written by the previous tile's P V, which completed before S(j) was signalled; at
    // the first tile it holds nothing yet
    if (rescale && j > t.j0) {
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld32(tO + c * 32, o);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fac);
        tmem_st32(tO + c * 32, o);
      }
    }
    // p = 2^(s scale log2 e - m); while every key was masked m is -inf: p = 2^(-inf - 0) = 0.
    // P is rounded to the inputs' 16 bits for the product (at most 2^-8 of each probability in
    // bf16, averaged over the keys); the sum l is of the unrounded ones, in fp32.
    const float nm = m == -INFINITY ? 0.f : -m;
    const uint64_t sl2x2 = f2_pack(sl2, sl2), nmx2 = f2_pack(nm, nm);
    uint64_t l4[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t pk[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x0, x1;
        f2_unpack(ffma2(f2_pack(sf[q * 32 + 2 * e], sf[q * 32 + 2 * e + 1]), sl2x2, nmx2), x0, x1);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
        l4[e & 3] = fadd2(l4[e & 3], f2_pack(p0, p1));
        pk[e] = pack2<F16>(p0, p1);
      }
      tmem_st16(tS + q * 16, pk);
      if (q & 1) {
        tmem_wait_st();
        tc_fence_before();
        named_arrive(p_barrier(X, q >> 1), kPThreads);
      }
    }
    float a, b;
    f2_unpack(fadd2(fadd2(l4[0], l4[1]), fadd2(l4[2], l4[3])), a, b);
    l += a + b;
  }
  m_out = m;
  l_out = l;
  return true;
}

template <int D, bool F16, int KEYS>
__device__ __forceinline__ bool softmax_group(const CUtensorMap* tmO, const CrossParams& p,
                                              const Work& w, int rank, int X,
                                              uint32_t tmem, uint8_t* smem, uint32_t bar0,
                                              volatile int* abort) {
  using C = Cfg<D>;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = (warp & 3) * 32 + lane;  // and lane of tensor memory
  const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
  const uint32_t tS = tmem + lane_base + X * 128, tO = tmem + lane_base + 256 + X * 128;
  uint4* stage = reinterpret_cast<uint4*>(smem + C::kOffStage + (warp - 4) * kTurnBytes);
  int64_t at = -1;  // byte offset of this thread's row in O
  int s_cnt = 0, o_cnt = 0;
  Item next;
  bool next_row = false;
  auto find = [&](int i) {  // the next item
    if (i >= w.items) return;
    next = get_item<KEYS>(p, w, i, rank);
    next_row = is_row(p, w, next, 2 * next.pair + X, row);
  };
  find(w.first);
#pragma unroll 1
  for (int i = w.first, turn = 0; i < w.items;) {
    const Item t = next;
    const bool valid = next_row;
    i += w.step[turn];
    turn ^= 1;
    const int tile = 2 * t.pair + X;
    if (tile >= w.tiles) {
      find(i);
      continue;
    }
    float m = -INFINITY, l = 0.f;
    bool ok = t.j0 >= t.j1 ||
              softmax_item<D, F16, KEYS>(p, w, t, X, valid, tS, tO, bar(C::kSFull + X), s_cnt, m, l, abort);
    // found while the last P V runs: behind it every cycle counts
    find(i);
    const int first = whole_tile(p, w, t, tile);
    // no key: zeros, not 0 * accumulator, which may hold anything
    const bool none = l == 0.f;
    const float inv_l = none ? 0.f : 1.0f / l;
    if (t.j0 < t.j1) {
      ok = ok && all_wait(bar(C::kODone + X), o_cnt & 1, abort);
      ++o_cnt;
      tc_fence_after();
    }
    if (!ok) {
      if (lane == 0) flag_error(p, 3);
      return false;
    }
    if (p.cluster > 1) {
      // the ring holds the other tile's keys until that one is done too
      const bool other = t.j0 < t.j1 && 2 * t.pair + 1 < w.tiles;
      if (other && !all_wait(bar(C::kODone + (X ^ 1)), 0, abort)) {
        if (lane == 0) flag_error(p, 4);
        return false;
      }
      float4* part = reinterpret_cast<float4*>(smem + C::kOffKV) + X * (D / 4 * 128) + row;
      if (t.j0 < t.j1)
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(tO + c * 32, o);
          tmem_wait_ld();
#pragma unroll
          for (int q = 0; q < 8; ++q)
            part[(c * 8 + q) * 128] =
                make_float4(__uint_as_float(o[4 * q]), __uint_as_float(o[4 * q + 1]),
                            __uint_as_float(o[4 * q + 2]), __uint_as_float(o[4 * q + 3]));
        }
      reinterpret_cast<float2*>(smem)[X * 128 + row] = make_float2(m, l);
      return true;  // one item per CTA; joined after the cluster's barrier
    }
    if (first < 0 || p.lse) {
      int head;
      const int64_t token = row_of(p, w, t, tile, row, head);
      at = token < 0 ? -1 : (token * p.o_row_stride + static_cast<int64_t>(head) * D) * 2;
      if (token >= 0 && p.lse)
        p.lse[static_cast<int64_t>(head) * p.rows.T + token] =
            none ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
    }
#pragma unroll 1
    for (int c = 0; c < D / 64; ++c) {
      uint32_t o[64];
      tmem_ld32(tO + c * 64, reinterpret_cast<uint32_t(&)[32]>(o[0]));
      tmem_ld32(tO + c * 64 + 32, reinterpret_cast<uint32_t(&)[32]>(o[32]));
      tmem_wait_ld();
      if (lane == 0) bulk_wait_read();  // the stage's last tile has been read
      __syncwarp();
#pragma unroll
      for (int q = 0; q < 8; ++q)
        stage_at(stage, lane, q) = none ? make_uint4(0u, 0u, 0u, 0u)
                                        : pack8<F16>(reinterpret_cast<const float*>(o) + q * 8, inv_l);
      if (first >= 0) {
        // 32 consecutive tokens: in the background
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          tma_store_3d(tmO, smem_u32(stage), c * 64, t.unit, first + (warp & 3) * 32);
          bulk_commit();
        }
      } else {
        store_rows(stage, reinterpret_cast<char*>(p.O) + c * 128, row_span(at, p.o_row_stride * 2),
                   p.o_row_stride * 2);
      }
    }
    // (the accumulator is read before the next item's first P, so before its first P V)
  }
  if (lane == 0) bulk_wait_all();
  __syncwarp();
  return true;
}

// A split item's rows from all CTAs of the cluster: O = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M)
// l_c.  Each CTA takes its share of the columns of every row.
template <int D, bool F16, int KEYS>
__device__ __forceinline__ void join(const CrossParams& p, const Work& w, int rank, int X,
                                     uint32_t sbase) {
  using C = Cfg<D>;
  const int i = w.first;
  if (i >= w.items) return;
  const Item t = get_item<KEYS>(p, w, i, rank);
  const int tile = 2 * t.pair + X;
  if (tile >= w.tiles) return;
  const int row = threadIdx.x & 127;
  int head;
  const int64_t token = row_of(p, w, t, tile, row, head);
  if (token < 0) return;
  float ms[8], M = -INFINITY, Lsum = 0.f;
  float ls[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    ms[c] = -INFINITY;
    ls[c] = 0.f;
    if (c < p.cluster) {
      const uint32_t at = map_to_rank(sbase + (X * 128 + row) * 8, c);
      ms[c] = ld_cluster_f(at);
      ls[c] = ld_cluster_f(at + 4);
    }
    M = fmaxf(M, ms[c]);
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    ms[c] = ls[c] == 0.f ? 0.f : ex2_approx(ms[c] - M);  // now the weight; no key seen: 0
    Lsum += ms[c] * ls[c];
  }
  const bool none = Lsum == 0.f;
  const float inv = none ? 0.f : 1.0f / Lsum;
  uint16_t* orow = p.O + token * p.o_row_stride + static_cast<int64_t>(head) * D;
  // columns in groups of 8: cluster <= 8 = D / 8 at D = 64
#pragma unroll 1
  for (int c8 = rank; c8 < D / 8; c8 += p.cluster) {
    float acc[8] = {};
    const uint32_t at = sbase + C::kOffKV + (X * (D / 4 * 128) + c8 * 2 * 128 + row) * 16;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c < p.cluster && ms[c] != 0.f) {
        const uint32_t r = map_to_rank(at, c);
        const float4 a = ld_cluster_f4(r), b = ld_cluster_f4(r + 128 * 16);
        acc[0] = fmaf(ms[c], a.x, acc[0]);
        acc[1] = fmaf(ms[c], a.y, acc[1]);
        acc[2] = fmaf(ms[c], a.z, acc[2]);
        acc[3] = fmaf(ms[c], a.w, acc[3]);
        acc[4] = fmaf(ms[c], b.x, acc[4]);
        acc[5] = fmaf(ms[c], b.y, acc[5]);
        acc[6] = fmaf(ms[c], b.z, acc[6]);
        acc[7] = fmaf(ms[c], b.w, acc[7]);
      }
    *reinterpret_cast<uint4*>(orow + c8 * 8) = pack8<F16>(acc, inv);
  }
  if (rank == 0 && p.lse)
    p.lse[static_cast<int64_t>(head) * p.rows.T + token] =
        none ? -INFINITY : (M + __log2f(Lsum)) * 0.69314718055994531f;
}

// A warp that gave up releases the MMA warp that waits for it, until that warp has left (2 s at
// most: it reads the abort flag, which is up, in every round).
__device__ __forceinline__ void release_mma(const volatile int* done, int bar_a, int bar_b,
                                            int threads) {
  for (int n = 0; n < 2000000 && !__all_sync(0xffffffffu, *done != 0); ++n) {
    named_arrive(bar_a, threads);
    if (bar_b != bar_a) named_arrive(bar_b, threads);
    __nanosleep(1000);
  }
}

template <int D, bool F16, int KEYS>
__global__ void __launch_bounds__(kThreads, 1)
    cross_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmMany,
                 const __grid_constant__ CUtensorMap tmUnit, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                 const __grid_constant__ CUtensorMap tmRowsK,
                 const __grid_constant__ CUtensorMap tmRowsV, const CrossParams p) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  if (sbase & 1023u) {  // (swizzled tiles; no room to align it here)
    if (threadIdx.x == 0) flag_error(p, 5);
    return;
  }
  const uint32_t sQ0 = sbase, sKV0 = sbase + C::kOffKV, bar0 = sbase + C::kOffBar;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  volatile int* mma_done = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 8);  // [2]
  const int warp = threadIdx.x >> 5;
  const int rank = p.cluster > 1 ? static_cast<int>(cluster_rank()) : 0;

  Work& work = *reinterpret_cast<Work*>(smem + C::kOffWork);
  if (threadIdx.x == 64) {
    cudaGridDependencySynchronize();
    make_work(p, work);
  }
  if (threadIdx.x == 0) {
    for (int X = 0; X < 2; ++X) {
      mbar_init(bar0 + 8 * (C::kQFull + X), 1);
      mbar_init(bar0 + 8 * (C::kQEmpty + X), 1);
      mbar_init(bar0 + 8 * (C::kSFull + X), 1);
      mbar_init(bar0 + 8 * (C::kODone + X), 1);
      mbar_init(bar0 + 8 * (C::kDrain + X), 1);
      mma_done[X] = 0;
    }
    for (int s = 0; s < C::kSlots; ++s) {
      mbar_init(bar0 + 8 * (C::kKVFull + s), 1);
      mbar_init(bar0 + 8 * (C::kKVEmpty + s), 2);
      mbar_init(bar0 + 8 * (C::kVClean + s), 1);
    }
    *abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Work& w = work;
  cudaGridDependencySynchronize();  // what was launched before is done (launch_early)
  if (KEYS != kAllKeys && p.key_mask) trim_states<KEYS>(p, work, rank);
  if (KEYS == kSomeKeys && w.sorted) sort_frames(p, work, reinterpret_cast<int*>(smem + C::kOffStage));

  // Every warp of warpgroup 0 gives registers back before any softmax warp asks for more, so the
  // increase below always finds them.
  if (warp < 4) {
    reg_dealloc<kRegsControl>();
    if (warp == 0) {
      auto produce = [&](auto gather) {
        producer<D, KEYS, gather.value>(
            {&tmQ, &tmMany, &tmUnit}, &tmK, &tmV, &tmRowsK, p, w, rank,
            reinterpret_cast<BoxList<kBM>*>(smem + C::kOffList),
            reinterpret_cast<int*>(smem + C::kOffKeys), sQ0, sKV0, bar0, abort);
      };
      if (gathers<KEYS>(w)) produce(std::bool_constant<KEYS == kSameKeys>{});
      else produce(std::false_type{});
    } else if (warp < 3) {
      const int X = warp - 1;
      auto issue = [&](auto gather) {
        return mma_issuer<D, F16, KEYS, gather.value>(p, w, rank, X, tmem, sQ0, sKV0, bar0, abort);
      };
      const bool ok = gathers<KEYS>(w) ? issue(std::bool_constant<KEYS == kSameKeys>{})
                                       : issue(std::false_type{});
      __syncwarp();
      mma_done[X] = 1;  // waits on no named barrier any more
      if (!ok) release_mma(mma_done + (X ^ 1), turn_barrier(X ^ 1), turn_barrier(X ^ 1), 64);
      // all MMAs issued so far complete before tensor memory is released
      if (elect_one()) tc_commit(bar0 + 8 * (C::kDrain + X));
      __syncwarp();
      mbar_drain(bar0 + 8 * (C::kDrain + X), 0, kDrainLimitNs);
    } else if (gathers<KEYS>(w)) {
      gather_values<D, KEYS>(&tmRowsV, p, w, rank, reinterpret_cast<int*>(smem + C::kOffKeys) + kBN, sKV0,
                       smem + C::kOffKV, bar0, abort);
    } else if (KEYS != kAllKeys) {
      cleaner<D, KEYS>(p, w, rank, sKV0, smem + C::kOffKV, bar0, abort);
    }
  } else {
    reg_alloc<kRegsSoftmax>();
    const int X = (warp - 4) >> 2;
    if (!softmax_group<D, F16, KEYS>(&tmO, p, w, rank, X, tmem, smem, bar0, abort))
      release_mma(mma_done + X, p_barrier(X, 0), p_barrier(X, 1), kPThreads);
  }
  __syncwarp();
  if (p.cluster > 1) {
    cluster_arrive();
    cluster_wait();
    if (warp >= 4) join<D, F16, KEYS>(p, w, rank, (warp - 4) >> 2, sbase);
    __syncwarp();
    cluster_arrive();  // every CTA has read the others' rows
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------
struct Maps {
  CUtensorMap q, many, unit, k, v, o, rows_k, rows_v;
};

// [rows][heads][d] elements of 16 bits, boxes of 64 x box_heads x box_rows.
rf_status map_heads(CUtensorMap* m, int dtype, const void* base, int d, int heads, int64_t rows,
                    int64_t row_stride, int box_heads, int box_rows) {
  const uint64_t dims[3] = {static_cast<uint64_t>(d), static_cast<uint64_t>(heads),
                            static_cast<uint64_t>(rows)};
  const uint64_t strides[2] = {static_cast<uint64_t>(d) * 2, static_cast<uint64_t>(row_stride) * 2};
  const uint32_t box[3] = {64, static_cast<uint32_t>(box_heads), static_cast<uint32_t>(box_rows)};
  return make_tensor_map(m, dtype, base, 3, dims, strides, box);
}

// [rows][cols] elements of 16 bits, boxes of 64 x 1.
rf_status map_rows(CUtensorMap* m, int dtype, const void* base, int cols, int64_t rows,
                   int64_t row_stride) {
  const uint64_t dims[2] = {static_cast<uint64_t>(cols), static_cast<uint64_t>(rows)};
  const uint64_t strides[1] = {static_cast<uint64_t>(row_stride) * 2};
  const uint32_t box[2] = {64, 1};
  return make_tensor_map(m, dtype, base, 2, dims, strides, box);
}

template <int D, bool F16, int KEYS>
rf_status launch(const Maps& m, const CrossParams& p, int grid, const DeviceInfo& di,
                 cudaStream_t s) {
  constexpr int smem = Cfg<D>::kSmem;
  static std::atomic<bool> done[64] = {};
  if (smem > di.max_smem_optin) return fail(RF_ERR_UNSUPPORTED, "rf_cross_attn: shared memory");
  if (!done[di.device]) {
    if (cudaError_t e = cudaFuncSetAttribute(cross_kernel<D, F16, KEYS>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, smem))
      return fail(RF_ERR_CUDA, "cudaFuncSetAttribute(rf_cross_attn)", e);
    done[di.device] = true;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  return launch_early(cfg, p.cluster, "rf_cross_attn launch", cross_kernel<D, F16, KEYS>, m.q, m.many,
                      m.unit, m.k, m.v, m.o, m.rows_k, m.rows_v, p);
}

template <int D, bool F16>
rf_status launch_type(int keys, const Maps& m, const CrossParams& p, int grid,
                      const DeviceInfo& di, cudaStream_t s) {
  switch (keys) {
    case kAllKeys: return launch<D, F16, kAllKeys>(m, p, grid, di, s);
    case kSomeKeys: return launch<D, F16, kSomeKeys>(m, p, grid, di, s);
    default: return launch<D, F16, kSameKeys>(m, p, grid, di, s);
  }
}
template <int D>
rf_status launch_dim(bool f16, int keys, const Maps& m, const CrossParams& p, int grid,
                     const DeviceInfo& di, cudaStream_t s) {
  return f16 ? launch_type<D, true>(keys, m, p, grid, di, s)
             : launch_type<D, false>(keys, m, p, grid, di, s);
}

// CTAs per item: the number whose busiest SM has the least to do, in K/V tiles.  A further round of
// items costs about kRound tiles (start, queries, results), a join kJoin more.
int cluster_size(int64_t items, int64_t kv_tiles, int sms) {
  constexpr int64_t kRound = 2, kJoin = 2;
  int best = 1;
  int64_t least = 0;
  for (int c = 1; c <= 8; c *= 2) {
    if (c > 1 && c > kv_tiles) break;
    const int64_t rounds = (items * c + sms - 1) / sms;
    const int64_t cost = rounds * ((kv_tiles + c - 1) / c + kRound + (c > 1 ? kJoin : 0));
    if (c == 1 || cost < least) {
      best = c;
      least = cost;
    }
  }
  return best;
}

}  // namespace
}  // namespace rf

using namespace rf;

extern "C" rf_status rf_cross_attn(void* d_O, float* d_lse, const void* d_Q, const void* d_K,
                                   const void* d_V, int64_t o_row_stride, int64_t q_row_stride,
                                   int64_t k_row_stride, int64_t v_row_stride, int dtype, int F,
                                   int N, int H, int Hkv, int d, int L, const int32_t* d_kv_range,
                                   const uint8_t* d_key_mask, const int32_t* d_active,
                                   const int32_t* d_counts, float softmax_scale, int32_t* d_status,
                                   rf_stream_t stream) {
  if (!d_O || !d_Q) return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: null pointer");
  if (L < 0 || (L > 0 && (!d_K || !d_V)))
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: keys and values");
  if (dtype != RF_BF16 && dtype != RF_FP16) return fail(RF_ERR_UNSUPPORTED, "rf_cross_attn: dtype");
  if (F < 1 || N < 1 || H < 1 || Hkv < 1 || H > 65535 || H % Hkv)
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: sizes >= 1, Hkv divides H");
  if (d != 64 && d != 128) return fail(RF_ERR_UNSUPPORTED, "rf_cross_attn: head dim 64 or 128");
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: softmax scale");
  if ((d_active == nullptr) != (d_counts == nullptr))
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: active list and counts come together");
  const int64_t q_row = static_cast<int64_t>(H) * d, kv_row = static_cast<int64_t>(Hkv) * d;
  if (q_row_stride < q_row || o_row_stride < q_row || k_row_stride < kv_row || v_row_stride < kv_row)
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: row stride below the row's length");
  if (q_row_stride % 8 || o_row_stride % 8 || k_row_stride % 8 || v_row_stride % 8 ||
      !aligned16(d_Q) || !aligned16(d_O) || !aligned16(d_K) || !aligned16(d_V))
    return fail(RF_ERR_MISALIGNED, "rf_cross_attn: bases and row strides on 16-byte boundaries");
  if ((reinterpret_cast<uintptr_t>(d_kv_range) & 7) || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return fail(RF_ERR_MISALIGNED, "rf_cross_attn: ranges on 8-byte boundaries, lse on 4-byte ones");
  const int64_t T = static_cast<int64_t>(F) * N;
  const int g = H / Hkv;
  // packed rows: where they save reading K and V (several heads), or a frame has few tokens
  const bool packed = static_cast<int64_t>(N) * g <= kBM && (d_kv_range || g > 1 || N < 8);
  // without a list and without ranges the tokens are one frame; packed rows need the frames
  const bool one = !d_active && !d_kv_range && !packed;
  const int64_t Fr = one ? 1 : F, Nr = one ? T : N;
  const int unit = row_unit(Nr);
  const int64_t Np = (Nr + unit - 1) / unit * unit;
  if (T > 0x7FFFFFFF - 65536 || Fr * Np > 0x7FFFFFFF - 65536 || L > 0x7FFFFFFF - 65536)
    return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: too many tokens");
  DeviceInfo di;
  if (rf_status st = current_device_info(&di)) return st;
  if (di.cc_major != 10 || di.cc_minor != 3) return fail(RF_ERR_UNSUPPORTED, "needs sm_103");

  CrossParams p{};
  p.O = static_cast<uint16_t*>(d_O);
  p.lse = d_lse;
  p.kv_range = reinterpret_cast<const int2*>(d_kv_range);
  p.key_mask = d_key_mask;
  p.status = d_status;
  p.rows = {d_active, d_counts, static_cast<int>(Fr), static_cast<int>(Nr), static_cast<int>(Np), unit,
            static_cast<int>(T), FastDiv(static_cast<uint32_t>(Np))};
  p.o_row_stride = o_row_stride;
  p.L = L;
  p.g = g;
  p.packed = packed;
  p.units = packed ? Hkv : H;
  p.tile_rows = d_kv_range ? kBM : tile_rows(unit, kBM);
  p.frame_rows = packed ? N * g : 0;
  p.tile_frames = packed ? (d_kv_range ? 1 : kBM / p.frame_rows) : 0;
  p.by_g = FastDiv(static_cast<uint32_t>(g));
  p.by_units = FastDiv(static_cast<uint32_t>(p.units));
  p.by_frame_rows = FastDiv(static_cast<uint32_t>(std::max(p.frame_rows, 1)));
  p.scale_log2 = static_cast<float>(static_cast<double>(softmax_scale) * 1.4426950408889634);

  // at most, with every frame active
  const int64_t groups = d_kv_range ? F : 1;
  const int64_t tiles = packed ? (d_kv_range ? 1 : (Fr + p.tile_frames - 1) / p.tile_frames)
                               : ((d_kv_range ? Nr : Fr * Np) + p.tile_rows - 1) / p.tile_rows;
  const int64_t items = p.units * groups * ((tiles + 1) / 2);
  if (items > 0x7FFFFFFF / 16) return fail(RF_ERR_INVALID_ARG, "rf_cross_attn: too many rows");
  // (the ranges are on the device: taken as shares of the states)
  const int64_t share = d_kv_range ? (static_cast<int64_t>(L) + F - 1) / F : L;
  const int64_t kv_tiles = (share + kBN - 1) / kBN;
  p.cluster = cluster_size(items, kv_tiles, di.sm_count);
  const int grid = p.cluster > 1 ? static_cast<int>(items) * p.cluster
                                 : static_cast<int>(std::min<int64_t>(items, di.sm_count));

  Maps m;
  // (no states: nothing is loaded, the maps only have to exist)
  const void* K = L > 0 ? d_K : d_Q;
  const void* V = L > 0 ? d_V : d_Q;
  const int64_t rows_kv = L > 0 ? L : 1;
  if (rf_status st = map_heads(&m.q, dtype, d_Q, d, H, T, q_row_stride, 1, kBM)) return st;
  m.many = m.unit = m.q;
  if (packed) {
    if (rf_status st = map_heads(&m.unit, dtype, d_Q, d, H, T, q_row_stride, g, N)) return st;
  } else if (Fr > 1 && !d_kv_range) {  // a tile can lie across frames
    if (rf_status st = map_heads(&m.many, dtype, d_Q, d, H, T, q_row_stride, 1, kBoxRows)) return st;
    if (rf_status st = map_heads(&m.unit, dtype, d_Q, d, H, T, q_row_stride, 1, unit)) return st;
  }
  if (rf_status st = map_heads(&m.k, dtype, K, d, Hkv, rows_kv, k_row_stride, 1, kBN)) return st;
  if (rf_status st = map_heads(&m.v, dtype, V, d, Hkv, rows_kv, v_row_stride, 1, kBN)) return st;
  m.rows_k = m.k;
  m.rows_v = m.v;
  if (d_key_mask && !d_kv_range && L > 0) {  // single rows, where the mask leaves few
    if (rf_status st = map_rows(&m.rows_k, dtype, d_K, Hkv * d, L, k_row_stride)) return st;
    if (rf_status st = map_rows(&m.rows_v, dtype, d_V, Hkv * d, L, v_row_stride)) return st;
  }
  if (rf_status st = map_heads(&m.o, dtype, d_O, d, H, T, o_row_stride, 1, 32)) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int keys = d_kv_range ? kSomeKeys : d_key_mask ? kSameKeys : kAllKeys;
  return d == 128 ? launch_dim<128>(dtype == RF_FP16, keys, m, p, grid, di, s)
                  : launch_dim<64>(dtype == RF_FP16, keys, m, p, grid, di, s);
}
