// rf_rows.cuh -- the rows of a launch over the active frames, and how a tile of them is loaded.
#pragma once
#include <cstdint>

#include "rf_div.h"
#include "rf_tc_ptx.cuh"

namespace rf {

// The active frames' tokens one frame after the other, each frame padded to Np rows; Np is N
// rounded up to `unit`, so that `unit` consecutive rows from a multiple of it lie in one frame.
struct RowMap {
  const int32_t* active;  // or null: frames 0 .. F-1
  const int32_t* counts;
  int F, N, Np, unit;
  int T;  // tokens: F * N
  FastDiv by_Np;

  __device__ __forceinline__ int frames() const {
    return active ? min(max(counts[0], 0), F) : F;
  }
  __device__ __forceinline__ int frame(int a) const { return active ? active[a] : a; }
};
// Frames of 8 tokens or more are padded to 8 rows, a swizzle atom of shared memory; shorter ones
// not at all, and are loaded whole (the swizzle goes by address, so a box may begin at any row):
// their tiles have whole frames, tile_rows of the rows that a tile could have.
constexpr int row_unit(int64_t N) { return N < 8 ? static_cast<int>(N) : 8; }
constexpr int tile_rows(int unit, int most) { return most / unit * unit; }

// How a tile of rows is loaded: in one TMA box where its rows lie in one frame, else in boxes of
// kBoxRows and of `unit` rows, listed in shared memory {first token, first row of the tile}: the
// larger ones from the front of the list, the others from its end.  One elected thread of a warp issues
// that warp's share of them, each from a fixed tensor map: a box issued by its own lane under a branch,
// or with the map chosen per box, held a product's 512-cycle step up to three times its length.
constexpr int kBoxRows = 32;
template <int CAP>  // boxes at most; a tile has at most 256 rows
struct BoxList {
  int tok[CAP];
  uint8_t row[CAP];
};
struct RowBoxes {
  int rows;           // rows that the boxes bring
  int n_many, n_unit; // both 0: one box of the whole tile, from token tok
  int tok;
};
// Rows [r0, r0 + n) of R, r0 and n multiples of the unit, a whole tile's box of `box` >= n rows;
// with room for n / unit boxes.  Warp-collective; the same in every lane.  Rows past R are not
// loaded, except that a tile with none at all gets a box of zeros.
template <int CAP>
__device__ __forceinline__ RowBoxes list_boxes(const RowMap& m, int R, int r0, int n, int box,
                                               BoxList<CAP>& list) {
  RowBoxes x{box, 0, 0, 0};
  const int lane = threadIdx.x & 31;
  const int end = min(r0 + n, R);
  const int a0 = m.by_Np.div(r0);
  if (r0 >= R || a0 == m.by_Np.div(end - 1)) {
    // rows past the frame bring the tokens that follow, past the last one zeros: never stored
    x.tok = r0 >= R ? m.T : m.frame(a0) * m.N + (r0 - a0 * m.Np);
    return x;
  }
  x.rows = end - r0;
  __syncwarp();  // the list's last use is over
  if (m.unit < 8) {  // frames of `unit` tokens
    x.n_unit = x.rows / m.unit;
#pragma unroll 1
    for (int i = lane; i < x.n_unit; i += 32) {
      list.tok[CAP - 1 - i] = m.frame(a0 + i) * m.N;
      list.row[CAP - 1 - i] = static_cast<uint8_t>(i * m.unit);
    }
  } else {
#pragma unroll 1
    for (int r = r0, a = a0; r < end; ++a) {
      const int q = r - a * m.Np, len = min(m.Np - q, end - r);
      const int many = len / kBoxRows, units = (len - many * kBoxRows) / 8;
      const int tok = m.frame(a) * m.N + q;
      if (lane < many) {
        const int o = lane * kBoxRows;
        list.tok[x.n_many + lane] = tok + o;
        list.row[x.n_many + lane] = static_cast<uint8_t>(r - r0 + o);
      }
      if (lane < units) {
        const int o = many * kBoxRows + lane * 8, i = CAP - 1 - (x.n_unit + lane);
        list.tok[i] = tok + o;
        list.row[i] = static_cast<uint8_t>(r - r0 + o);
      }
      x.n_many += many;
      x.n_unit += units;
      r += len;
    }
  }
  __syncwarp();
  return x;
}
// list_boxes(...).rows, without the list.
__device__ __forceinline__ int boxed_rows(const RowMap& m, int R, int r0, int n, int box) {
  const int end = min(r0 + n, R);
  return r0 >= R || m.by_Np.div(r0) == m.by_Np.div(end - 1) ? box : end - r0;
}

}  // namespace rf
