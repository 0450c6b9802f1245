// rf_deal.h -- a tile's boxes of rows dealt to the warps that load them.
#pragma once
#include "rf_div.h"

namespace rf {

// Warps that load a tile of `boxes` boxes, of `most` there are: never more than boxes.  A stage of the
// ring is full only when all of its boxes have landed, so a warp with a box in every stage cannot fall
// behind by a turn of the ring; one without would wait on a barrier's parity that nothing keeps from
// passing it twice.  Up to two boxes one warp is enough.
RF_HOST_DEVICE constexpr int loading_warps(int boxes, int most) {
  return boxes <= 2 ? 1 : boxes < most ? boxes : most;
}

// The boxes of warp `who` of `of`: numbers below an end, first who, then every of-th.  The larger
// boxes and the others are one sequence, so that `of` boxes or more leave no warp without one.
struct Deal {
  int next, of;
  RF_HOST_DEVICE bool more(int end) const { return next < end; }
  RF_HOST_DEVICE int take() {
    const int i = next;
    next += of;
    return i;
  }
};

}  // namespace rf
