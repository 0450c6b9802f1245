// Every way to deal a tile's boxes (larger ones and others) to the warps of rf_linear's kernels:
// each box goes to one warp, and every warp that loads has one.  The kernels' loops are repeated here
// over the library's own Deal and loading_warps.  Exits 0 if all hold.
#include <cstdio>
#include <vector>

#include "rf_deal.h"

static int deal(int n_many, int n_unit, int of) {
  std::vector<int> many(n_many), unit(n_unit);
  for (int who = 0; who < of; ++who) {
    rf::Deal d{who, of};
    int own = 0;
    while (d.more(n_many)) ++many[d.take()], ++own;
    while (d.more(n_many + n_unit)) ++unit[d.take() - n_many], ++own;
    if (own == 0) return std::printf("%d + %d boxes: warp %d of %d has none\n", n_many, n_unit, who, of);
  }
  for (int i = 0; i < n_many; ++i)
    if (many[i] != 1) return std::printf("%d + %d boxes: larger box %d\n", n_many, n_unit, i);
  for (int i = 0; i < n_unit; ++i)
    if (unit[i] != 1) return std::printf("%d + %d boxes: box %d\n", n_many, n_unit, i);
  return 0;
}

int main() {
  int bad = 0;
  for (int n_many = 0; n_many <= 8; ++n_many)      // of 32 rows, of at most 256
    for (int n_unit = 0; n_unit <= 256; ++n_unit) {
      const int boxes = n_many + n_unit;
      if (boxes < 2) continue;                     // a tile across frames has two or more
      bad += deal(n_many, n_unit, rf::loading_warps(boxes, 7)) != 0;
      bad += deal(n_many, n_unit, 2) != 0;         // a pair's CTA: always two warps
    }
  for (int boxes = 0; boxes < 2; ++boxes) bad += rf::loading_warps(boxes, 7) != 1;
  return bad != 0;
}
