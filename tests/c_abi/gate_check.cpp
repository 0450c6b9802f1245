// The row of a per-frame gate that each CTA of rf_linear_i8's pairs reads for its half of a tile: of a frame that
// there is, and the right one where rows of the half are stored.  The launch's and the kernel's arithmetic of
// rows is repeated here over the library's own rows_frame.  Exits 0 if all hold.
#include <algorithm>
#include <cstdio>

#include "rf_deal.h"

struct By {
  int d;
  int div(int x) const { return x / d; }
};

// F frames of N tokens, A of them active (0: no list)
static int halves(int F, int N, int A) {
  const long long T = static_cast<long long>(F) * N;
  const int Fr = A ? F : 1, Nr = A ? N : static_cast<int>(T), unit = Nr < 8 ? Nr : 8;
  const int Np = (Nr + unit - 1) / unit * unit, R = (A ? A : Fr) * Np, half = 128 / unit * unit;
  const int frames = A ? A : F;  // that a gate's row may be of
  const int tiles = (R + 2 * half - 1) / (2 * half);
  for (int m = 0; m < tiles; ++m)
    for (int rank = 0; rank < 2; ++rank) {
      const int r0 = (2 * m + rank) * half;
      const rf::RowsFrame f = A ? rf::rows_frame(r0, half, R, By{Np}) : rf::rows_frame(r0, half, static_cast<int>(T), By{N});
      int lo = frames, hi = -1;  // the frames of the half's tokens
      for (int r = r0; r < std::min(r0 + half, R); ++r) {
        const int a = A ? r / Np : r / N;
        if (A ? r % Np >= N : r >= T) continue;
        lo = std::min(lo, a);
        hi = std::max(hi, a);
      }
      if (f.a < 0 || f.a >= frames || (f.one && hi >= 0 && (lo != f.a || hi != f.a)) || (hi >= 0 && lo == hi && !f.one))
        return std::printf("%d x %d, %d active: half from row %d reads frame %d (%d), its tokens are of %d to %d\n", F, N,
                           A, r0, f.a, f.one, lo, hi);
    }
  return 0;
}

int main() {
  int bad = 0;
  for (int F : {1, 2, 3, 7, 33})
    for (int N = 1; N <= 1400; N += N < 300 ? 1 : 37) {
      bad += halves(F, N, 0) != 0;
      for (int A : {1, F / 2, F})
        if (A > 0) bad += halves(F, N, A) != 0;
    }
  bad += halves(3, 1111, 0) != 0;
  return bad != 0;
}
