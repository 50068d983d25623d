// Prints the choices of csrc/mx4_choice.h for the sizes on stdin, a line each.
#include <cstdio>
#include <cstring>

#include "mx4_choice.h"

int main() {
  char what[32];
  long long a, b, c, d, e, f;
  while (std::scanf("%31s %lld %lld %lld %lld %lld %lld", what, &a, &b, &c, &d, &e, &f) == 7) {
    if (!std::strcmp(what, "form")) {   // m n: the form and the workgroups of a direct one along x and y
      const rslm::Mx4MatmulForm form = rslm::matmul_form(a, b);
      const int side = form == rslm::kMmDirect64 ? 64 : form == rslm::kMmDirect32 ? 32 : form == rslm::kMmDirect16 ? 16 : 0;
      const rslm::Mx4DirectGrid g = side ? rslm::matmul_direct_grid(a, b, side) : rslm::Mx4DirectGrid{0, 0};
      std::printf("%d %lld %lld\n", side ? side : form == rslm::kMmTile256 ? 256 : 128, (long long)g.x, (long long)g.y);
    } else if (!std::strcmp(what, "slab_row")) {   // own slab
      std::printf("%lld\n", (long long)rslm::slab_row(int(a), int(b)));
    } else if (!std::strcmp(what, "gemm")) {   // type m n dim, backward or not: rows of a tile (0: few rows) and parts
      const bool few = !e && rslm::score_few_ok(int(a), b, int(d));
      const long long cols = e ? d : c, len = e ? c : d;
      std::printf("%d %d\n", few ? 0 : rslm::tile_rows(int(a), b, cols, len, e), few ? 1 : rslm::sum_splits(int(a), b, cols, len, e));
    } else if (!std::strcmp(what, "parts")) {   // the same and rows of a tile: its parts
      std::printf("%d\n", rslm::splits_of(int(a), b, e ? d : c, e ? c : d, e, int(f)));
    } else {
      return 1;
    }
  }
  return 0;
}
