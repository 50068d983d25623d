// Prints the choices of csrc/mx4_choice.h for the sizes on stdin, a line each.
#include <cstdio>
#include <cstring>

#include "mx4_choice.h"

int main() {
  char what[32];
  long long a, b;
  while (std::scanf("%31s %lld %lld", what, &a, &b) == 3) {
    if (!std::strcmp(what, "form")) {   // m n: the form and the workgroups of a direct one along x and y
      const rslm::Mx4MatmulForm f = rslm::matmul_form(a, b);
      const int side = f == rslm::kMmDirect64 ? 64 : f == rslm::kMmDirect32 ? 32 : f == rslm::kMmDirect16 ? 16 : 0;
      const rslm::Mx4DirectGrid g = side ? rslm::matmul_direct_grid(a, b, side) : rslm::Mx4DirectGrid{0, 0};
      std::printf("%d %lld %lld\n", side ? side : f == rslm::kMmTile256 ? 256 : 128, (long long)g.x, (long long)g.y);
    } else if (!std::strcmp(what, "slab_row")) {   // own slab
      std::printf("%lld\n", (long long)rslm::slab_row(int(a), int(b)));
    } else {
      return 1;
    }
  }
  return 0;
}
