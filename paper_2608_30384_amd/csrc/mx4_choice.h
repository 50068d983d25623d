// Which arrangement of the kernels a product of MX4 rows takes, by its sizes.
// Plain C++, so that the choice can be looked at without a GPU.
#pragma once

#include <cstdint>

namespace rslm {

// ---- 4-bit by 4-bit (mx4_matmul.hip)

constexpr int kMmN = 256;               // rows of b of an LDS tile

// LDS tiles of 256 or 128 rows of a; straight from memory, a wavefront taking a
// square of 64, 32 or 16.
enum Mx4MatmulForm { kMmTile256, kMmTile128, kMmDirect64, kMmDirect32, kMmDirect16 };

// Workgroups of 256 threads of a direct form: four squares side by side.
struct Mx4DirectGrid {
  int64_t x, y;
};
constexpr Mx4DirectGrid matmul_direct_grid(int64_t m, int64_t n, int side) {
  return Mx4DirectGrid{(n + 4 * side - 1) / (4 * side), (m + side - 1) / side};
}
// A grid counts its threads along x in 32 bits.
constexpr int64_t kMostWorkgroups = 0xffffffffll / 256;

// LDS tiles where there are 64 of 128 x 256, and of 256 x 256 where those fill the
// GPU's 256 CUs and no quarter of their rows is past the end; else straight from
// memory, a wavefront taking 64 x 64 of out, or 32 x 32 or 16 x 16 where there
// would be less than four wavefronts to a CU.  us, m x n x dim to float32 (three
// as marked to bfloat16):
//                                tiles 256   128  direct 64    32     16
//     256 x   4,096 x   768           13.7   9.1       10.9   6.1    9.0
//     512 x   4,096 x   768           14.4   9.7       11.4  10.0   16.2
//   1,024 x   1,024 x 1,024           15.0  10.0       18.5   9.8   16.3
//     256 x   8,192 x 4,096           29.9  21.0       60.0  58.5  112.9
//   1,024 x   4,096 x   768           15.6  10.9       13.1  17.6   30.9
//   2,048 x   4,096 x   768           17.2  12.8       21.5  34.9   57.8
//   4,096 x   4,096 x   128           15.2  16.7       15.4  15.9   18.8
//     300 x 100,000 x 1,024 bfloat16  59.1  43.2
//     700 x 100,000 x   768 bfloat16  65.9  72.1
//   8,192 x  32,768 x 4,096 bfloat16   607   850
//      37 x 100,003 x    96           18.3  13.5        7.5   8.1    8.3
//      64 x   4,096 x 4,096           26.8  19.3       58.3  30.0   16.1
//       1 x 100,000 x 1,024                                  19.0   16.7
// Where the 16 x 16 form would be more workgroups than a grid counts (the last 63
// rows of b up to 2^30, and any more), 32 x 32.
inline Mx4MatmulForm matmul_form(int64_t m, int64_t n) {
  auto pieces = [&](int64_t rows, int64_t cols) { return ((m + rows - 1) / rows) * ((n + cols - 1) / cols); };
  if (m > 64 && n > 64 && pieces(128, kMmN) >= 64)
    return pieces(256, kMmN) >= 256 && 2 * pieces(128, kMmN) > 3 * pieces(256, kMmN) ? kMmTile256 : kMmTile128;
  if (m > 32 && pieces(64, 64) >= 1024) return kMmDirect64;
  if ((m > 16 || matmul_direct_grid(m, n, 16).x > kMostWorkgroups) && pieces(32, 32) >= 1024) return kMmDirect32;
  return kMmDirect16;
}

// ---- float by 4-bit (mx4_score.hip)

// The gradient's row of b, from the first of its part of the sum, whose code a thread
// takes in a slab of 32 rows, `own` its place among them; at and past the part's end
// too.  Unsigned: slabs ahead of the last group pass 2^31 where one part has all of
// 2^31 - 256 rows.
constexpr uint32_t slab_row(int own, int slab) { return uint32_t(own) + 32u * uint32_t(slab); }

}  // namespace rslm
