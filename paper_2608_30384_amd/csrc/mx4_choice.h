// Which arrangement of the kernels a product of MX4 rows takes, by its sizes.
// Plain C++, so that the choice can be looked at without a GPU.
#pragma once

#include <cstddef>
#include <cstdint>

#include "rslm.h"

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

inline int type_parts(int type) { return type == RSLM_BF16 ? 1 : type == RSLM_F16 ? 2 : 3; }
inline int64_t groups_of(int64_t len) { return (len + 127) / 128; }

// Few rows of x straight from LDS: whether a workgroup's holds their parts.
constexpr int kFewRows = 16, kFewLds = 65536;
constexpr int few_pitch(int steps) { return steps * 256 + 16; }   // bytes of a row of a part
inline bool score_few_ok(int type, int64_t m, int dim) {
  return m <= kFewRows && int64_t(type_parts(type)) * m * few_pitch((dim + 127) / 128) <= kFewLds;
}

// Parts into which the sums over `len` values are split where m x cols has too
// few tiles of bm rows for the GPU: at least two groups of 128 each, none without
// any.  As many workgroups as the GPU holds at once (one of 8 wavefronts to a CU, two of
// 4), and not one more, which all others would be waiting for: gradients of 256 x
// 131,072 x 768 bfloat16 with 255 workgroups 62 us, with 258 103; 100 x 100,000 x 768
// 41 and 64; 64 x 51,200 x 1,024 with 512 24, with 1,024 34.  The gradient has long
// sums and small outputs; for scores, the parts (about 8 bytes written and read
// for a value of each, at 5 TB/s) have to cost less than the groups that a
// workgroup is spared (2 us each, for every part of a number).  us, whole and
// split: 118 x 100 x 2,917 float16 80.0, 19.2; 100 x 8,192 x 4,096 float32 146,
// 42; 300 x 2,000 x 1,024 bfloat16 32.9, 24.1; but 128 x 20,000 x 768 bfloat16 22.3,
// 30.7, which stays whole.
inline int splits_of(int type, int64_t m, int64_t cols, int64_t len, bool backward, int bm) {
  const int64_t tiles = (cols + 255) / 256 * ((m + bm - 1) / bm), groups = groups_of(len);
  const int64_t want = (backward && bm <= 64 ? 512 : 256) / tiles;
  const int64_t most = (groups + 1) / 2;
  int64_t s = want < most ? want : most;
  if (!backward)
    while (s > 1 && m * cols * s > 1200000 * type_parts(type) * (groups - (groups + s - 1) / s)) --s;
  if (s < 1) s = 1;
  const int64_t per = (groups + s - 1) / s;
  return int((groups + per - 1) / per);
}

// Rows of x in a workgroup's tile.  Of 128 and 256, of which a CU holds one
// workgroup, what keeps the CU for less time: rounds of 256 workgroups times the
// groups of each, a group of 256 rows taking 1.6 times that of 128 rows.  Scores, us
// with tiles of 128 and 256: 300 x 100,000 x 768 bfloat16 90, 115; 257 x 20,000 x 1,024
// float32 49, 74; 384 x 30,000 x 1,536 float16 93, 74; 256 x 32,000 x 1,024 bfloat16,
// whose sums stay whole, 27, 38.
inline int tile_rows(int type, int64_t m, int64_t cols, int64_t len, bool backward) {
  if (m <= 128) return m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 128;
  auto time = [&](int rows) {
    const int64_t tiles = (cols + 255) / 256 * ((m + rows - 1) / rows);
    const int64_t parts = splits_of(type, m, cols, len, backward, rows);
    return (tiles * parts + 255) / 256 * ((groups_of(len) + parts - 1) / parts);
  };
  return 5 * time(128) < 8 * time(256) ? 128 : 256;
}
inline int sum_splits(int type, int64_t m, int64_t cols, int64_t len, bool backward) {
  return splits_of(type, m, cols, len, backward, tile_rows(type, m, cols, len, backward));
}

// The gradient's row of b, from the first of its part of the sum, whose code a thread
// takes in a slab of 32 rows, `own` its place among them; at and past the part's end
// too.  Unsigned: slabs ahead of the last group pass 2^31 where one part has all of
// 2^31 - 256 rows.
constexpr uint32_t slab_row(int own, int slab) { return uint32_t(own) + 32u * uint32_t(slab); }

}  // namespace rslm
