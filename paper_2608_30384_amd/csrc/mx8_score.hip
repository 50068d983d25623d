// Products of MX8 rows with MX4 rows (mx4_dev.h):  out[i][j] = sum_d a[i][d] b[j][d].
//
// To 16-bit results by the scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4,
// which takes both kinds of code as they are.  Of every 8 products that it adds first it
// drops what lies more than 13 places below the largest's leading one (each product is cut
// toward zero): less than 2^-13 of the largest for each of the others, of Gaussian rows
// about 6e-6 of a result.  That is far below the rounding to 16 bits, but not float32.
// Float32 results therefore take the bfloat16 instruction, in which every value of either
// row is exact.
#include "mx4_choice.h"
#include "mx4_dev.h"

#include <type_traits>
#include <utility>

namespace rslm {

struct Mx8ScoreCall {
  const uint8_t *ac, *as;
  int64_t m;
  const uint8_t *bc, *bs;
  int64_t n;
  int steps;
  void *out;
  int64_t stride;
  hipStream_t s;
};

// A lane's part of 16 rows' group of 128 coordinates.  Lane l has row l % 16; with
// g = l / 16, of 4-bit codes coordinates 32 g .. + 31, of 8-bit codes 16 g .. + 15 and
// 64 + 16 g .. + 15; the scale is that of coordinates 32 g .. + 31 in either.
struct Mx8Frag {
  i32x4 lo, hi;
  int s;
};
struct Mx4FragB {
  i32x4 q;
  int s;
};
__device__ __forceinline__ f32x4 mx84_mfma(const Mx4FragB &b, const Mx8Frag &a, f32x4 c) {
  const i32x8 x = {b.q[0], b.q[1], b.q[2], b.q[3], 0, 0, 0, 0};
  const i32x8 y = {a.lo[0], a.lo[1], a.lo[2], a.lo[3], a.hi[0], a.hi[1], a.hi[2], a.hi[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 0, 0, b.s, 0, a.s);
}
__device__ __forceinline__ f32x4 mx_mfma_bf16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// ---- few rows of a -----------------------------------------------------------
//
// Up to 16 rows of a to a workgroup.  Bound by reading b, once for these: 1 x 1,000,000 x
// 768 72 us (5.7 TB/s), 1 x 131,072 x 768 11.3.  A wavefront takes 16 rows of b, with two
// groups of them asked for at once; a's rows are in LDS (HELD) where they fit.  Where there
// are few rows of b, the wavefronts of a workgroup share out the groups of the same 16
// (SPLIT), and their sums are added in a fixed order: 1 x 4,096 x 4,096 in less than the 7 us
// of a call, 19 with one wavefront for all groups.
constexpr int kFew8Flight = 2;   // us with 1, 2, 4, 6: 1 x 1,000,000 x 768 92, 72, 90, 80; 16 x 131,072 x 4,096 88, 69, 69, 77

template <int T, bool SPLIT, bool HELD>
__global__ void __launch_bounds__(256) k_mx8_score_few(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                       int64_t rows, const uint8_t *__restrict__ bc,
                                                       const uint8_t *__restrict__ bs, int64_t n, int steps,
                                                       void *__restrict__ out, int64_t stride, int64_t tiles) {
  constexpr bool kExact = T == RSLM_F32;
  constexpr int U = kFew8Flight, kStep = SPLIT ? 4 : 1;
  extern __shared__ uint4 few8_lds[];   // codes, 128 bytes of a row after another's, then scales
  __shared__ f32x4 sums[SPLIT ? 256 : 1];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // rows 16 y .. 16 y + m - 1
  const int64_t row0 = 16 * int64_t(blockIdx.y);
  ac += row0 * steps * 128, as += row0 * steps * 4;
  out = static_cast<typename FloatType<T>::type *>(out) + row0 * stride;
  const int m = int(min(rows - row0, int64_t(16)));
  uint32_t *held_scales = reinterpret_cast<uint32_t *>(few8_lds + m * steps * 8);
  const int64_t each = SPLIT ? int64_t(gridDim.x) : int64_t(gridDim.x) * 4;
  int64_t tile = SPLIT ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wid;
  const int t0 = SPLIT ? wid : 0;
  // the tile's place, the same for all lanes, and a lane's place in it
  const uint8_t *pc, *ps;
  uint32_t own;
  Mx4FragB b[U];
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(t + kStep * u, steps - 1);
      b[u].q = *reinterpret_cast<const i32x4 *>(pc + at * 64 + (own * 64 + 16 * g));
      b[u].s = (ps + at * 4)[own * 4 + g];
    }
  };
  auto begin = [&] {   // past the last tile: its rows again
    const int64_t from = min(tile, tiles - 1) * 16;
    own = uint32_t(min(int64_t(r), n - 1 - from)) * uint32_t(steps);
    pc = bc + from * steps * 64, ps = bs + from * steps * 4;
    fetch(t0);
  };
  begin();
  if constexpr (HELD) {
    for (int i = tid; i < m * steps * 8; i += 256) {
      // piece i % 8 of line i / 8, exchanged by the row's number
      const int line = i >> 3, row = line % m, t = line / m;
      few8_lds[(i & ~7) | ((i ^ row) & 7)] =
          reinterpret_cast<const uint4 *>(ac)[(int64_t(row) * steps + t) * 8 + (i & 7)];
    }
    for (int i = tid; i < m * steps; i += 256)
      held_scales[i] = reinterpret_cast<const uint32_t *>(as)[int64_t(i % m) * steps + i / m];
    __syncthreads();
  }
  const int row_a = min(r, m - 1);
  const int first_piece = kExact ? 2 * g : g, second_piece = kExact ? 2 * g + 1 : 4 + g;
  while (tile < tiles) {
    const int64_t here = tile;
    tile += each;
    f32x4 acc = {};
    for (int t = t0; t < steps; t += kStep * U) {
      Mx4FragB now[U];
#pragma unroll
      for (int u = 0; u < U; ++u) now[u] = b[u];
      if (t + kStep * U < steps) fetch(t + kStep * U);
      else begin();   // the next tile's
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = t + kStep * u;
        if (at >= steps) break;
        Mx8Frag a;
        if constexpr (HELD) {
          const i32x4 *line = reinterpret_cast<const i32x4 *>(few8_lds) + (at * m + row_a) * 8;
          a.lo = line[first_piece ^ (row_a & 7)], a.hi = line[second_piece ^ (row_a & 7)];
          a.s = reinterpret_cast<const uint8_t *>(held_scales)[(at * m + row_a) * 4 + g];
        } else {
          const int64_t from = int64_t(row_a) * steps + at;
          const i32x4 *line = reinterpret_cast<const i32x4 *>(ac) + from * 8;
          a.lo = line[first_piece], a.hi = line[second_piece];
          a.s = as[from * 4 + g];
        }
        if constexpr (kExact) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const i32x4 w = q < 2 ? a.lo : a.hi;
            acc = mx_mfma_bf16(mx4_bf16x8(uint32_t(now[u].q[q]), e8m0_arg(now[u].s)),
                               mx8_bf16x8(make_uint2(uint32_t(w[2 * (q & 1)]), uint32_t(w[2 * (q & 1) + 1])), e8m0_arg(a.s)),
                               acc);
          }
        } else {
          acc = mx84_mfma(now[u], a, acc);
        }
      }
    }
    if constexpr (SPLIT) {
      sums[tid] = acc;
      __syncthreads();
      if (wid == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) acc += sums[64 * w + lane];
      }
      __syncthreads();
      if (wid) continue;
    }
    if (r < m)
      store_float4<T>(static_cast<typename FloatType<T>::type *>(out) + r * stride, here * 16 + 4 * g, n, acc);
  }
}

// ---- large products: tiles in LDS ------------------------------------------
//
// A workgroup of 4 wavefronts takes 32 MF rows of a by 256 of b, each wavefront 16 MF by
// 128, one group of 128 coordinates after another.  The memory unit writes codes and
// scales to LDS by itself.  With 256 rows of a there are three places for a group: in group
// t those of t + 2 are asked for, and one barrier, behind the last read of group t's place,
// waits for those of t + 1 alone, a group and a half old.  With 128 rows there are two, and
// two workgroups to a CU: those of t + 2 are asked for behind the barrier, which waits for
// all, and the other workgroup multiplies meanwhile.  The rows of b of the next group, and
// the first two fragments of a's, are then read to registers under the group's last
// instructions, each fragment of b behind the last one that uses the register; the others
// of a two fragments ahead.  A read or a load or two fit behind a matrix instruction, which
// the unit works on for 32 cycles.  8,192 x 32,768 x 4,096 in 833 to 922 us (up to 2,640
// TFLOP/s; the instruction alone reaches 4,700), 1,133 with 128 rows, which LDS bounds; 300 x
// 100,000 x 768 33 us with 128 rows, 43 with one workgroup to a CU.  A workgroup that went
// on from tile to tile took more (1,024 us): its loads' places and addresses do not leave
// room for the sums in the registers.
//
// LDS, by lines of 128 bytes: a row of a, or two of b.  A line's eight 16-byte pieces are
// exchanged by its number, so that the rows of a read fall on different banks; the
// exchange is in the address that a lane of the load gives.  Rows of b are dealt to the
// fragments so that two of them share out 32 rows, eight to a lane, which are 16 bytes of
// out.
constexpr int kS8LineA = 128;   // bytes of a row of a
constexpr int kS8LineB = 64;    // bytes of a row of b

// f(0), .., f(N - 1), each with a constant of its own.
template <int... I, class F>
__device__ __forceinline__ void for_each_of(std::integer_sequence<int, I...>, F &&f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void for_each(F &&f) {
  for_each_of(std::make_integer_sequence<int, N>{}, f);
}

template <int T, int MF>
__global__ void __launch_bounds__(256, MF == 4 ? 2 : 1) k_mx8_score_tile(
    const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as, int64_t m, const uint8_t *__restrict__ bc,
    const uint8_t *__restrict__ bs, int64_t n, int steps, void *__restrict__ out, int64_t stride, int mtiles) {
  static_assert(T != RSLM_F32, "16-bit results");
  static_assert(MF == 8 || MF == 4, "the places of reads and loads between the instructions");
  constexpr int BM = 32 * MF, BN = kMmN;
  constexpr int LA = BM / 32, LB = BN / 64, kLoads = LA + LB + 2;   // loads of a wavefront and group
  constexpr int kA = BM * kS8LineA, kB = BN * kS8LineB, kS = 4 * (BM + BN);
  constexpr int kPlaces = MF == 4 ? 2 : 3;
  constexpr int kB0 = kPlaces * kA, kS0 = kB0 + kPlaces * kB, kNone = kS0 + kPlaces * kS;
  __shared__ __align__(1024) uint8_t lds[kNone + 256];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the 8 XCDs in turn: each XCD takes a run of tiles, in which those of
  // 8 rows of tiles are neighbours.
  const int tiles = gridDim.x, per = tiles / 8, rest = tiles % 8;
  const int xcd = blockIdx.x % 8, at = blockIdx.x / 8 + xcd * per + min(xcd, rest);
  const int ntiles = tiles / mtiles;
  const int band = at / (8 * ntiles), rows = min(8, mtiles - 8 * band), in = at - band * 8 * ntiles;
  const int64_t m0 = int64_t(8 * band + in % rows) * BM, n0 = int64_t(in / rows) * BN;
  const uint32_t cpa = 128u * steps, cpb = 64u * steps, sp = 4u * steps;
  const i32x4 ra = buffer_of(ac + m0 * cpa, (m - m0) * cpa), rb = buffer_of(bc + n0 * cpb, (n - n0) * cpb);
  const i32x4 rsa = buffer_of(as + m0 * sp, (m - m0) * sp), rsb = buffer_of(bs + n0 * sp, (n - n0) * sp);
  const uint32_t lds0 = lds_address(lds);

  // ---- loads.  A lane of one has line l / 8 of 8 and place l % 8 of it.
  const int line = lane >> 3, place = lane & 7;
  const uint32_t va = (wid * (8 * LA) + line) * cpa + ((place ^ line) << 4);
  // b: line / 2 rows; the exchange, by bit 0 and bits 2 and 3 of the line
  uint32_t vb[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int slot = place ^ ((line & 1) | ((((line + 8 * j) >> 2) & 3) << 1));
    vb[j] = (wid * (16 * LB) + 16 * j + 2 * line + (slot >> 2)) * cpb + ((slot & 3) << 4);
  }
  const uint32_t vs = (wid * 64 + lane) * sp;
  // load i of group t, to place p.  Past the last group the loads keep their number, from past
  // the end or, of buffers of over 2 GiB, from other rows: what they bring is not multiplied.
  auto load = [&](int t, int p, int i) {
    const uint32_t past = t < steps ? 0u : 0x80000000u;
    if (i < LA)
      load_to_lds(ra, lds0 + p * kA + (wid * LA + i) * 1024, (va + (8 * i) * cpa + t * kS8LineA) | past);
    else if (i < LA + LB)
      load_to_lds(rb, lds0 + kB0 + p * kB + (wid * LB + i - LA) * 1024,
                  (vb[(i - LA) & 1] + (32 * ((i - LA) >> 1)) * cpb + t * kS8LineB) | past);
    else if (i == LA + LB)
      load_to_lds<4>(rsa, lds0 + (wid * 64 < BM ? kS0 + p * kS + wid * 256 : kNone), (vs + t * 4) | past);
    else
      load_to_lds<4>(rsb, lds0 + kS0 + p * kS + 4 * BM + wid * 256, (vs + t * 4) | past);
  };

  // ---- reads
  const int wm = (wid >> 1) * (16 * MF), wn = (wid & 1) * 128;
  // row of b of lane l's part of fragment j
  auto b_row = [](int l, int j) { return 32 * (j >> 1) + 8 * (l >> 2) + 4 * (j & 1) + (l & 3); };
  const int ra_lo = (wm + r) * kS8LineA + ((g ^ (r & 7)) << 4);
  const int ra_hi = (wm + r) * kS8LineA + (((4 + g) ^ (r & 7)) << 4);
  const int rb_row = wn + b_row(r, 0);
  const int rb_off = kB0 + (rb_row >> 1) * 128 + (((4 * (r & 1) + g) ^ (((r >> 1) & 1) | ((r >> 2) << 1))) << 4);
  const int rsa_off = kS0 + (wm + r) * 4 + g, rsb_off = kS0 + 4 * BM + rb_row * 4 + g;
  Mx8Frag fa[4];
  Mx4FragB fb[8];
  auto read_a = [&](int p, int k, int part) {
    if (part == 0) fa[k & 3].lo = *reinterpret_cast<const i32x4 *>(&lds[p * kA + ra_lo + 16 * k * kS8LineA]);
    else if (part == 1) fa[k & 3].hi = *reinterpret_cast<const i32x4 *>(&lds[p * kA + ra_hi + 16 * k * kS8LineA]);
    else fa[k & 3].s = lds[p * kS + rsa_off + 64 * k];
  };
  auto read_b = [&](int p, int j) {
    fb[j].q = *reinterpret_cast<const i32x4 *>(&lds[p * kB + rb_off + (b_row(0, j) >> 1) * 128]);
    fb[j].s = lds[p * kS + rsb_off + b_row(0, j) * 4];
  };

  f32x4 acc[MF][8] = {};
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(p, p, i);
  arrive<kLoads>();   // the first group's
#pragma unroll
  for (int j = 0; j < 8; ++j) read_b(0, j);
#pragma unroll
  for (int i = 0; i < 6; ++i) read_a(0, i / 3, i % 3);

  // Group t is in place p, the next one in p1, and p2 is free to be written.
  int p = 0;
  for (int t = 0; t < steps; ++t) {
    const int p1 = p == kPlaces - 1 ? 0 : p + 1, p2 = p1 == kPlaces - 1 ? 0 : p1 + 1;
    for_each<8 * MF>([&](auto q_) __attribute__((always_inline)) {
      constexpr int q = decltype(q_)::value;
      constexpr int k = q / 8, j = q % 8;
      if constexpr (q == 8 * (MF - 2)) arrive<MF == 4 ? 0 : kLoads>();
      acc[k][j] = mx84_mfma(fb[j], fa[k & 3], acc[k][j]);
      if constexpr (k < MF - 2 && j % 2 == 1 && j < 7) read_a(p, k + 2, j >> 1);
      if constexpr (MF == 8 && q % 3 == 0 && q / 3 < kLoads) load(t + 2, p2, q / 3);
      if constexpr (MF == 4 && q >= 16 && q - 16 < kLoads) load(t + 2, p, q - 16);
      if constexpr (k == MF - 2 && j < 6) read_a(p1, j / 3, j % 3);
      if constexpr (k == MF - 1) read_b(p1, j);
      __builtin_amdgcn_sched_barrier(0);
    });
    p = p1;
  }

  // Through LDS, so that a store writes 4 rows of 256 consecutive bytes, a part of LDS
  // for each wavefront.
  typedef typename FloatType<T>::type Out;
  struct __attribute__((packed, aligned(alignof(Out)))) Wide {
    uint32_t v[4];
  };
  constexpr int kOwn = MF == 8 ? 32768 : 16384;
  static_assert(4 * kOwn <= kNone, "LDS of the stores");
  arrive<0>();   // the last operands have been read, and the last loads have come, everywhere
  uint8_t *own = lds + wid * kOwn;
#pragma unroll
  for (int k = 0; k < MF; ++k)
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const int piece = b_row(4 * g, j) / 8, row = 16 * k + r;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = uint32_t(float_to_h16<T>(acc[k][j + (i >> 1)][2 * (i & 1)])) |
               uint32_t(float_to_h16<T>(acc[k][j + (i >> 1)][2 * (i & 1) + 1])) << 16;
      *reinterpret_cast<uint4 *>(own + row * 256 + 16 * (piece ^ r)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wavefront's own part
#pragma unroll 4
  for (int i = 0; i < 4 * MF; ++i) {
    const int row = 4 * i + (lane >> 4), piece = lane & 15;
    const uint4 v = *reinterpret_cast<const uint4 *>(own + row * 256 + 16 * (piece ^ (row & 15)));
    const int64_t orow = m0 + wm + row, c = n0 + wn + piece * 8;
    if (orow >= m) continue;
    Out *o = static_cast<Out *>(out) + orow * stride + c;
    if (c + 8 <= n) {   // rows may begin anywhere
      *reinterpret_cast<Wide *>(o) = __builtin_bit_cast(Wide, v);
    } else {
      Out e[8];
      __builtin_memcpy(e, &v, 16);
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (c + q < n) o[q] = e[q];
    }
  }
}

// ---- large products to float32 -------------------------------------------------
//
// The same tiles and places, multiplied in bfloat16.  A group is taken in two passes, of 16
// of each lane's 32 coordinates: in a pass a wavefront has its 128 rows of b in bfloat16 and
// goes through its fragments of a, 16 instructions to one.  A step ahead a's 16 codes of a
// lane are turned to bfloat16, two ahead they are read; at a pass's last step b's are turned,
// each fragment behind the last instruction that uses the register.  The barrier, late in
// the second pass, waits for the next group, and those after it are asked for behind it.
// Two workgroups to a CU (MF 2) leave 256 registers, which are 5 too few: 24 bytes a lane go to
// scratch memory, and one of these, an address, is read back in each group behind the barrier,
// where all but the first matrix instruction wait for it.
template <int MF>
__global__ void __launch_bounds__(256, MF == 2 ? 2 : 1) k_mx8_score_tile_f32(
    const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as, int64_t m, const uint8_t *__restrict__ bc,
    const uint8_t *__restrict__ bs, int64_t n, int steps, float *__restrict__ out, int64_t stride, int mtiles) {
  static_assert(MF == 8 || MF == 2, "the places of reads and loads between the instructions");
  constexpr int BM = 32 * MF, BN = kMmN;
  constexpr int LA = BM / 32, LB = BN / 64, kLoads = LA + LB + 2;   // loads of a wavefront and group
  constexpr int kA = BM * kS8LineA, kB = BN * kS8LineB, kS = 4 * (BM + BN);
  constexpr int kB0 = 3 * kA, kS0 = kB0 + 3 * kB, kNone = kS0 + 3 * kS;
  __shared__ __align__(1024) uint8_t lds[kNone + 256];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles = gridDim.x, per = tiles / 8, rest = tiles % 8;
  const int xcd = blockIdx.x % 8, at = blockIdx.x / 8 + xcd * per + min(xcd, rest);
  const int ntiles = tiles / mtiles;
  const int band = at / (8 * ntiles), rows = min(8, mtiles - 8 * band), in = at - band * 8 * ntiles;
  const int64_t m0 = int64_t(8 * band + in % rows) * BM, n0 = int64_t(in / rows) * BN;
  const uint32_t cpa = 128u * steps, cpb = 64u * steps, sp = 4u * steps;
  const i32x4 ra = buffer_of(ac + m0 * cpa, (m - m0) * cpa), rb = buffer_of(bc + n0 * cpb, (n - n0) * cpb);
  const i32x4 rsa = buffer_of(as + m0 * sp, (m - m0) * sp), rsb = buffer_of(bs + n0 * sp, (n - n0) * sp);
  const uint32_t lds0 = lds_address(lds);

  // ---- loads, as above; a line of b is exchanged by its number
  const int line = lane >> 3, place = lane & 7, slot = place ^ line;
  const uint32_t va = (wid * (8 * LA) + line) * cpa + (slot << 4);
  const uint32_t vb = (wid * (16 * LB) + 2 * line + (slot >> 2)) * cpb + ((slot & 3) << 4);
  const uint32_t vs = (wid * 64 + lane) * sp;
  auto load = [&](int t, int p, int i) {
    const uint32_t past = t < steps ? 0u : 0x80000000u;
    if (i < LA)
      load_to_lds(ra, lds0 + p * kA + (wid * LA + i) * 1024, (va + (8 * i) * cpa + t * kS8LineA) | past);
    else if (i < LA + LB)
      load_to_lds(rb, lds0 + kB0 + p * kB + (wid * LB + i - LA) * 1024, (vb + (16 * (i - LA)) * cpb + t * kS8LineB) | past);
    else if (i == LA + LB)
      load_to_lds<4>(rsa, lds0 + (wid * 64 < BM ? kS0 + p * kS + wid * 256 : kNone), (vs + t * 4) | past);
    else
      load_to_lds<4>(rsb, lds0 + kS0 + p * kS + 4 * BM + wid * 256, (vs + t * 4) | past);
  };

  // ---- reads: a's 16 bytes 32 g + 16 pass .. of a fragment's rows, b's 32 g .. of all
  const int wm = (wid >> 1) * (16 * MF), wn = (wid & 1) * 128;
  const int ra0 = (wm + r) * kS8LineA + (((2 * g) ^ (r & 7)) << 4), ra1 = (wm + r) * kS8LineA + (((2 * g + 1) ^ (r & 7)) << 4);
  const int rb_off = kB0 + ((wn + r) >> 1) * 128 + (((4 * (r & 1) + g) ^ ((r >> 1) & 7)) << 4);
  const int rsa_off = kS0 + (wm + r) * 4 + g, rsb_off = kS0 + 4 * BM + (wn + r) * 4 + g;
  i32x4 code[2];   // of a, by the step's parity
  int scale[2];
  uint4 x[2][2];   // in bfloat16, both halves
  Mx4FragB fb[8];
  uint4 y[2][8];
  auto read_a = [&](int p, int step) {   // steps of the next group are 2 MF and 2 MF + 1
    const int k = step % MF, pass = step / MF % 2;
    code[step & 1] = *reinterpret_cast<const i32x4 *>(&lds[p * kA + (pass ? ra1 : ra0) + 16 * k * kS8LineA]);
    scale[step & 1] = lds[p * kS + rsa_off + 64 * k];
  };
  auto turn_a = [&](int step, int q) {
    const i32x4 w = code[step & 1];
    x[step & 1][q] = mx8_bf16x8(make_uint2(uint32_t(w[2 * q]), uint32_t(w[2 * q + 1])), e8m0_arg(scale[step & 1]));
  };
  auto read_b = [&](int p, int j) {
    fb[j].q = *reinterpret_cast<const i32x4 *>(&lds[p * kB + rb_off + 8 * j * 128]);
    fb[j].s = lds[p * kS + rsb_off + 64 * j];
  };
  auto turn_b = [&](int pass, int q, int j) { y[q][j] = mx4_bf16x8(uint32_t(fb[j].q[2 * pass + q]), e8m0_arg(fb[j].s)); };

  f32x4 acc[MF][8] = {};
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(p, p, i);
  arrive<kLoads>();
#pragma unroll
  for (int j = 0; j < 8; ++j) read_b(0, j);
  read_a(0, 0);
  read_a(0, 1);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    turn_a(0, q);
#pragma unroll
    for (int j = 0; j < 8; ++j) turn_b(0, q, j);
  }

  // Group t is in place p, the next one in p1, and p2 is free behind the barrier.
  int p = 0;
  for (int t = 0; t < steps; ++t) {
    const int p1 = p == 2 ? 0 : p + 1, p2 = p1 == 2 ? 0 : p1 + 1;
    for_each<32 * MF>([&](auto i_) __attribute__((always_inline)) {
      constexpr int i = decltype(i_)::value, step = i / 16, q = i / 8 % 2, j = i % 8, k = step % MF;
      constexpr int late = i - 16 * (2 * MF - 4);   // behind the barrier
      if constexpr (late == 0) arrive<0>();
      acc[k][j] = mx_mfma_bf16(y[q][j], x[step & 1][q], acc[k][j]);
      if constexpr (i % 16 == 0) read_a(step + 2 < 2 * MF ? p : p1, step + 2);
      if constexpr (i % 16 == 6) turn_a(step + 1, 0);
      if constexpr (i % 16 == 12) turn_a(step + 1, 1);
      // the next group's rows of b, behind the first pass's end and ahead of the second's
      constexpr int from = MF == 2 ? 32 : 0, each = MF == 2 ? 2 : 4;
      if constexpr (late >= from && late < from + 8 * each && late % each == each / 2) read_b(p1, (late - from) / each);
      if constexpr (late >= 0 && late % 4 == 0 && late / 4 < kLoads) load(t + 2, p2, late / 4);
      if constexpr (k == MF - 1) turn_b(1 - step / MF, q, j);
      __builtin_amdgcn_sched_barrier(0);
    });
    p = p1;
  }

  // Through LDS, so that a store writes 2 rows of 512 consecutive bytes, a part of LDS for
  // each wavefront.  Of small tiles past the caches' order: us, with and without, and with the
  // log probabilities that read the scores behind them
  //     255 x 100,003 x 1,024   67   71    89   92    2,048 x 131,072 x 768   464  570   723  806
  //   1,000 x  50,000 x    96   46   50    87   85
  // Large tiles gain less and the readers lose it: 2,048 x 32,768 x 4,096 440, 453, then 510, 482;
  // 16-bit results of 2,048 x 131,072 x 768 217, 265, then 403, 399.
  typedef uint32_t Wide __attribute__((ext_vector_type(4), aligned(4)));
  constexpr int kOwn = MF == 8 ? 32768 : 16384, kRows = kOwn / 512;   // rows at a time
  static_assert(4 * kOwn <= kNone, "LDS of the stores");
  arrive<0>();   // the last operands have been read, and the last loads have come, everywhere
  uint8_t *own = lds + wid * kOwn;
#pragma unroll
  for (int k0 = 0; k0 < MF; k0 += kRows / 16) {
#pragma unroll
    for (int k = k0; k < k0 + kRows / 16; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint4 *>(own + (16 * (k - k0) + r) * 512 + 16 * ((4 * j + g) ^ r)) =
            __builtin_bit_cast(uint4, acc[k][j]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wavefront's own part
#pragma unroll 4
    for (int i = 0; i < kRows / 2; ++i) {
      const int row = 2 * i + (lane >> 5), piece = lane & 31;
      const uint4 v = *reinterpret_cast<const uint4 *>(own + row * 512 + 16 * (piece ^ (row & 15)));
      const int64_t orow = m0 + wm + 16 * k0 + row, c = n0 + wn + piece * 4;
      if (orow >= m) continue;
      float *o = out + orow * stride + c;
      if (c + 4 <= n) {   // rows may begin anywhere
        if constexpr (MF == 2) __builtin_nontemporal_store(__builtin_bit_cast(Wide, v), reinterpret_cast<Wide *>(o));
        else *reinterpret_cast<Wide *>(o) = __builtin_bit_cast(Wide, v);
      } else {
        const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (c + q < n) o[q] = __uint_as_float(e[q]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <int T, int MF>
static void launch_score8_tile(const Mx8ScoreCall &c) {
  const int64_t mt = (c.m + 32 * MF - 1) / (32 * MF), nt = (c.n + kMmN - 1) / kMmN;
  const dim3 grid(unsigned(mt * nt));
  if constexpr (T == RSLM_F32)
    hipLaunchKernelGGL(k_mx8_score_tile_f32<MF>, grid, dim3(256), 0, c.s, c.ac, c.as, c.m, c.bc, c.bs, c.n, c.steps,
                       static_cast<float *>(c.out), c.stride, int(mt));
  else
    hipLaunchKernelGGL((k_mx8_score_tile<T, MF>), grid, dim3(256), 0, c.s, c.ac, c.as, c.m, c.bc, c.bs, c.n, c.steps,
                       c.out, c.stride, int(mt));
}

template <int T, bool SPLIT, bool HELD>
static void launch_score8_few_one(const Mx8ScoreCall &c) {
  const int64_t tiles = (c.n + 15) / 16, wg = SPLIT ? tiles : (tiles + 3) / 4, groups = (c.m + 15) / 16;
  const size_t lds = HELD ? size_t(c.m < 16 ? c.m : 16) * c.steps * 132 : 0;
  // no more workgroups than the GPU holds at once, so that each fills its LDS once, and the
  // same number of tiles to each
  const int64_t all = 256 * (lds > 40960 ? 2 : lds > 20480 ? 3 : 4), most = all > groups ? all / groups : 1;
  const int64_t rounds = (wg + most - 1) / most;
  hipLaunchKernelGGL((k_mx8_score_few<T, SPLIT, HELD>), dim3(unsigned((wg + rounds - 1) / rounds), unsigned(groups)), dim3(256),
                     lds, c.s, c.ac, c.as, c.m, c.bc, c.bs, c.n, c.steps, c.out, c.stride, tiles);
}
template <int T>
static void launch_score8_few(const Mx8ScoreCall &c) {
  const bool split = few8_split(c.n, c.steps), held = few8_held(c.m, c.steps);
  if (split && held) launch_score8_few_one<T, true, true>(c);
  else if (split) launch_score8_few_one<T, true, false>(c);
  else if (held) launch_score8_few_one<T, false, true>(c);
  else launch_score8_few_one<T, false, false>(c);
}

template <int T>
static void launch_score8(const Mx8ScoreCall &c) {
  switch (score8_form(c.m, c.n, c.steps, T == RSLM_F32)) {
    case kS8Few: launch_score8_few<T>(c); break;
    case kS8Tile256: launch_score8_tile<T, 8>(c); break;
    default: launch_score8_tile<T, T == RSLM_F32 ? 2 : 4>(c);
  }
}

}  // namespace rslm

using namespace rslm;

extern "C" {

int rslm_mx8_score(const uint8_t *a_codes, const uint8_t *a_scales, int64_t m, const uint8_t *b_codes,
                   const uint8_t *b_scales, int64_t n, int32_t dim, void *out, int32_t dtype, int64_t stride,
                   void *stream) {
  if (m < 0 || n < 0 || m > 65535 * 64ll || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim ||
      !float_type_ok(dtype) || (m > 1 && stride < n))
    return RSLM_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return RSLM_OK;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out || !aligned_to(a_codes, 16) ||
      !aligned_to(b_codes, 16) || !aligned_to(a_scales, 4) || !aligned_to(b_scales, 4) ||
      !aligned_to(out, float_bytes(dtype)))
    return RSLM_ERR_INVALID_ARG;
  const Mx8ScoreCall c{a_codes, a_scales, m, b_codes, b_scales, n, mx4_steps(dim), out, stride, as_stream(stream)};
  if (dtype == RSLM_F32) launch_score8<RSLM_F32>(c);
  else if (dtype == RSLM_F16) launch_score8<RSLM_F16>(c);
  else launch_score8<RSLM_BF16>(c);
  return check_launch();
}

}  // extern "C"
