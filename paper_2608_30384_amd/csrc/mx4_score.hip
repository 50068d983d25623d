// Products of float rows with MX4 rows, and their gradient:
//   score    out[i][j] = sum_d x[i][d] b[j][d]
//   gradient dx[i][d]  = sum_j dout[i][j] b[j][d]
// on the bfloat16 matrix cores, without rounding an operand: every MX4 value is
// a bfloat16 (v_cvt_scalef32_pk_bf16_fp4), and a float is the sum of 1 (bfloat16),
// 2 (float16) or 3 (float32) bfloat16 parts, cut off the top of its significand
// one after the other.  The products of the parts are exact in the matrix
// cores' float32, so the result has the error of a float32 sum.
#include "mx4_choice.h"
#include "mx4_dev.h"

#include <type_traits>

namespace rslm {

template <int T>
struct Parts {
  static constexpr int n = T == RSLM_BF16 ? 1 : T == RSLM_F16 ? 2 : 3;
};

// The bfloat16 parts of 8 floats, two to a word.  Cutting (not rounding) keeps
// a part from overflowing, and 8 bits at a time take 24 in three.  An infinity
// or a NaN is one part (a NaN whose upper bits are zero is kept one).
template <int NS>
__device__ __forceinline__ void split8(uint4 (&p)[NS], const float (&v)[8]) {
  uint32_t w[NS][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float rest = v[i];
    const uint32_t bits = __float_as_uint(rest);
    const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      w[s][i] = __float_as_uint(rest) & 0xffff0000u;
      rest -= __uint_as_float(w[s][i]);
    }
    if (NS > 1 && !finite) {
      w[0][i] |= (bits & 0x007fffffu) ? 0x00400000u : 0u;
#pragma unroll
      for (int s = 1; s < NS; ++s) w[s][i] = 0u;
    }
  }
#pragma unroll
  for (int s = 0; s < NS; ++s)
    p[s] = make_uint4((w[s][0] >> 16) | w[s][1], (w[s][2] >> 16) | w[s][3], (w[s][4] >> 16) | w[s][5],
                      (w[s][6] >> 16) | w[s][7]);
}

__device__ __forceinline__ f32x4 mfma_bf16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

typedef short i16x4 __attribute__((ext_vector_type(4)));

// ---- few rows of x: b is read once, straight to the operands -----------------
//
// Bound by reading b where b is large: 1 x 1,000,000 x 768 bfloat16 79 us, 5.2 TB/s.  A
// wavefront walks all groups of its rows, so that few rows of b leave most of the GPU
// idle: 1 x 4,096 x 4,096 17 us a call, of 2 us of bytes.  It takes 16 NT rows of b;
// lane group g has the 32 coordinates 32 g .. + 31 of a group of 128, as the rows are stored, and
// multiplies eight of them at a time: the order of the sum is free, so x is read
// in that order from LDS, where a workgroup keeps its parts for all its tiles.

template <int T, int TO, int NT>
__global__ void __launch_bounds__(256) k_mx4_score_few(const void *__restrict__ x, int m, int64_t stride,
                                                       const uint8_t *__restrict__ bc,
                                                       const uint8_t *__restrict__ bs, int64_t n, int dim, int steps,
                                                       void *__restrict__ out, int64_t ostride, int64_t tiles) {
  constexpr int NS = Parts<T>::n;
  extern __shared__ uint4 few_lds[];
  char *lds = reinterpret_cast<char *>(few_lds);
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int pitch = few_pitch(steps);
  for (int i = tid; i < m * steps * 16; i += 256) {
    const int row = i / (steps * 16), c = i - row * (steps * 16);
    float v[8];
    load_float8<T>(v, static_cast<const typename FloatType<T>::type *>(x) + row * stride, 8 * c, dim);
    uint4 p[NS];
    split8<NS>(p, v);
#pragma unroll
    for (int s = 0; s < NS; ++s) *reinterpret_cast<uint4 *>(lds + (s * m + row) * pitch + 16 * c) = p[s];
  }
  __syncthreads();
  const char *xr = lds + min(r, m - 1) * pitch + 64 * g;
  for (int64_t tile = int64_t(blockIdx.x) * 4 + (tid >> 6); tile < tiles; tile += int64_t(gridDim.x) * 4) {
    const uint8_t *pc[NT], *ps[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t row = min(tile * (16 * NT) + 16 * j + r, n - 1);
      pc[j] = bc + row * steps * 64 + 16 * g;
      ps[j] = bs + row * steps * 4 + g;
    }
    f32x4 acc[NT] = {};
    constexpr int U = 4 / NT < 1 ? 1 : 4 / NT;   // groups read at once
    i32x4 q[U][NT];
    uint32_t sc[U][NT];
    auto fetch = [&](int t) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int at = min(t + u, steps - 1);
          q[u][j] = *reinterpret_cast<const i32x4 *>(pc[j] + at * 64);
          sc[u][j] = ps[j][at * 4];
        }
    };
    fetch(0);
    for (int t = 0; t < steps; t += U) {
      i32x4 w[U][NT];
      float a[U][NT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < NT; ++j) w[u][j] = q[u][j], a[u][j] = e8m0_arg(sc[u][j]);
      if (t + U < steps) fetch(t + U);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (t + u >= steps) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4 fb[NT];
#pragma unroll
          for (int j = 0; j < NT; ++j) fb[j] = mx4_bf16x8(uint32_t(w[u][j][i]), a[u][j]);
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            const uint4 fa = *reinterpret_cast<const uint4 *>(xr + s * m * pitch + (t + u) * 256 + 16 * i);
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[j] = mfma_bf16(fb[j], fa, acc[j]);
          }
        }
      }
    }
    if (r < m) {
      typename FloatType<TO>::type *orow = static_cast<typename FloatType<TO>::type *>(out) + r * ostride;
#pragma unroll
      for (int j = 0; j < NT; ++j) store_float4<TO>(orow, tile * (16 * NT) + 16 * j + 4 * g, n, acc[j]);
    }
  }
}

// ---- more rows: tiles in LDS --------------------------------------------------
//
// Parts of x as planes of bfloat16 rows, zero past the contracted length and
// padded to groups of 128: what the tiles load to LDS as it is.
template <int T>
__global__ void __launch_bounds__(256) k_mx4_split(const void *__restrict__ x, int64_t m, int64_t stride, int64_t len,
                                                   int64_t pad, uint4 *__restrict__ planes) {
  constexpr int NS = Parts<T>::n;
  const int64_t pieces = pad / 8;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < m * pieces; i += int64_t(gridDim.x) * 256) {
    const int64_t row = i / pieces, c = 8 * (i - row * pieces), left = len - c;
    float v[8];
    load_float8<T>(v, static_cast<const typename FloatType<T>::type *>(x) + row * stride + c, 0,
                   int(left < 0 ? 0 : left > 8 ? 8 : left));
    uint4 p[NS];
    split8<NS>(p, v);
#pragma unroll
    for (int s = 0; s < NS; ++s) planes[s * m * pieces + i] = p[s];
  }
}

// WM x WN wavefronts, each 16 MF rows of x by 16 NF columns, over slabs of 32
// contracted values (one matrix instruction), four to a group of 128.  x's
// planes come to LDS by themselves, AG slabs at a time, the next ones while these
// are multiplied; b's codes come to registers up to eight slabs ahead, are turned
// to bfloat16 and written to LDS a slab ahead of their use.
// TRANS false: columns are rows of b, contracted over their coordinates.  TRANS
// true: columns are coordinates, contracted over the rows of b, which the
// matrix operand needs across the rows as they are stored: read from LDS through
// the transposing 64-bit loads (lane i of 16 gives the address of row i / 4,
// columns 4 (i % 4) .. + 3, and takes column i of the four rows).
// 16-byte pieces of LDS rows change places by the row's number, so that the
// lanes of a read or write fall on different banks: 16 lanes of a 128-bit
// access are {0..3, 20..23, 4..7, 16..19}, ..., and go to 64 banks at once.
template <int TO, int NS, int MF, int WM, int NF, int WN, int AG, bool TRANS>
__global__ void __launch_bounds__(64 * WM * WN, WM * WN == 8 ? 1 : 2) k_mx4_gemm(
    const uint8_t *__restrict__ xp, int64_t m, int64_t pitch, int64_t plane, const uint8_t *__restrict__ bc,
    const uint8_t *__restrict__ bs, int64_t n, int dim, int steps, void *__restrict__ out, int64_t ostride,
    float *__restrict__ part, int64_t groups, int64_t per, int mtiles, int tiles) {
  constexpr int W = WM * WN, BM = 16 * MF * WM, BN = 16 * NF * WN;
  constexpr int kWords = 16 / W, kPer = 4 / kWords;     // 4-byte words of codes of a thread in a slab; threads of a block
  static_assert(BN == 256 && (W == 4 || W == 8), "256 blocks of 32 codes in a slab");
  constexpr int kARow = 64 * AG;                        // bytes of a row of a plane in LDS
  constexpr int kABytes = BM * kARow;                   // of a plane
  __shared__ __align__(1024) uint8_t la[2][NS * kABytes];
  __shared__ __align__(1024) uint8_t lb[2][BN * 64];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t cols = TRANS ? dim : n;
  // Workgroups go to the 8 XCDs in turn: each XCD takes a run of them, in which
  // the tiles of one part of the sum are neighbours, rows of x first.
  const int all = gridDim.x, tper = all / 8, trest = all % 8, xcd = blockIdx.x % 8;
  const int at = blockIdx.x / 8 + xcd * tper + min(xcd, trest);
  const int split = at / tiles, tile = at - split * tiles;
  const int64_t m0 = int64_t(tile % mtiles) * BM, c0 = int64_t(tile / mtiles) * BN;
  const int64_t g0 = int64_t(split) * per;
  const int count = int(min(groups, g0 + per) - g0);    // groups
  const int wm = (wid / WN) * (16 * MF), wn = (wid % WN) * (16 * NF);

  // x: 64 lanes take 16 / AG rows of 64 AG bytes; rows past the last read it again
  constexpr int kARows = 16 / AG, kLoads = (BM / kARows + W - 1) / W;  // loads of a plane by a wavefront
  auto turn = [](int row) { return AG == 1 ? (row >> 1) & 2 : row & (4 * AG - 1); };
  const uint32_t la0 = lds_address(la);
  const uint8_t *pa[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (W * i + wid) * kARows + lane / (4 * AG), piece = lane % (4 * AG);
    pa[i] = xp + min(m0 + row, m - 1) * pitch + g0 * 256 + 16 * (piece ^ turn(row));
  }
  auto load_a = [&](int slab, int buf) {   // AG slabs from `slab` on, or the last ones
    const int64_t off = int64_t(min(slab, 4 * count - AG)) * 64;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (W * kLoads * kARows == BM || W * i + wid < BM / kARows)
          load_to_lds(pa[i] + (s * plane + off), la0 + (buf * NS + s) * kABytes + (W * i + wid) * 1024);
  };
  // b: codes and scale of a slab, block tid / kPer, part tid % kPer; slab s in
  // place s % 8
  typedef int words __attribute__((ext_vector_type(kWords)));
  words q[8];
  uint32_t sc[8];
  const int own = tid / kPer, in_block = 4 * kWords * (tid % kPer);
  const int64_t row0 = TRANS ? g0 * 128 : min(c0 + own, n - 1);
  const int block = TRANS ? min(int(c0 / 32) + (own & 7), 4 * steps - 1) : 0;
  const uint8_t *pc = bc + (TRANS ? (row0 * steps * 4 + block) * 16 : (row0 * steps + g0) * 64) + in_block;
  const uint8_t *ps = bs + (TRANS ? row0 * steps * 4 + block : (row0 * steps + g0) * 4);
  const uint32_t last = TRANS ? uint32_t(min(n - g0 * 128, int64_t(count) * 128)) - 1u : 0u;   // row of b, from row0
  auto load_b = [&](int slab, int place) {   // TRANS
    const uint32_t row = min(slab_row(own >> 3, slab), last);   // past the end: the last one, and zeros (put_b)
    q[place] = *reinterpret_cast<const words *>(pc + uint64_t(row) * uint32_t(64 * steps));
    sc[place] = ps[uint64_t(row) * uint32_t(4 * steps)];
  };
  auto load_b4 = [&](int grp, int place) {   // not TRANS: a whole group
    const int t = min(grp, count - 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) q[place + j] = *reinterpret_cast<const words *>(pc + t * 64 + 16 * j);
    const uint32_t w = *reinterpret_cast<const uint32_t *>(ps + t * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) sc[place + j] = w;
  };
  auto turn_b = [](int row) {
    return TRANS ? 2 * ((row ^ (row >> 1)) & 1) | 4 * ((row >> 1) & 1) | (row & 8) : (row >> 1) & 2;
  };
  const int brow = TRANS ? own >> 3 : own;
  // in which order a thread writes its pieces
  const int first = TRANS ? (own >> 2) & 1 : ((own >> 3) ^ (own >> 4)) & 1;
  auto put_b = [&](int slab, int place, int buf) {
    // the loads are waited for here: the compiler would do the selections and
    // shifts below, of all places, where the loads were just issued
    asm volatile("" : "+v"(q[place]), "+v"(sc[place]));
    const int in = TRANS ? -int(slab_row(own >> 3, slab) <= last) : -1;
    const float a = e8m0_arg((TRANS ? sc[place] : sc[place] >> (8 * (place & 3)) & 255u) & uint32_t(in));
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int piece = kWords * (tid % kPer) + (i ^ first);
      const int p = TRANS ? brow * 512 + 16 * ((4 * (own & 7) + piece) ^ turn_b(brow)) : brow * 64 + 16 * (piece ^ turn_b(brow));
      const int c = q[place][i], d = q[place][i ^ 1];
      *reinterpret_cast<uint4 *>(&lb[buf][p]) = mx4_bf16x8(uint32_t((first ? d : c) & in), a);
    }
  };
  // The turns of the rows that a lane reads go by r (and g) alone: one address
  // each, and constants.
  const int b_at = TRANS ? (8 * g + (r >> 2)) * 512 + 8 * (r & 1) : (wn + r) * 64 + 16 * (g ^ turn_b(r));
  const int b_turn = ((r & 3) >> 1) ^ turn_b(8 * g + (r >> 2));
  auto read_b = [&](int buf, int j) {
    if constexpr (TRANS) {
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      i16x4 w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)&lb[buf][b_at + 16 * ((wn / 8 + 2 * j) ^ b_turn) + 2048 * e]);
      const uint2 lo = __builtin_bit_cast(uint2, w[0]), hi = __builtin_bit_cast(uint2, w[1]);
      return make_uint4(lo.x, lo.y, hi.x, hi.y);
    } else {
      return *reinterpret_cast<const uint4 *>(&lb[buf][b_at + 1024 * j]);
    }
  };
  int a_at[AG];
#pragma unroll
  for (int j = 0; j < AG; ++j) a_at[j] = (wm + r) * kARow + 16 * ((4 * j + g) ^ turn(r));
  auto read_a = [&](int buf, int slab, int s, int i) {   // slab: its place among AG
    return *reinterpret_cast<const uint4 *>(&la[buf][s * kABytes + a_at[slab] + 16 * i * kARow]);
  };
  f32x4 acc[MF][NF] = {};
  if (count > 0) {
    // group grp, whose slabs of b are in places p .. p + 3 (the first one in LDS);
    // ahead: later groups of b are loaded
    auto group = [&](int grp, auto p_, auto ahead_) {
      constexpr int p = decltype(p_)::value;
      constexpr bool ahead = decltype(ahead_)::value;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int abuf = (AG < 4 ? j / AG : p / 4) & 1, next = (p + j + 1) & 7;
        if (j % AG == 0) load_a(4 * grp + j + AG, abuf ^ 1);
        uint4 fb[NF];
#pragma unroll
        for (int c = 0; c < NF; ++c) fb[c] = read_b(j & 1, c);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            const uint4 fa = read_a(abuf, j % AG, s, i);
#pragma unroll
            for (int c = 0; c < NF; ++c) acc[i][c] = mfma_bf16(fb[c], fa, acc[i][c]);
          }
        put_b(4 * grp + j + 1, next, (j + 1) & 1);
        if (TRANS && ahead) load_b(4 * grp + j + 9, next);
        else if (ahead && j == 3) load_b4(grp + 2, p);
        // b's next slab is written; and x's next slabs are there, after which
        // only the loads of b, where there are any, were issued
        constexpr int kAfter = !ahead ? 0 : TRANS ? 2 * AG : 5;
        if (j % AG != AG - 1) arrive_lds();
        else if (TRANS || j == 3) arrive<kAfter>();
        else arrive<0>();
      }
    };
    load_a(0, 0);
    if (TRANS) {
#pragma unroll
      for (int j = 0; j < 9; ++j) {
        if (j == 8) put_b(0, 0, 0);
        load_b(j, j & 7);
      }
    } else {
      load_b4(0, 0);
      load_b4(1, 4);
      put_b(0, 0, 0);
    }
    arrive<0>();
    int grp = 0;
    for (; grp + 1 < count; grp += 2) {
      group(grp, std::integral_constant<int, 0>{}, std::true_type{});
      group(grp + 1, std::integral_constant<int, 4>{}, std::true_type{});
    }
    if (grp < count) group(grp, std::integral_constant<int, 0>{}, std::false_type{});
  }
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t row = m0 + wm + 16 * i + r;
    if (row >= m) continue;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      const int64_t c = c0 + wn + 16 * j + 4 * g;
      if (part) store_float4<RSLM_F32>(part + (int64_t(split) * m + row) * cols, c, cols, acc[i][j]);
      else store_float4<TO>(static_cast<typename FloatType<TO>::type *>(out) + row * ostride, c, cols, acc[i][j]);
    }
  }
  // loads that nobody waits for may not write to LDS after its workgroup's end
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Sum of the parts of a split product, always in the same order: 32 adjacent
// values by a workgroup, of which eight groups of threads take every eighth
// part, and the eight sums one after another.
template <int T>
__global__ void __launch_bounds__(256) k_mx4_join(const float *__restrict__ part, int splits, int64_t m, int64_t cols,
                                                  void *__restrict__ out, int64_t stride) {
  __shared__ float sums[8][32];
  const int v = threadIdx.x & 31, k0 = threadIdx.x >> 5;
  const int64_t all = m * cols;
  for (int64_t base = int64_t(blockIdx.x) * 32; base < all; base += int64_t(gridDim.x) * 32) {
    const float *p = part + min(base + v, all - 1);
    float s = 0.f;
#pragma unroll 4
    for (int k = k0; k < splits; k += 8) s += p[k * all];
    sums[k0][v] = s;
    __syncthreads();
    if (threadIdx.x < 32 && base + v < all) {
#pragma unroll
      for (int k = 1; k < 8; ++k) s += sums[k][v];
      const int64_t row = (base + v) / cols;
      store_float<T>(out, row * stride + (base + v - row * cols), s);
    }
    __syncthreads();
  }
}

// The same of few parts and many values: four adjacent ones by a thread.
template <int T>
__global__ void __launch_bounds__(256) k_mx4_join_many(const float *__restrict__ part, int splits, int64_t m, int64_t cols,
                                                       void *__restrict__ out, int64_t stride) {
  const int64_t all = m * cols;
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; at < all; at += int64_t(gridDim.x) * 1024) {
    float s[4] = {};
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
      const float *p = part + k * all + at;
      if (at + 4 <= all) {
        const F32x4u v = *reinterpret_cast<const F32x4u *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += v.v[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i < all) s[i] += p[i];
      }
    }
    int64_t row = at / cols, c = at - row * cols;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at + i < all) store_float<T>(out, row * stride + c, s[i]);
      if (++c == cols) c = 0, ++row;
    }
  }
}

// Which of the two joins, us with the product: the gradient of 2,048 x 32,768 x
// 4,096 bfloat16 (2 parts) 545 by the first, 471 by the second; of 64 x 51,200 x
// 1,024 (100 parts) 37 and 87.
constexpr int64_t kManyValues = 1 << 16;
constexpr int kFewParts = 16;

struct Mx4GemmCall {
  const void *x;
  int64_t m, stride;
  const uint8_t *bc, *bs;
  int64_t n;
  int dim;
  void *out;
  int64_t ostride;
  hipStream_t s;
};

// Workgroups over n values, which stride over more.
static unsigned value_groups(int64_t n) {
  const int64_t g = (n + 255) / 256;
  return unsigned(g < (1 << 20) ? g : (1 << 20));
}

static size_t parts_bytes(int64_t m, int64_t cols, int splits) {
  return splits > 1 ? (size_t(splits) * size_t(m) * size_t(cols) * sizeof(float) + 255) & ~size_t(255) : 0;
}

// Bytes of x's planes, 0 where x can be used as it is.
static size_t planes_bytes(int type, int64_t m, int64_t len) {
  return size_t(type_parts(type)) * size_t(m) * size_t(groups_of(len)) * 256;
}
static bool planes_needed(const void *x, int type, int64_t stride, int64_t len) {
  return type != RSLM_BF16 || len % 128 != 0 || !aligned_to(x, 16) || stride % 8 != 0;
}

template <int TO, int NS, int MF, int WM, int NF, int WN, int AG, bool TRANS>
static void launch_gemm(const Mx4GemmCall &c, const void *xp, int64_t pitch, int64_t plane, int splits, float *part) {
  const int64_t cols = TRANS ? c.dim : c.n, groups = groups_of(TRANS ? c.n : c.dim);
  const int64_t per = (groups + splits - 1) / splits, mt = (c.m + 16 * MF * WM - 1) / (16 * MF * WM);
  const int64_t tiles = (cols + 255) / 256 * mt;
  const dim3 grid(unsigned(tiles * splits));
  hipLaunchKernelGGL((k_mx4_gemm<TO, NS, MF, WM, NF, WN, AG, TRANS>), grid, dim3(64 * WM * WN), 0, c.s,
                     static_cast<const uint8_t *>(xp), c.m, pitch, plane, c.bc, c.bs, c.n, c.dim, mx4_steps(c.dim),
                     c.out, c.ostride, splits > 1 ? part : nullptr, groups, per, int(mt), int(tiles));
  const int64_t values = c.m * cols;
  if (splits > 1 && splits <= kFewParts && values >= kManyValues)
    hipLaunchKernelGGL((k_mx4_join_many<TO>), dim3(value_groups((values + 3) / 4)), dim3(256), 0, c.s, part, splits,
                       c.m, cols, c.out, c.ostride);
  else if (splits > 1)
    hipLaunchKernelGGL((k_mx4_join<TO>), dim3(value_groups(8 * values)), dim3(256), 0, c.s, part, splits, c.m,
                       cols, c.out, c.ostride);
}

// ws: partial sums of the splits, then the planes.
template <int T, int TO, bool TRANS>
static void launch_gemm_rows(const Mx4GemmCall &c, int splits, char *ws) {
  constexpr int NS = Parts<T>::n;
  const int64_t len = TRANS ? c.n : c.dim;
  float *part = reinterpret_cast<float *>(ws);
  const void *xp = c.x;
  int64_t pitch = c.stride * 2, plane = 0;
  if (planes_needed(c.x, T, c.stride, len)) {
    char *planes = ws + parts_bytes(c.m, TRANS ? c.dim : c.n, splits);
    pitch = groups_of(len) * 256;
    plane = c.m * pitch;
    hipLaunchKernelGGL(k_mx4_split<T>, dim3(value_groups(c.m * pitch / 16)), dim3(256), 0, c.s, c.x, c.m, c.stride, len,
                       pitch / 2, reinterpret_cast<uint4 *>(planes));
    xp = planes;
  }
  constexpr int kAG = NS == 1 ? 2 : 1, kSmall = NS == 1 ? 4 : NS == 2 ? 2 : 1;
  switch (tile_rows(T, c.m, TRANS ? c.dim : c.n, len, TRANS)) {
    case 16: launch_gemm<TO, NS, 1, 1, 4, 4, 4, TRANS>(c, xp, pitch, plane, splits, part); break;
    case 32: launch_gemm<TO, NS, 2, 1, 4, 4, 4, TRANS>(c, xp, pitch, plane, splits, part); break;
    case 64: launch_gemm<TO, NS, 4, 1, 4, 4, kSmall, TRANS>(c, xp, pitch, plane, splits, part); break;
    case 128: launch_gemm<TO, NS, 4, 2, 4, 4, kSmall, TRANS>(c, xp, pitch, plane, splits, part); break;
    default: launch_gemm<TO, NS, 4, 4, 8, 2, kAG, TRANS>(c, xp, pitch, plane, splits, part);
  }
}

template <bool TRANS>
static void launch_gemm_types(const Mx4GemmCall &c, int type, int out_type, int splits, void *ws) {
  char *w = static_cast<char *>(ws);
  if (type == RSLM_F32) launch_gemm_rows<RSLM_F32, RSLM_F32, TRANS>(c, splits, w);
  else if (type == RSLM_F16 && out_type == RSLM_F16) launch_gemm_rows<RSLM_F16, RSLM_F16, TRANS>(c, splits, w);
  else if (type == RSLM_F16) launch_gemm_rows<RSLM_F16, RSLM_F32, TRANS>(c, splits, w);
  else if (out_type == RSLM_BF16) launch_gemm_rows<RSLM_BF16, RSLM_BF16, TRANS>(c, splits, w);
  else launch_gemm_rows<RSLM_BF16, RSLM_F32, TRANS>(c, splits, w);
}

template <int T, int TO>
static void launch_score_few(const Mx4GemmCall &c) {
  constexpr int NT = 2;
  const int steps = mx4_steps(c.dim);
  const size_t shm = size_t(Parts<T>::n) * c.m * few_pitch(steps);
  const int64_t tiles = (c.n + 16 * NT - 1) / (16 * NT), most = 256 * (shm > 32768 ? 2 : 4), wgs = (tiles + 3) / 4;
  hipLaunchKernelGGL((k_mx4_score_few<T, TO, NT>), dim3(unsigned(wgs < most ? wgs : most)), dim3(256), shm, c.s, c.x,
                     int(c.m), c.stride, c.bc, c.bs, c.n, c.dim, steps, c.out, c.ostride, tiles);
}
static void launch_score_few_types(const Mx4GemmCall &c, int type, int out_type) {
  if (type == RSLM_F32) launch_score_few<RSLM_F32, RSLM_F32>(c);
  else if (type == RSLM_F16 && out_type == RSLM_F16) launch_score_few<RSLM_F16, RSLM_F16>(c);
  else if (type == RSLM_F16) launch_score_few<RSLM_F16, RSLM_F32>(c);
  else if (out_type == RSLM_BF16) launch_score_few<RSLM_BF16, RSLM_BF16>(c);
  else launch_score_few<RSLM_BF16, RSLM_F32>(c);
}

// What both products ask of their arguments.
static int check_gemm(const void *x, int type, int64_t m, int64_t stride, const uint8_t *bc, const uint8_t *bs,
                      int64_t n, int dim, const void *out, int out_type, int64_t out_stride, int64_t out_cols) {
  if (m < 0 || n < 0 || m > 65535 * 128ll || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim ||
      !float_type_ok(type) || !float_type_ok(out_type) || stride < 0 || (m > 1 && out_stride < out_cols))
    return RSLM_ERR_INVALID_ARG;
  if (out_type != type && out_type != RSLM_F32) return RSLM_ERR_UNSUPPORTED;
  if (m == 0 || out_cols == 0) return RSLM_OK;
  if (!out || !aligned_to(out, float_bytes(out_type))) return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;   // a gradient of zeros
  if (!x || !bc || !bs || !aligned_to(x, float_bytes(type)) || !aligned_to(bc, 16) || !aligned_to(bs, 4))
    return RSLM_ERR_INVALID_ARG;
  return RSLM_OK;
}

// A gradient over no rows.
template <int T>
__global__ void __launch_bounds__(256) k_mx4_zero(int64_t m, int cols, void *out, int64_t stride) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < m * cols; i += int64_t(gridDim.x) * 256)
    store_float<T>(out, i / cols * stride + i % cols, 0.f);
}

}  // namespace rslm

using namespace rslm;

extern "C" {

size_t rslm_mx4_score_workspace(int64_t m, int64_t n, int32_t dim, int32_t dtype) {
  if (m < 1 || n < 1 || m > 65535 * 128ll || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim || !float_type_ok(dtype))
    return 0;
  if (score_few_ok(dtype, m, dim)) return 0;
  return parts_bytes(m, n, sum_splits(dtype, m, n, dim, false)) + planes_bytes(dtype, m, dim);
}

int rslm_mx4_score(const void *x, int32_t dtype, int64_t m, int64_t stride, const uint8_t *codes,
                   const uint8_t *scales, int64_t n, int32_t dim, void *out, int32_t out_dtype, int64_t out_stride,
                   void *ws, size_t ws_bytes, void *stream) {
  const int st = check_gemm(x, dtype, m, stride, codes, scales, n, dim, out, out_dtype, out_stride, n);
  if (st != RSLM_OK || m == 0 || n == 0) return st;
  const Mx4GemmCall c{x, m, stride, codes, scales, n, dim, out, out_stride, as_stream(stream)};
  if (score_few_ok(dtype, m, dim)) {
    launch_score_few_types(c, dtype, out_dtype);
    return check_launch();
  }
  const int splits = sum_splits(dtype, m, n, dim, false);
  const size_t need =
      parts_bytes(m, n, splits) + (planes_needed(x, dtype, stride, dim) ? planes_bytes(dtype, m, dim) : 0);
  if (ws_bytes < need) return RSLM_ERR_WORKSPACE;
  if (need && (!ws || !aligned_to(ws, 16))) return RSLM_ERR_INVALID_ARG;
  launch_gemm_types<false>(c, dtype, out_dtype, splits, ws);
  return check_launch();
}

size_t rslm_mx4_score_backward_workspace(int64_t m, int64_t n, int32_t dim, int32_t dtype) {
  if (m < 1 || n < 1 || m > 65535 * 128ll || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim || !float_type_ok(dtype))
    return 0;
  return parts_bytes(m, dim, sum_splits(dtype, m, dim, n, true)) + planes_bytes(dtype, m, n);
}

int rslm_mx4_score_backward(const void *dout, int32_t dtype, int64_t m, int64_t stride, const uint8_t *codes,
                            const uint8_t *scales, int64_t n, int32_t dim, void *dx, int32_t dx_dtype,
                            int64_t dx_stride, void *ws, size_t ws_bytes, void *stream) {
  const int st = check_gemm(dout, dtype, m, stride, codes, scales, n, dim, dx, dx_dtype, dx_stride, dim);
  if (st != RSLM_OK || m == 0) return st;
  const hipStream_t s = as_stream(stream);
  if (n == 0) {
    const dim3 grid(value_groups(m * dim));
    if (dx_dtype == RSLM_F32) hipLaunchKernelGGL(k_mx4_zero<RSLM_F32>, grid, dim3(256), 0, s, m, dim, dx, dx_stride);
    else hipLaunchKernelGGL(k_mx4_zero<RSLM_F16>, grid, dim3(256), 0, s, m, dim, dx, dx_stride);
    return check_launch();
  }
  const int splits = sum_splits(dtype, m, dim, n, true);
  const size_t need =
      parts_bytes(m, dim, splits) + (planes_needed(dout, dtype, stride, n) ? planes_bytes(dtype, m, n) : 0);
  if (ws_bytes < need) return RSLM_ERR_WORKSPACE;
  if (need && (!ws || !aligned_to(ws, 16))) return RSLM_ERR_INVALID_ARG;
  launch_gemm_types<true>(Mx4GemmCall{dout, m, stride, codes, scales, n, dim, dx, dx_stride, s}, dtype, dx_dtype,
                          splits, ws);
  return check_launch();
}

}  // extern "C"
