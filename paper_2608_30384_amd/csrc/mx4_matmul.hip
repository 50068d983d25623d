// Products of MX4 rows with MX4 rows (mx4_dev.h) on the scaled matrix
// instruction v_mfma_scale_f32_16x16x128_f8f6f4: 16 x 16 sums of 128 products of
// 4-bit codes, each lane's 32 products times the two scales that it gives.
//
// A lane l of an operand holds row l % 16 and the 32 coordinates 32 (l / 16)
// .. + 31 of a group of 128: 16 consecutive bytes of codes and one scale, as
// the rows are stored.  The rows of b are the instruction's first operand, so
// that a lane ends with four consecutive columns of one row of the output.
#include "mx4_choice.h"
#include "mx4_dev.h"

#include <type_traits>

namespace rslm {

// One lane's part of 16 rows' group: 16 bytes of codes and a scale.
struct Mx4Frag {
  i32x4 q;
  int s;
};
__device__ __forceinline__ Mx4Frag mx4_frag(const uint8_t *codes, const uint8_t *scales, int64_t row, int steps,
                                            int t, int g) {
  const int64_t at = row * steps + t;
  Mx4Frag f;
  f.q = *reinterpret_cast<const i32x4 *>(codes + at * 64 + 16 * g);
  f.s = scales[at * 4 + g];
  return f;
}
__device__ __forceinline__ f32x4 mx4_mfma(const Mx4Frag &a, const Mx4Frag &b, f32x4 c) {
  const i32x8 x = {a.q[0], a.q[1], a.q[2], a.q[3], 0, 0, 0, 0};
  const i32x8 y = {b.q[0], b.q[1], b.q[2], b.q[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, a.s, 0, b.s);
}

// Each wavefront: 16 MT rows of a by 16 NT rows of b, operands straight from
// memory, a group asked for when the one before it has been multiplied.  Bound by that
// chain of loads: 256 x 4,096 x 768 6.5 us, 64 x 4,096 x 4,096 16 a call, of 1 and 2 us of
// bytes.
template <int T, int MT, int NT>
__global__ void __launch_bounds__(256) k_mx4_matmul(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                    int64_t m, const uint8_t *__restrict__ bc,
                                                    const uint8_t *__restrict__ bs, int64_t n, int steps,
                                                    void *__restrict__ out, int64_t stride) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6)) * (16 * NT);
  const int64_t m0 = int64_t(blockIdx.y) * (16 * MT);
  if (n0 >= n) return;
  f32x4 acc[MT][NT] = {};
  for (int t = 0; t < steps; ++t) {
    Mx4Frag a[MT], b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = mx4_frag(ac, as, min(m0 + 16 * i + r, m - 1), steps, t, g);
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = mx4_frag(bc, bs, min(n0 + 16 * j + r, n - 1), steps, t, g);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mx4_mfma(b[j], a[i], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = m0 + 16 * i + r;
    if (row >= m) continue;
    typename FloatType<T>::type *orow = static_cast<typename FloatType<T>::type *>(out) + row * stride;
#pragma unroll
    for (int j = 0; j < NT; ++j) store_float4<T>(orow, n0 + 16 * j + 4 * g, n, acc[i][j]);
  }
}

// ---- large products: tiles in LDS ------------------------------------------
//
// A workgroup of 4 wavefronts takes 32 MF rows of a by 256 of b, each wavefront
// 16 MF by 128, one group of 128 coordinates after another.  The memory unit
// writes the codes to LDS by itself, two groups (a 128-byte line of every row)
// at a time and up to four ahead, a few loads between any two rows of matrix
// instructions; all operands of the next group are read from LDS to a second
// set of registers while this group is multiplied, so that a wavefront, alone
// on its SIMD, does not wait for those; every second group it waits for all loads
// that are out, about two groups old.  8,192 x 32,768 x 4,096 to bfloat16: 611 us, the
// matrix unit 44 % busy.  Scales come four groups at a time.  A row's
// eight 16-byte pieces are exchanged by its number, so that the rows of a read
// fall on different banks; the exchange is in the address that a lane of the
// load gives.  Rows of b are dealt to the fragments so that 16 lanes x 4 write
// 64 consecutive bytes of each row of out.
constexpr int kMmRow = 128;             // bytes of a row's two groups

template <int T, int MF>
__global__ void __launch_bounds__(256, 1) k_mx4_matmul_tile(
    const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as, int64_t m, const uint8_t *__restrict__ bc,
    const uint8_t *__restrict__ bs, int64_t n, int steps, void *__restrict__ out, int64_t stride, int mtiles) {
  constexpr int BM = 32 * MF;
  static_assert(MF == 8 || MF == 4, "the places of reads and loads between the instructions");
  constexpr int LA = BM / 32, LB = kMmN / 32, kLoads = LA + LB;   // loads of a wavefront, 8 rows each
  constexpr int kCodesA = 2 * BM * kMmRow;
  __shared__ __align__(1024) uint8_t la[kCodesA + 2 * kMmN * kMmRow];   // a's, then b's
  uint8_t *const lb = la + kCodesA;
  __shared__ __align__(1024) uint8_t sa[2][BM * 16];
  __shared__ __align__(1024) uint8_t sb[2][kMmN * 16];
  __shared__ __align__(1024) uint8_t none[1024];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the 8 XCDs in turn: each XCD takes a run of tiles, in
  // which those of 8 rows of tiles are neighbours.
  const int tiles = gridDim.x, per = tiles / 8, rest = tiles % 8;
  const int xcd = blockIdx.x % 8, at = blockIdx.x / 8 + xcd * per + min(xcd, rest);
  const int ntiles = tiles / mtiles;
  const int band = at / (8 * ntiles), rows = min(8, mtiles - 8 * band), in = at - band * 8 * ntiles;
  const int64_t m0 = int64_t(8 * band + in % rows) * BM, n0 = int64_t(in / rows) * kMmN;
  const uint32_t cp = 64u * steps, sp = 4u * steps;
  const i32x4 ra = buffer_of(ac + m0 * cp, (m - m0) * cp), rb = buffer_of(bc + n0 * cp, (n - n0) * cp);
  const i32x4 rsa = buffer_of(as + m0 * sp, (m - m0) * sp), rsb = buffer_of(bs + n0 * sp, (n - n0) * sp);
  const uint32_t la0 = lds_address(la), lb0 = lds_address(lb), sa0 = lds_address(sa), sb0 = lds_address(sb),
                 none0 = lds_address(none);
  // Row of b of lane l's part of fragment j: 4-byte results take it as it comes,
  // for 2-byte ones two fragments share out 32 rows, eight to a lane.
  constexpr bool kPair = T != RSLM_F32;
  auto b_row = [&](int l, int j) {
    return kPair ? 32 * (j >> 1) + 8 * (l >> 2) + 4 * (j & 1) + (l & 3) : 16 * j + l;
  };
  // The exchange of a row's pieces, by l % 8 of the lane that reads it: 128-bit
  // reads take their lanes in groups {0..3, 20..23}, {4..7, 16..19}, ..., which
  // get the 64 banks once each.
  auto b_turn = [](int row) { return kPair ? (row & 3) | ((row >> 1) & 4) : row & 7; };
  // a lane of a load: row l / 8 of 8, piece l % 8
  const uint32_t va = (wid * (8 * LA) + (lane >> 3)) * cp + (((lane & 7) ^ (lane >> 3)) << 4);
  uint32_t vb[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    vb[j] = (wid * (8 * LB) + (lane >> 3)) * cp + (((lane & 7) ^ b_turn(8 * j + (lane >> 3))) << 4);
  // load i of groups 2 p and 2 p + 1
  auto load = [&](int p, int i) {
    const int buf = p & 1;
    if (i < LA)
      load_to_lds(ra, la0 + buf * (BM * kMmRow) + (wid * LA + i) * 1024, va + ((8 * i) * cp + p * kMmRow));
    else
      load_to_lds(rb, lb0 + buf * (kMmN * kMmRow) + (wid * LB + i - LA) * 1024,
                  vb[(i - LA) & 1] + ((8 * (i - LA)) * cp + p * kMmRow));
  };
  // The scales of groups 4 q .. 4 q + 3; or, where not `on`, nothing (an offset
  // past the end, and a place that nobody reads: without a branch, the loop
  // stays one block and its instructions in their places).
  auto load_scales = [&](int q, bool on) {
    const uint32_t at = (wid * 64 + lane) * sp + q * 16;
    const bool a_on = on && wid * 64 < BM;
    load_to_lds(rsa, a_on ? sa0 + (q & 1) * (BM * 16) + wid * 1024 : none0, a_on ? at : 0xfffffff0u);
    load_to_lds(rsb, on ? sb0 + (q & 1) * (kMmN * 16) + wid * 1024 : none0, on ? at : 0xfffffff0u);
  };
  const int wm = (wid >> 1) * (16 * MF), wn = (wid & 1) * 128;
  const int ra_off[2] = {(wm + r) * kMmRow + ((g ^ (r & 7)) << 4), (wm + r) * kMmRow + (((4 + g) ^ (r & 7)) << 4)};
  const int rb_row = wn + b_row(r, 0);
  const int rb_off[2] = {rb_row * kMmRow + ((g ^ (r & 7)) << 4), rb_row * kMmRow + (((4 + g) ^ (r & 7)) << 4)};
  const int rsa_off = (wm + r) * 16 + g, rsb_off = rb_row * 16 + g;
  // read i of group st (set: its lowest bit): the fragments of b, then those of a
  Mx4Frag fa[2][MF], fb[2][8];
  auto read = [&](int st, int set, int i) {
    const int buf = (st >> 1) & 1, sbuf = (st >> 2) & 1, by = 4 * (st & 3);
    if (i < 8) {
      const int row = b_row(0, i);
      fb[set][i].q = *reinterpret_cast<const i32x4 *>(&lb[buf * (kMmN * kMmRow) + rb_off[set] + row * kMmRow]);
      fb[set][i].s = sb[sbuf][rsb_off + by + row * 16];
    } else {
      const int row = 16 * (i - 8);
      fa[set][i - 8].q = *reinterpret_cast<const i32x4 *>(&la[buf * (BM * kMmRow) + ra_off[set] + row * kMmRow]);
      fa[set][i - 8].s = sa[sbuf][rsa_off + by + row * 16];
    }
  };
  f32x4 acc[MF][8] = {};
  load_scales(0, true);
#pragma unroll
  for (int p = 0; p < 2; ++p)
    if (2 * p < steps) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(p, i);
    }
  if (steps > 2) arrive<kLoads>();
  else arrive<0>();
#pragma unroll
  for (int i = 0; i < 8 + MF; ++i) read(0, 0, i);
  // Group st, whose operands are in set st & 1.  more: there is a group after
  // it; loads: and a third one.
  auto group = [&](int st, auto set_, auto more_, auto loads_) {
    constexpr int c = decltype(set_)::value;
    constexpr bool more = decltype(more_)::value, loads = decltype(loads_)::value && c == 1;
    // The matrix unit takes an instruction in 4 cycles and works on it for 16:
    // one read or load after each fits in between, several at once do not.
#pragma unroll
    for (int t = 0; t < 8 * MF; ++t) {
      constexpr int each = MF == 8 ? 3 : 1;
      const int k = t / 8, j = t % 8, at = t - 9;
      acc[k][j] = mx4_mfma(fb[c][j], fa[c][k], acc[k][j]);
      if (t == 7 && c == 1 && more) {
        // the next two groups are there; and all have read these two, whose
        // place may be written again
        arrive<0>();
        if (loads) load_scales((st >> 2) + 1, (st & 2) == 0);
      }
      if (more && at >= 0 && at % each == 0 && at / each < 8 + MF) read(st + 1, c ^ 1, at / each);
      if (loads && at >= 1 && (at - 1) % each == 0 && (at - 1) / each < kLoads)
        load((st + 3) >> 1, (at - 1) / each);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const std::integral_constant<int, 0> set0;
  const std::integral_constant<int, 1> set1;
  const std::true_type yes;
  const std::false_type no;
  int st = 0;
  for (; st + 4 < steps; st += 2) {
    group(st, set0, yes, yes);
    group(st + 1, set1, yes, yes);
  }
  if (st + 2 < steps) {
    group(st, set0, yes, no);
    group(st + 1, set1, yes, no);
    st += 2;
  }
  if (st + 1 < steps) {
    group(st, set0, yes, no);
    group(st + 1, set1, no, no);
  } else {
    group(st, set0, no, no);
  }
  // Through LDS, so that a store writes 4 rows of 256 consecutive bytes (f32: 2 of
  // 512), a part of LDS for each wavefront.
  typedef typename FloatType<T>::type Out;
  constexpr int kEach = 16 / sizeof(Out);              // values of a piece
  struct __attribute__((packed, aligned(alignof(Out)))) Wide {
    uint32_t v[4];
  };
  constexpr int kPieces = 128 / kEach;                 // pieces of a row
  constexpr int kOwn = MF == 8 ? 32768 : 16384;
  constexpr int kRows = kOwn / (128 * int(sizeof(Out)));   // rows at a time
  arrive<0>();   // the last operands have been read everywhere
  static_assert(4 * kOwn <= int(sizeof(la)), "LDS of the stores");
  uint8_t *own = la + wid * kOwn;
#pragma unroll
  for (int k0 = 0; k0 < MF; k0 += kRows / 16) {
#pragma unroll
    for (int k = k0; k < k0 + kRows / 16 && k < MF; ++k) {
#pragma unroll
      for (int j = 0; j < 8; j += kPair ? 2 : 1) {
        const int piece = b_row(4 * g, j) / kEach, row = 16 * (k - k0) + r;
        uint4 v;
        if constexpr (kPair) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = uint32_t(float_to_h16<T>(acc[k][j + (i >> 1)][2 * (i & 1)])) |
                   uint32_t(float_to_h16<T>(acc[k][j + (i >> 1)][2 * (i & 1) + 1])) << 16;
          v = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          v = __builtin_bit_cast(uint4, acc[k][j]);
        }
        *reinterpret_cast<uint4 *>(own + row * (128 * sizeof(Out)) + 16 * (piece ^ r)) = v;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wavefront's own part
    constexpr int kAt = 64 / kPieces;                    // rows of a store
#pragma unroll 4
    for (int i = 0; i < kRows / kAt && 16 * k0 + i * kAt < 16 * MF; ++i) {
      const int row = i * kAt + lane / kPieces, piece = lane % kPieces;
      const uint4 v = *reinterpret_cast<const uint4 *>(own + row * (128 * sizeof(Out)) + 16 * (piece ^ (row & 15)));
      const int64_t orow = m0 + wm + 16 * k0 + row, c = n0 + wn + piece * kEach;
      if (orow >= m) continue;
      Out *p = static_cast<Out *>(out) + orow * stride + c;
      if (c + kEach <= n) {   // rows may begin anywhere
        *reinterpret_cast<Wide *>(p) = __builtin_bit_cast(Wide, v);
      } else {
        Out e[kEach];
        __builtin_memcpy(e, &v, 16);
#pragma unroll
        for (int q = 0; q < kEach; ++q)
          if (c + q < n) p[q] = e[q];
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

struct Mx4MatmulCall {
  const uint8_t *ac, *as;
  int64_t m;
  const uint8_t *bc, *bs;
  int64_t n;
  int steps;
  void *out;
  int64_t stride;
  hipStream_t s;
};

template <int T, int MF>
static void launch_matmul_tile(const Mx4MatmulCall &c) {
  const int64_t mt = (c.m + 32 * MF - 1) / (32 * MF), nt = (c.n + kMmN - 1) / kMmN;
  const dim3 grid(unsigned(mt * nt));
  hipLaunchKernelGGL((k_mx4_matmul_tile<T, MF>), grid, dim3(256), 0, c.s, c.ac, c.as, c.m, c.bc, c.bs, c.n, c.steps,
                     c.out, c.stride, int(mt));
}

template <int T, int F>
static void launch_matmul_direct(const Mx4MatmulCall &c) {
  const Mx4DirectGrid g = matmul_direct_grid(c.m, c.n, 16 * F);
  hipLaunchKernelGGL((k_mx4_matmul<T, F, F>), dim3(unsigned(g.x), unsigned(g.y)), dim3(256), 0, c.s, c.ac, c.as, c.m,
                     c.bc, c.bs, c.n, c.steps, c.out, c.stride);
}

template <int T>
static void launch_matmul(const Mx4MatmulCall &c) {
  switch (matmul_form(c.m, c.n)) {
    case kMmTile256: launch_matmul_tile<T, 8>(c); break;
    case kMmTile128: launch_matmul_tile<T, 4>(c); break;
    case kMmDirect64: launch_matmul_direct<T, 4>(c); break;
    case kMmDirect32: launch_matmul_direct<T, 2>(c); break;
    default: launch_matmul_direct<T, 1>(c);
  }
}

}  // namespace rslm

using namespace rslm;

extern "C" {

int rslm_mx4_matmul(const uint8_t *a_codes, const uint8_t *a_scales, int64_t m, const uint8_t *b_codes,
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
  const Mx4MatmulCall c{a_codes, a_scales, m, b_codes, b_scales, n, mx4_steps(dim), out, stride, as_stream(stream)};
  if (dtype == RSLM_F32) launch_matmul<RSLM_F32>(c);
  else if (dtype == RSLM_F16) launch_matmul<RSLM_F16>(c);
  else launch_matmul<RSLM_BF16>(c);
  return check_launch();
}

}  // extern "C"
