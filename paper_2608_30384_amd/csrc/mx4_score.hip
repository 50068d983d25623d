// Products of float rows with MX4 rows, and their gradient:
//   score    out[i][j] = sum_d x[i][d] b[j][d]
//   gradient dx[i][d]  = sum_j dout[i][j] b[j][d]
// on the bfloat16 matrix cores, without rounding an operand: every MX4 value is
// a bfloat16 (v_cvt_scalef32_pk_bf16_fp4), and a float is the sum of 1 (bfloat16),
// 2 (float16) or 3 (float32) bfloat16 parts, cut off the top of its significand
// one after the other.  The products of the parts are exact in the matrix
// cores' float32, so the result has the error of a float32 sum.
#include "mx4_dev.h"

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

constexpr int kTileN = 128, kTileK = 64;

// out tile of BM rows of x by 128 columns, 256 threads, over the contracted
// range [k0, k1) in pieces of 64: both operands in LDS as bfloat16, the parts
// of x in planes.  TRANS false: columns are rows of b, contracted over their
// coordinates.  TRANS true: columns are coordinates, contracted over the rows of
// b, which the matrix operand needs across the rows as they are stored: read
// from LDS through the transposing 64-bit loads (lane i of 16 gives the address
// of row i / 4, columns 4 (i % 4) .. + 3, and takes column i of the four rows).
// Rows are split into 16-byte pieces whose places are exchanged by the row's
// number, so that the lanes of a read fall on different banks.
template <int T, int TO, int BM, bool TRANS>
__global__ void __launch_bounds__(256) k_mx4_gemm(const void *__restrict__ x, int64_t m, int64_t stride,
                                                  const uint8_t *__restrict__ bc,
                                                  const uint8_t *__restrict__ bs, int64_t n, int dim, int steps,
                                                  void *__restrict__ out, int64_t ostride,
                                                  float *__restrict__ part, int64_t per) {
  constexpr int NS = Parts<T>::n;
  constexpr int WM = BM >= 128 ? 2 : 1, WN = 4 / WM;         // wavefronts
  constexpr int MF = BM / WM / 16, NF = kTileN / WN / 16;    // fragments of a wavefront
  constexpr int kLoads = BM * kTileK / 8 / 256 > 0 ? BM * kTileK / 8 / 256 : 1;
  __shared__ uint4 xa[NS][BM * 8];
  __shared__ uint4 xb[kTileN * 8];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, r = lane & 15, g = lane >> 4;
  const int64_t cols = TRANS ? dim : n, len = TRANS ? n : dim;
  const int64_t c0 = int64_t(blockIdx.x) * kTileN, m0 = int64_t(blockIdx.y) * BM;
  const int64_t k0 = int64_t(blockIdx.z) * per, k1 = min(len, k0 + per);
  const int wm = (wid / WN) * (MF * 16), wn = (wid % WN) * (NF * 16);
  f32x4 acc[MF][NF] = {};
  for (int64_t k = k0; k < k1; k += kTileK) {
    // x: 8 values of a row by a thread
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = tid + 256 * u, row = i >> 3, c = i & 7;
      if (BM * 8 >= 256 || i < BM * 8) {
        float v[8];
        const int64_t at = m0 + row < m ? k1 - k - 8 * c : 0;   // values left of the row
        load_float8<T>(v, static_cast<const char *>(x) + ((m0 + row) * stride + k + 8 * c) * (T == RSLM_F32 ? 4 : 2),
                       0, int(at < 0 ? 0 : at > 8 ? 8 : at));
        uint4 p[NS];
        split8<NS>(p, v);
#pragma unroll
        for (int s = 0; s < NS; ++s) xa[s][row * 8 + (c ^ (row & 7))] = p[s];
      }
    }
    // b: the 32 codes of a scale by a thread
    {
      const int row = TRANS ? tid >> 2 : tid >> 1, blk = TRANS ? tid & 3 : tid & 1;
      int64_t at;
      bool in = true;
      if (TRANS) {
        in = k + row < k1;
        at = (min(k + row, n - 1) * steps + blockIdx.x) * 4 + blk;
      } else {
        at = min(c0 + row, n - 1) * steps * 4 + k / 32 + blk;
      }
      i32x4 q = *reinterpret_cast<const i32x4 *>(bc + at * 16);
      uint32_t s = bs[at];
      if (!in) q = i32x4{0, 0, 0, 0}, s = 0u;
      const float a = e8m0_arg(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 w = mx4_bf16x8(uint32_t(q[i]), a);
        if (TRANS) xb[row * 16 + ((4 * blk + i) ^ (2 * (row & 7)))] = w;
        else xb[row * 8 + ((4 * blk + i) ^ (row & 7))] = w;
      }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 fb[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        if constexpr (TRANS) {
          // rows 32 h + 8 g + (0..3) and + 4, columns wn + 16 j
          typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
          i16x4 w[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = 32 * h + 8 * g + 4 * e + (r >> 2);
            const int piece = (wn + 16 * j) / 8 + ((r & 3) >> 1);
            const char *p = reinterpret_cast<const char *>(xb) + (row * 16 + (piece ^ (2 * (row & 7)))) * 16 + 8 * (r & 1);
            w[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p);
          }
          const uint2 lo = __builtin_bit_cast(uint2, w[0]), hi = __builtin_bit_cast(uint2, w[1]);
          fb[j] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        } else {
          const int row = wn + 16 * j + r;
          fb[j] = xb[row * 8 + ((4 * h + g) ^ (row & 7))];
        }
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        const int row = wm + 16 * i + r;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const uint4 fa = xa[s][row * 8 + ((4 * h + g) ^ (row & 7))];
#pragma unroll
          for (int j = 0; j < NF; ++j) acc[i][j] = mfma_bf16(fb[j], fa, acc[i][j]);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t row = m0 + wm + 16 * i + r;
    if (row >= m) continue;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      const int64_t c = c0 + wn + 16 * j + 4 * g;
      if (part) store_float4<RSLM_F32>(part + (int64_t(blockIdx.z) * m + row) * cols, c, cols, acc[i][j]);
      else store_float4<TO>(static_cast<typename FloatType<TO>::type *>(out) + row * ostride, c, cols, acc[i][j]);
    }
  }
}

// Sum of the parts of a split product, in the order of the parts.
template <int T>
__global__ void __launch_bounds__(256) k_mx4_join(const float *__restrict__ part, int splits, int64_t m, int cols,
                                                  void *__restrict__ out, int64_t stride) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < m * cols; i += int64_t(gridDim.x) * 256) {
    float s = 0.f;
    for (int k = 0; k < splits; ++k) s += part[int64_t(k) * m * cols + i];
    const int64_t row = i / cols;
    store_float<T>(out, row * stride + (i - row * cols), s);
  }
}

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

// Rows of x in a workgroup's tile.
static int tile_rows(int64_t m) { return m <= 16 ? 16 : m <= 64 ? 64 : 128; }

// Parts into which the gradient's sum over the rows of b is split: enough
// workgroups for the GPU, at least 256 rows each.
static int backward_splits(int64_t m, int64_t n, int dim) {
  const int bm = tile_rows(m);
  const int64_t tiles = int64_t(mx4_steps(dim)) * ((m + bm - 1) / bm);
  const int64_t want = (1024 + tiles - 1) / tiles, most = (n + 255) / 256;
  return int(want < most ? want : most < 1 ? 1 : most);
}

template <int T, int TO, int BM, bool TRANS>
static void launch_gemm(const Mx4GemmCall &c, int splits, float *part) {
  const int64_t cols = TRANS ? c.dim : c.n, len = TRANS ? c.n : c.dim;
  const int64_t per = (len + int64_t(splits) * kTileK - 1) / (int64_t(splits) * kTileK) * kTileK;
  const dim3 grid(unsigned((cols + kTileN - 1) / kTileN), unsigned((c.m + BM - 1) / BM), unsigned(splits));
  hipLaunchKernelGGL((k_mx4_gemm<T, TO, BM, TRANS>), grid, dim3(256), 0, c.s, c.x, c.m, c.stride, c.bc, c.bs, c.n,
                     c.dim, mx4_steps(c.dim), c.out, c.ostride, splits > 1 ? part : nullptr, per);
  if (splits > 1)
    hipLaunchKernelGGL((k_mx4_join<TO>), dim3(value_groups(c.m * cols)), dim3(256), 0, c.s, part, splits,
                       c.m, int(cols), c.out, c.ostride);
}

template <bool TRANS>
static void launch_gemm_types(const Mx4GemmCall &c, int type, int out_type, int splits, float *part) {
#define RSLM_GEMM(T, TO)                                                  \
  switch (tile_rows(c.m)) {                                               \
    case 16: launch_gemm<T, TO, 16, TRANS>(c, splits, part); break;       \
    case 64: launch_gemm<T, TO, 64, TRANS>(c, splits, part); break;       \
    default: launch_gemm<T, TO, 128, TRANS>(c, splits, part);             \
  }
  if (type == RSLM_F32) RSLM_GEMM(RSLM_F32, RSLM_F32)
  else if (type == RSLM_F16 && out_type == RSLM_F16) RSLM_GEMM(RSLM_F16, RSLM_F16)
  else if (type == RSLM_F16) RSLM_GEMM(RSLM_F16, RSLM_F32)
  else if (out_type == RSLM_BF16) RSLM_GEMM(RSLM_BF16, RSLM_BF16)
  else RSLM_GEMM(RSLM_BF16, RSLM_F32)
#undef RSLM_GEMM
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

int rslm_mx4_score(const void *x, int32_t dtype, int64_t m, int64_t stride, const uint8_t *codes,
                   const uint8_t *scales, int64_t n, int32_t dim, void *out, int32_t out_dtype, int64_t out_stride,
                   void *stream) {
  const int st = check_gemm(x, dtype, m, stride, codes, scales, n, dim, out, out_dtype, out_stride, n);
  if (st != RSLM_OK || m == 0 || n == 0) return st;
  launch_gemm_types<false>(Mx4GemmCall{x, m, stride, codes, scales, n, dim, out, out_stride, as_stream(stream)},
                           dtype, out_dtype, 1, nullptr);
  return check_launch();
}

size_t rslm_mx4_score_backward_workspace(int64_t m, int64_t n, int32_t dim) {
  if (m < 1 || n < 1 || m > 65535 * 128ll || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim) return 0;
  const int splits = backward_splits(m, n, dim);
  return splits > 1 ? size_t(splits) * size_t(m) * size_t(dim) * sizeof(float) : 0;
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
  if (ws_bytes < rslm_mx4_score_backward_workspace(m, n, dim)) return RSLM_ERR_WORKSPACE;
  const int splits = backward_splits(m, n, dim);
  if (splits > 1 && (!ws || !aligned_to(ws, 16))) return RSLM_ERR_INVALID_ARG;
  launch_gemm_types<true>(Mx4GemmCall{dout, m, stride, codes, scales, n, dim, dx, dx_stride, s}, dtype, dx_dtype,
                          splits, static_cast<float *>(ws));
  return check_launch();
}

}  // extern "C"
