// The residual's addition and the root-mean-square norm, to floats and to MX8 rows
// (mx4_dev.h), and its gradient:
//   h = round(x + residual),  rstd = (mean h^2 + eps)^(-1/2),  y = (h rstd) w;
//   dx = dh + rstd (g - n mean(g n)),  g = dy w,  n = h rstd;  dw = sum over rows of dy n.
// Sums are float32; h is rounded to its type first, as the next layer reads it.
//
// Bound by memory: x and the residual are read, h and y (or 1.03 bytes a coordinate of
// codes and scales) are written, once each; backward h, dy and dh are read and dx written.
// us, 8,192 x 4,096 bfloat16: forward 51 (5.2 TB/s), backward with the weight's gradient 45
// (6.0 TB/s, some of it from the last-level cache) and 5; 20,001 x 2,049 float32 to 8 bits
// 107 (5.0 TB/s).  Reading rows twice, and the weight's gradient by a kernel of its own,
// took 82, 162 and 143.
#include "mx4_dev.h"
#include "rows_dev.h"

namespace rslm {

constexpr int kNormThreads = 256;

struct NormArgs {
  const void *x, *residual, *weight;
  int wtype;
  int64_t n;
  int dim;
  int64_t xstride, rstride, hstride, ystride;
  float eps;
  void *h, *y;
  uint8_t *codes, *scales;
  float *rstd;
};

template <int T>
__device__ __forceinline__ const typename FloatType<T>::type *row_of(const void *p, int64_t row, int64_t stride) {
  return static_cast<const typename FloatType<T>::type *>(p) + row * stride;
}
template <int T>
__device__ __forceinline__ typename FloatType<T>::type *row_of(void *p, int64_t row, int64_t stride) {
  return static_cast<typename FloatType<T>::type *>(p) + row * stride;
}

// w[c .. c + 7] of a weight of any type; ones without a weight.
__device__ __forceinline__ void load_weight8(float (&w)[8], const void *p, int type, int c, int dim) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
  } else if (type == RSLM_F32) {
    load_float8<RSLM_F32>(w, p, c, dim);
  } else if (type == RSLM_F16) {
    load_float8<RSLM_F16>(w, p, c, dim);
  } else {
    load_float8<RSLM_BF16>(w, p, c, dim);
  }
}

constexpr int kNormMost = 1024;   // threads of a workgroup

// The sum of the workgroup's v, in every thread; `sums` has a place for each
// wavefront, and is free again after the caller's next barrier.
__device__ __forceinline__ float group_sum(float v, float *sums) {
  const int waves = blockDim.x / 64;
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
  if (threadIdx.x >= waves && threadIdx.x < kNormMost / 64) sums[threadIdx.x] = 0.f;   // sums of four are added
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < waves; i += 4) {
    const float4 v4 = *reinterpret_cast<const float4 *>(sums + i);
    s += (v4.x + v4.y) + (v4.z + v4.w);
  }
  return s;
}

__device__ __forceinline__ uint32_t quad_top(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), kDppQuadXor1, 0xf, 0xf, true)));
  return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x4E, 0xf, 0xf, true)));   // quad_perm [2, 3, 0, 1]
}

// Codes of 8 coordinates, four adjacent lanes having the 32 of a scale.
__device__ __forceinline__ void put_mx8(const float (&v)[8], uint8_t *codes, uint8_t *scales, int chunk) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  const uint32_t s = e8m0_code8(quad_top(top));
  *reinterpret_cast<uint2 *>(codes + 8 * chunk) = mx8_codes8(v, s);
  if ((chunk & 3) == 0) scales[chunk >> 2] = uint8_t(s);
}

// ---- rows held in registers
//
// LANES lanes of a workgroup of 256 to a row, or a workgroup (LANES 0), NV pieces of 8
// coordinates each.  A row's last coordinates are read 8 at a time too, from dim - 8 on, and
// moved to their places: no branch keeps a thread's loads apart.

// One of 8 coordinates from c on: read from `at`, the first `skip` of them another piece's.
struct Piece {
  int c, at, skip;
};
__device__ __forceinline__ Piece piece_at(int c, int dim) {
  const int at = min(c, dim - 8);
  return Piece{c, at, c - at};
}
template <int T>
__device__ __forceinline__ void load_piece(Raw8<T> &p, const typename FloatType<T>::type *row, const Piece &e) {
  if constexpr (T == RSLM_F32) {
    const F32x8u a = *reinterpret_cast<const F32x8u *>(row + e.at);
    __builtin_memcpy(&p, &a, sizeof(a));
  } else {
    const H16x8u a = *reinterpret_cast<const H16x8u *>(row + e.at);
    __builtin_memcpy(&p, &a, sizeof(a));
  }
}
// Coordinates c .. c + 7 of what was read, 0 past dim.
__device__ __forceinline__ void place_piece(float (&v)[8], const Piece &e, bool odd) {
  if (odd) {   // dim % 8, the same for all
#pragma unroll
    for (int by = 1; by < 8; by <<= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = e.skip & by ? (i + by < 8 ? v[i + by] : 0.f) : v[i];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = e.skip >= 8 ? 0.f : v[i];
}
template <int T>
__device__ __forceinline__ void piece_values(float (&v)[8], const Raw8<T> &p, const Piece &e, bool odd) {
  raw_values<T>(v, p);
  place_piece(v, e, odd);
}
__device__ __forceinline__ void piece_weight(float (&w)[8], const void *p, int type, const Piece &e, bool odd) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    return;
  }
  if (type == RSLM_F32) {
    Raw8<RSLM_F32> r;
    load_piece<RSLM_F32>(r, static_cast<const float *>(p), e);
    raw_values<RSLM_F32>(w, r);
  } else if (type == RSLM_F16) {
    Raw8<RSLM_F16> r;
    load_piece<RSLM_F16>(r, static_cast<const _Float16 *>(p), e);
    raw_values<RSLM_F16>(w, r);
  } else {
    Raw8<RSLM_BF16> r;
    load_piece<RSLM_BF16>(r, static_cast<const __bf16 *>(p), e);
    raw_values<RSLM_BF16>(w, r);
  }
  place_piece(w, e, odd);
}

constexpr int norm_rows(int lanes) { return lanes ? kNormThreads / lanes : 1; }          // of a workgroup
constexpr int norm_bound(int lanes) { return lanes ? kNormThreads : kNormMost; }         // its threads
template <int LANES>
__device__ __forceinline__ int norm_lanes() {
  return LANES ? LANES : int(blockDim.x);
}

// The sum over a row's lanes, in each of them.  `sums`: LANES 0 alone, as group_sum.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v, float *sums) {
  if constexpr (LANES == 0) return group_sum(v, sums);
#pragma unroll
  for (int off = LANES / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// 1 / sqrt of the mean of squares and eps, of their sum.  The sum of up to 65,536 = 2^16 of them
// may pass float32 where their mean does not: `again` then gives that of the values' 2^-8ths.
template <class Again>
__device__ __forceinline__ float norm_rstd(float sum, int dim, float eps, Again &&again) {
  float mean = sum / float(dim);
  if (sum == INFINITY) mean = again() / float(dim) * 0x1p16f;   // the same for all of a row's lanes
  return 1.f / sqrtf(mean + eps);
}
constexpr float kNormLess = 0x1p-8f;

template <int T, int LANES, int NV>
__global__ void __launch_bounds__(norm_bound(LANES)) k_norm(NormArgs a) {
  constexpr int R = norm_rows(LANES);
  __shared__ __align__(16) float sums[2][kNormMost / 64];
  const int lanes = norm_lanes<LANES>(), lane = R == 1 ? threadIdx.x : threadIdx.x % lanes;
  const int mine0 = R == 1 ? 0 : threadIdx.x / lanes;
  const int chunks = mx4_steps(a.dim) * 16;
  const bool odd = a.dim & 7;
  Piece e[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) e[u] = piece_at(8 * (lane + lanes * u), a.dim);
  int turn = 0;
  for (int64_t row0 = int64_t(blockIdx.x) * R; row0 < a.n; row0 += int64_t(gridDim.x) * R, turn ^= 1) {
    // past the last row: that one again, without writing
    const int64_t mine = row0 + mine0, row = min(mine, a.n - 1);
    const bool on = mine < a.n;
    Raw8<T> rx[NV], rr[NV];
    const auto *x = row_of<T>(a.x, row, a.xstride);
#pragma unroll
    for (int u = 0; u < NV; ++u) load_piece<T>(rx[u], x, e[u]);
    if (a.residual) {
      const auto *r = row_of<T>(a.residual, row, a.rstride);
#pragma unroll
      for (int u = 0; u < NV; ++u) load_piece<T>(rr[u], r, e[u]);
    }
    float h[NV][8], sum = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      piece_values<T>(h[u], rx[u], e[u], odd);
      if (a.residual) {
        float r[8];
        piece_values<T>(r, rr[u], e[u], odd);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[u][i] = float(typename FloatType<T>::type(h[u][i] + r[i]));
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(h[u][i], h[u][i], sum);
    }
    if (a.residual && on) {
#pragma unroll
      for (int u = 0; u < NV; ++u) store_float8<T>(h[u], row_of<T>(a.h, row, a.hstride), e[u].c, a.dim);
    }
    float w[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) piece_weight(w[u], a.weight, a.wtype, e[u], odd);
    const float rstd = norm_rstd(lanes_sum<LANES>(sum, sums[turn]), a.dim, a.eps, [&] {
      float less = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) less = fmaf(h[u][i] * kNormLess, h[u][i] * kNormLess, less);
      less = lanes_sum<LANES>(less, sums[turn ^ 1]);
      if (LANES == 0) __syncthreads();   // the next row's sums go there
      return less;
    });
    if (lane == 0 && on) a.rstd[row] = rstd;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[u][i] = h[u][i] * rstd * w[u][i] + 0.f;
      if (a.y && on) store_float8<T>(h[u], row_of<T>(a.y, row, a.ystride), e[u].c, a.dim);
      const int k = lane + lanes * u;   // whole quads: chunks is a multiple of 16
      if (a.codes && on && k < chunks) {
        if (e[u].c + 8 > a.dim) {   // 0 past dim, though rstd may be no number
#pragma unroll
          for (int i = 0; i < 8; ++i) h[u][i] = e[u].c + i < a.dim ? h[u][i] : 0.f;
        }
        put_mx8(h[u], a.codes + row * chunks * 8, a.scales + row * (chunks / 4), k);
      }
    }
  }
}

// ---- rows too long for that, or of less than 8 coordinates
//
// A row to a workgroup, which reads it twice (h, written in between, the second time; from
// the cache).
template <int T>
__global__ void __launch_bounds__(kNormMost) k_norm_long(NormArgs a) {
  __shared__ __align__(16) float sums[2][kNormMost / 64];
  const int tid = threadIdx.x, lanes = blockDim.x, chunks = mx4_steps(a.dim) * 16;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const auto *x = row_of<T>(a.x, row, a.xstride);
    float sum = 0.f;
    for (int c = 8 * tid; c < a.dim; c += 8 * lanes) {
      float v[8];
      load_float8<T>(v, x, c, a.dim);
      if (a.residual) {
        float r[8];
        load_float8<T>(r, row_of<T>(a.residual, row, a.rstride), c, a.dim);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float(typename FloatType<T>::type(v[i] + r[i]));
        store_float8<T>(v, row_of<T>(a.h, row, a.hstride), c, a.dim);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
    }
    // a thread reads back what it wrote itself
    const auto *h = a.residual ? row_of<T>(static_cast<const void *>(a.h), row, a.hstride) : x;
    const float rstd = norm_rstd(group_sum(sum, sums[turn]), a.dim, a.eps, [&] {
      float less = 0.f;
      for (int c = 8 * tid; c < a.dim; c += 8 * lanes) {
        float v[8];
        load_float8<T>(v, h, c, a.dim);
#pragma unroll
        for (int i = 0; i < 8; ++i) less = fmaf(v[i] * kNormLess, v[i] * kNormLess, less);
      }
      less = group_sum(less, sums[turn ^ 1]);
      __syncthreads();   // the next row's sums go there
      return less;
    });
    if (tid == 0) a.rstd[row] = rstd;
    if (!a.y && !a.codes) continue;
    for (int k = tid; k < chunks; k += lanes) {
      float v[8], w[8];
      load_float8<T>(v, h, 8 * k, a.dim);
      load_weight8(w, a.weight, a.wtype, 8 * k, a.dim);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 8 * k + i < a.dim ? v[i] * rstd * w[i] + 0.f : 0.f;
      if (a.y) store_float8<T>(v, row_of<T>(a.y, row, a.ystride), 8 * k, a.dim);
      if (a.codes) put_mx8(v, a.codes + row * chunks * 8, a.scales + row * (chunks / 4), k);
    }
  }
}

struct NormBackArgs {
  const void *dy, *h, *weight, *dh;
  int wtype;
  int64_t n;
  int dim;
  int64_t dystride, hstride, dhstride, dxstride;
  const float *rstd;
  void *dx;
  float *partial;   // strips x dim
  int64_t per;      // rows of a strip
};

// Rows of a strip by a workgroup, R at a time, which sums dweight's part in registers.
template <int T, int LANES, int NV>
__global__ void __launch_bounds__(norm_bound(LANES)) k_norm_backward(NormBackArgs a) {
  constexpr int R = norm_rows(LANES);
  // rows of over 8,192, 16 wavefronts, which have 128 registers each: the weight is read for
  // each row and no row ahead (16,384 bfloat16: 4.4 TB/s, with 4 registers, 20 bytes a lane, in
  // scratch memory; with both 3.0)
  constexpr bool HELD = LANES || NV == 1;
  __shared__ __align__(16) float sums[2][kNormMost / 64];
  __shared__ float parts[R > 1 ? kNormThreads * NV * 8 : 1];
  const int lanes = norm_lanes<LANES>(), lane = R == 1 ? threadIdx.x : threadIdx.x % lanes;
  const int mine0 = R == 1 ? 0 : threadIdx.x / lanes;
  const bool odd = a.dim & 7;
  Piece e[NV];
  float w[NV][8], acc[NV][8] = {};
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    e[u] = piece_at(8 * (lane + lanes * u), a.dim);
    if constexpr (HELD) piece_weight(w[u], a.weight, a.wtype, e[u], odd);
  }
  const int64_t r0 = int64_t(blockIdx.x) * a.per, r1 = min(a.n, r0 + a.per);
  Raw8<T> rd[NV], rh[NV], re[NV];
  float rstd = 0.f;
  auto fetch = [&](int64_t row0) {
    const int64_t row = min(row0 + mine0, r1 - 1);
    const auto *d = row_of<T>(a.dy, row, a.dystride), *h = row_of<T>(a.h, row, a.hstride);
#pragma unroll
    for (int u = 0; u < NV; ++u) load_piece<T>(rd[u], d, e[u]);
#pragma unroll
    for (int u = 0; u < NV; ++u) load_piece<T>(rh[u], h, e[u]);
    if (a.dh) {
      const auto *f = row_of<T>(a.dh, row, a.dhstride);
#pragma unroll
      for (int u = 0; u < NV; ++u) load_piece<T>(re[u], f, e[u]);
    }
    rstd = a.rstd[row];
  };
  int turn = 0;
  if (HELD && r0 < r1) fetch(r0);
  for (int64_t row0 = r0; row0 < r1; row0 += R, turn ^= 1) {
    const int64_t row = row0 + mine0;
    const bool on = row < r1;
    if (!HELD) fetch(row0);
    float g[NV][8], n[NV][8], sum = 0.f;
    const float now = rstd;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      float d[8];
      piece_values<T>(d, rd[u], e[u], odd);
      piece_values<T>(n[u], rh[u], e[u], odd);
      if constexpr (!HELD) piece_weight(w[u], a.weight, a.wtype, e[u], odd);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[u][i] *= now;
        if (on) acc[u][i] = fmaf(d[i], n[u][i], acc[u][i]);
        g[u][i] = d[i] * w[u][i];
        sum = fmaf(g[u][i], n[u][i], sum);
      }
    }
    if (a.dx) {
      const float mean = lanes_sum<LANES>(sum, sums[turn]) / float(a.dim);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float f[8] = {};
        if (a.dh) piece_values<T>(f, re[u], e[u], odd);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[u][i] = fmaf(now, fmaf(-n[u][i], mean, g[u][i]), f[i]);
      }
    }
    // the next rows' loads, before this one's stores (which may be to dy, h or dh, but of
    // rows that are done)
    if (HELD && row0 + R < r1) fetch(row0 + R);
    if (a.dx && on) {
#pragma unroll
      for (int u = 0; u < NV; ++u) store_float8<T>(g[u], row_of<T>(a.dx, row, a.dxstride), e[u].c, a.dim);
    }
  }
  if (!a.partial) return;
  float *out = a.partial + int64_t(blockIdx.x) * a.dim;
  if constexpr (R > 1) {
    // the R rows' parts, in their order
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) parts[mine0 * (LANES * NV * 8) + (u * LANES + lane) * 8 + i] = acc[u][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += kNormThreads) {
      float s = parts[c];
#pragma unroll
      for (int r = 1; r < R; ++r) s += parts[r * (LANES * NV * 8) + c];
      out[c] = s;
    }
  } else {
#pragma unroll
    for (int u = 0; u < NV; ++u) store_float8<RSLM_F32>(acc[u], out, e[u].c, a.dim);
  }
}

template <int T>
__global__ void __launch_bounds__(kNormMost) k_norm_backward_long(NormBackArgs a) {
  __shared__ __align__(16) float sums[2][kNormMost / 64];
  const int tid = threadIdx.x, lanes = blockDim.x;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const auto *dy = row_of<T>(a.dy, row, a.dystride), *h = row_of<T>(a.h, row, a.hstride);
    const float rstd = a.rstd[row];
    float sum = 0.f;
    for (int c = 8 * tid; c < a.dim; c += 8 * lanes) {
      float d[8], v[8], w[8];
      load_float8<T>(d, dy, c, a.dim);
      load_float8<T>(v, h, c, a.dim);
      load_weight8(w, a.weight, a.wtype, c, a.dim);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(d[i] * w[i], v[i] * rstd, sum);
    }
    const float mean = group_sum(sum, sums[turn]) / float(a.dim);
    for (int c = 8 * tid; c < a.dim; c += 8 * lanes) {
      float d[8], v[8], w[8], e[8];
      load_float8<T>(d, dy, c, a.dim);
      load_float8<T>(v, h, c, a.dim);
      load_weight8(w, a.weight, a.wtype, c, a.dim);
      if (a.dh) load_float8<T>(e, row_of<T>(a.dh, row, a.dhstride), c, a.dim);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float g = rstd * (d[i] * w[i] - v[i] * rstd * mean);
        d[i] = a.dh ? g + e[i] : g;
      }
      store_float8<T>(d, row_of<T>(a.dx, row, a.dxstride), c, a.dim);
    }
  }
}

// dy n summed over the rows of a strip, 2,048 columns to a workgroup.
template <int T>
__global__ void __launch_bounds__(kNormThreads) k_norm_dweight(NormBackArgs a) {
  const int c = (int(blockIdx.x) * kNormThreads + int(threadIdx.x)) * 8;
  if (c >= a.dim) return;
  const int64_t r0 = int64_t(blockIdx.y) * a.per, r1 = min(a.n, r0 + a.per);
  float acc[8] = {};
  for (int64_t row = r0; row < r1; ++row) {
    float d[8], v[8];
    load_float8<T>(d, row_of<T>(a.dy, row, a.dystride), c, a.dim);
    load_float8<T>(v, row_of<T>(a.h, row, a.hstride), c, a.dim);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = fmaf(d[i], v[i] * rstd, acc[i]);
  }
  store_float8<RSLM_F32>(acc, a.partial + int64_t(blockIdx.y) * a.dim, c, a.dim);
}

// The strips' sums of a column, 32 parts of them to 32 threads, in a fixed order.
__global__ void __launch_bounds__(1024) k_norm_join(const float *__restrict__ partial, int strips, int dim,
                                                    void *__restrict__ dweight, int wtype) {
  __shared__ float sums[32][33];
  const int col = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = int(blockIdx.x) * 32 + col;
  float s = 0.f;
#pragma unroll 8
  for (int i = part; i < strips; i += 32) s += partial[int64_t(i) * dim + min(c, dim - 1)];
  sums[part][col] = s;
  __syncthreads();
  if (part || c >= dim) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += sums[i][col];
  if (wtype == RSLM_F32) store_float<RSLM_F32>(dweight, c, s);
  else if (wtype == RSLM_F16) store_float<RSLM_F16>(dweight, c, s);
  else store_float<RSLM_BF16>(dweight, c, s);
}

constexpr int kNormHeld = 16384;                       // coordinates of a row in registers
constexpr int kNormOne = 4096, kNormBackOne = 8192;    // of one in single pieces

// Strips of the backward pass: as many of its workgroups as 16 wavefronts to a CU make,
// which is what all types' registers allow.  (bfloat16, dx and the weight's gradient: rows of
// 2,049, 5 wavefronts each, 4.0 TB/s with 768 of them, 3.5 with 1,024; of 768 4.4, with half
// as many 4.2.)
static int64_t norm_strips(int64_t n, int dim) {
  const int waves = dim < 8 || dim > kNormHeld ? 8 : dim <= 1024 ? 4 : dim <= kNormBackOne ? (dim + 511) / 512 : (dim + 1023) / 1024;
  const int64_t most = 256 * (16 / waves);
  return n < most ? n : most;
}

// The lanes of a row and its pieces: a row of up to 128 coordinates to 16 lanes, of up to
// 1,024 to a wavefront, of more (or of over 512 where there are few) to a workgroup, of as
// many wavefronts as it fills: of one piece to a lane up to ONE coordinates, else two.
// (Forward, 5,120 bfloat16: 5.5 TB/s; 256 lanes of four pieces 3.2, 640 of one 3.5.)
#define RSLM_NORM_SWITCH(DIM, N, ONE, CALL)                     \
  if ((DIM) <= 128) CALL(16, 1)                                 \
  else if ((DIM) <= 512) CALL(64, 1)                            \
  else if ((DIM) <= 1024 && (N) >= 1024) CALL(64, 2)            \
  else if ((DIM) <= ONE) CALL(0, 1)                             \
  else CALL(0, 2)
// The threads of a workgroup with NV pieces of 8 coordinates each.
static unsigned norm_group(int lanes, int nv, int dim) {
  return lanes ? kNormThreads : unsigned((dim + 8 * nv - 1) / (8 * nv) + 63) / 64 * 64;
}
static unsigned norm_long_group(int dim) { return dim < 8 ? 64u : unsigned(kNormMost); }

template <int T>
static void launch_norm(const NormArgs &a, hipStream_t s) {
  if (a.dim < 8 || a.dim > kNormHeld) {
    const dim3 grid(unsigned(a.n < 65536 ? a.n : 65536));
    hipLaunchKernelGGL(k_norm_long<T>, grid, dim3(norm_long_group(a.dim)), 0, s, a);
    return;
  }
#define RSLM_NORM(LANES, NV)                                                                       \
  {                                                                                                \
    const int64_t wg = (a.n + norm_rows(LANES) - 1) / norm_rows(LANES);                            \
    const dim3 grid(unsigned(wg < 65536 ? wg : 65536));                                            \
    hipLaunchKernelGGL((k_norm<T, LANES, NV>), grid, dim3(norm_group(LANES, NV, a.dim)), 0, s, a); \
  }
  RSLM_NORM_SWITCH(a.dim, a.n, kNormOne, RSLM_NORM)
#undef RSLM_NORM
}

template <int T>
static void launch_norm_backward(const NormBackArgs &b, void *dweight, int dwtype, hipStream_t s) {
  NormBackArgs a = b;
  int64_t strips = norm_strips(a.n, a.dim);
  if (a.n > 0) {
    a.per = (a.n + strips - 1) / strips;
    if (a.dim < 8 || a.dim > kNormHeld) {
      const dim3 grid(unsigned(a.n < 65536 ? a.n : 65536));
      // the weight's gradient first: dx may be dy or h
      if (dweight)
        hipLaunchKernelGGL(k_norm_dweight<T>, dim3(unsigned((a.dim + 2047) / 2048), unsigned(strips)),
                           dim3(kNormThreads), 0, s, a);
      if (a.dx) hipLaunchKernelGGL(k_norm_backward_long<T>, grid, dim3(norm_long_group(a.dim)), 0, s, a);
    } else {
      if (!dweight) a.partial = nullptr;
#define RSLM_NORM(LANES, NV)                                                                       \
  {                                                                                                \
    a.per = (a.per + norm_rows(LANES) - 1) / norm_rows(LANES) * norm_rows(LANES);                  \
    strips = (a.n + a.per - 1) / a.per;                                                            \
    hipLaunchKernelGGL((k_norm_backward<T, LANES, NV>), dim3(unsigned(strips)),                    \
                       dim3(norm_group(LANES, NV, a.dim)), 0, s, a);                               \
  }
      RSLM_NORM_SWITCH(a.dim, a.n, kNormBackOne, RSLM_NORM)
#undef RSLM_NORM
    }
  }
  if (dweight)
    hipLaunchKernelGGL(k_norm_join, dim3(unsigned((a.dim + 31) / 32)), dim3(1024), 0, s, a.partial, int(strips), a.dim,
                       dweight, dwtype);
}

static bool norm_sizes_ok(int64_t n, int dim, int dtype) {
  return n >= 0 && n <= kMx4MaxRows && dim >= 1 && dim <= kMx4MaxDim && float_type_ok(dtype);
}

}  // namespace rslm

using namespace rslm;

extern "C" {

int rslm_rmsnorm(const void *x, int32_t dtype, int64_t n, int32_t dim, int64_t x_stride, const void *residual,
                 int64_t residual_stride, const void *weight, int32_t weight_dtype, float eps, void *h,
                 int64_t h_stride, void *y, int64_t y_stride, uint8_t *codes, uint8_t *scales, float *rstd,
                 void *stream) {
  if (!norm_sizes_ok(n, dim, dtype) || x_stride < 0 || residual_stride < 0 || !(eps > 0.f) || !(eps < INFINITY) ||
      (weight && !float_type_ok(weight_dtype)) || (residual && n > 1 && h_stride < dim) ||
      (y && n > 1 && y_stride < dim) || !codes != !scales)
    return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;
  const int e = float_bytes(dtype);
  if (!x || !rstd || (residual && !h) || !aligned_to(x, e) || !aligned_to(residual, e) || !aligned_to(h, e) ||
      !aligned_to(y, e) || !aligned_to(weight, weight ? float_bytes(weight_dtype) : 1) || !aligned_to(codes, 16) ||
      !aligned_to(scales, 4) || !aligned_to(rstd, 4))
    return RSLM_ERR_INVALID_ARG;
  const NormArgs a{x,        residual, weight, weight_dtype, n, dim,   x_stride, residual_stride, h_stride,
                   y_stride, eps,      h,      y,            codes, scales, rstd};
  const hipStream_t s = as_stream(stream);
  if (dtype == RSLM_F32) launch_norm<RSLM_F32>(a, s);
  else if (dtype == RSLM_F16) launch_norm<RSLM_F16>(a, s);
  else launch_norm<RSLM_BF16>(a, s);
  return check_launch();
}

size_t rslm_rmsnorm_backward_workspace(int64_t n, int32_t dim) {
  if (!norm_sizes_ok(n, dim, RSLM_F32)) return 0;
  return size_t(norm_strips(n, dim)) * dim * sizeof(float);
}

int rslm_rmsnorm_backward(const void *dy, int32_t dtype, int64_t n, int32_t dim, int64_t dy_stride, const void *h,
                          int64_t h_stride, const float *rstd, const void *weight, int32_t weight_dtype,
                          const void *dh, int64_t dh_stride, void *dx, int64_t dx_stride, void *dweight, void *ws,
                          size_t ws_bytes, void *stream) {
  if (!norm_sizes_ok(n, dim, dtype) || dy_stride < 0 || h_stride < 0 || dh_stride < 0 ||
      ((weight || dweight) && !float_type_ok(weight_dtype)) || (dx && n > 1 && dx_stride < dim))
    return RSLM_ERR_INVALID_ARG;
  const int e = float_bytes(dtype), we = weight || dweight ? float_bytes(weight_dtype) : 1;
  if ((n > 0 && (!dy || !h || !rstd)) || !aligned_to(dy, e) || !aligned_to(h, e) || !aligned_to(dh, e) ||
      !aligned_to(dx, e) || !aligned_to(rstd, 4) || !aligned_to(weight, we) || !aligned_to(dweight, we))
    return RSLM_ERR_INVALID_ARG;
  if (dweight && n > 0) {
    if (ws_bytes < rslm_rmsnorm_backward_workspace(n, dim)) return RSLM_ERR_WORKSPACE;
    if (!ws || !aligned_to(ws, 16)) return RSLM_ERR_INVALID_ARG;
  }
  if ((n == 0 || !dx) && !dweight) return RSLM_OK;
  const NormBackArgs a{dy,        h,        weight,    dh,        weight_dtype, n, dim,
                       dy_stride, h_stride, dh_stride, dx_stride, rstd, n > 0 ? dx : nullptr, static_cast<float *>(ws), 0};
  const hipStream_t s = as_stream(stream);
  if (dtype == RSLM_F32) launch_norm_backward<RSLM_F32>(a, dweight, weight_dtype, s);
  else if (dtype == RSLM_F16) launch_norm_backward<RSLM_F16>(a, dweight, weight_dtype, s);
  else launch_norm_backward<RSLM_BF16>(a, dweight, weight_dtype, s);
  return check_launch();
}

}  // extern "C"
