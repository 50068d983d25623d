// Quantisation of float rows to MX4 or MX8 rows (mx4_dev.h; the kernels' B is the
// bits of a code), with the rotation of rotate.hip in the same pass where a plan asks
// for it, and back to floats.
//
// Both directions are bound by memory: a row of D float32 is read (4 D bytes)
// and 0.53 D bytes (MX8: 1.03 D) are written, or the reverse.  16 lanes take 128
// coordinates, 8 consecutive ones each: one 16- or 32-byte load, one 4-byte
// word of codes (8-byte for MX8), and the 32 coordinates of a scale are those of four adjacent
// lanes, whose largest magnitude is found by two exchanges inside the quad.  65,536 x 768
// float32, rotated: 67 us to MX4, 58 to 64 to MX8 (4.0 TB/s and more, VALU 83 to 85 % busy); from MX8 to bfloat16 24.
#include "mx4_dev.h"
#include "rows_dev.h"

namespace rslm {

// The largest of the values of the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), kDppQuadXor1, 0xf, 0xf, true)));
  return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), kDppQuadXor2, 0xf, 0xf, true)));
}

// One group of 128 coordinates: lane r of 16 holds coordinates 8 r + i and
// writes their codes; the first lane of each quad writes its scale.
template <int B>
__device__ __forceinline__ void mx_put8(const float (&x)[8], uint8_t *codes, uint8_t *scales, int r) {
  uint32_t top = 0u;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = x[i] + 0.f;   // -0 to +0: the sign of a cancelled sum depends on its order
    top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  }
  top = quad_max(top);
  const uint32_t s = B == 4 ? e8m0_code(top) : e8m0_code8(top);
  if constexpr (B == 4) *reinterpret_cast<uint32_t *>(codes + 4 * r) = mx4_codes8(v, s);
  else *reinterpret_cast<uint2 *>(codes + 8 * r) = mx8_codes8(v, s);
  if ((r & 3) == 0) scales[r >> 2] = uint8_t(s);
}

// A run of `each` groups of 128 coordinates of a row by 16 lanes, four at a time
// in flight; blockIdx.y: which run.  Whole rows where there are many, so that they
// are read on end: 40,001 x 2,049 bfloat16 in 77 us, and in 107 with one group
// to 16 lanes in the order of the columns (back to floats 37 and 52).
constexpr int kFlight = 4;
template <int B, int T>
__global__ void __launch_bounds__(256) k_mx_quantize(const void *__restrict__ x, int64_t n, int dim,
                                                      int64_t stride, int steps, int each,
                                                      uint8_t *__restrict__ codes,
                                                      uint8_t *__restrict__ scales) {
  const int r = threadIdx.x & 15;
  const int t0 = blockIdx.y * each, t1 = min(steps, t0 + each);
  // whole groups of 16 lanes leave together
  for (int64_t row = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); row < n; row += int64_t(gridDim.x) * 16) {
    const typename FloatType<T>::type *xr = static_cast<const typename FloatType<T>::type *>(x) + row * stride;
    for (int t = t0; t < t1; t += kFlight) {
      Raw8<T> raw[kFlight];
#pragma unroll
      for (int u = 0; u < kFlight; ++u) load_raw8<T>(raw[u], xr, 128 * (t + u) + 8 * r, t + u < t1 ? dim : 0);
#pragma unroll
      for (int u = 0; u < kFlight; ++u)
        if (t + u < t1) {
          float v[8];
          raw_values<T>(v, raw[u]);
          mx_put8<B>(v, codes + (row * steps + t + u) * (16 * B), scales + (row * steps + t + u) * 4, r);
        }
    }
  }
}

template <int B, int T>
__global__ void __launch_bounds__(256) k_mx_dequantize(const uint8_t *__restrict__ codes,
                                                        const uint8_t *__restrict__ scales, int64_t n,
                                                        int dim, int steps, int each, void *__restrict__ out,
                                                        int64_t stride) {
  const int r = threadIdx.x & 15;
  const int t0 = blockIdx.y * each, t1 = min(steps, t0 + each);
  for (int64_t row = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); row < n; row += int64_t(gridDim.x) * 16) {
    typename FloatType<T>::type *orow = static_cast<typename FloatType<T>::type *>(out) + row * stride;
    for (int t = t0; t < t1; t += kFlight) {
      if constexpr (T == RSLM_F32) {
        // coordinates 4 r .. + 3 of both halves, so that each of the two stores
        // writes 256 bytes on end: 40,001 x 2,049 125 us and 139 with 8 r .. + 7,
        // 3,000 x 4,096 9.5 and 12.4 (500,000 x 96 40 and 37)
        uint32_t w[kFlight][2], s[kFlight][2];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
          const int64_t g = row * steps + min(t + u, t1 - 1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint8_t *at = codes + g * (16 * B) + (8 * h * B + r * (B / 2));
            w[u][h] = B == 4 ? *reinterpret_cast<const uint16_t *>(at) : *reinterpret_cast<const uint32_t *>(at);
            s[u][h] = scales[g * 4 + 2 * h + (r >> 3)];
          }
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            store_float4<T>(orow, 128 * (t + u) + 64 * h + 4 * r, t + u < t1 ? dim : 0,
                            B == 4 ? mx4_values4(w[u][h], s[u][h]) : mx8_values4(w[u][h], s[u][h]));
      } else {
        uint2 w[kFlight];
        uint32_t s[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
          const int64_t g = row * steps + min(t + u, t1 - 1);
          const uint8_t *at = codes + g * (16 * B) + B * r;
          if constexpr (B == 4) w[u].x = *reinterpret_cast<const uint32_t *>(at);
          else w[u] = *reinterpret_cast<const uint2 *>(at);
          s[u] = scales[g * 4 + (r >> 2)];
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
          float v[8];
          if constexpr (B == 4) mx4_values8(v, w[u].x, s[u]);
          else mx8_values8(v, w[u], s[u]);
          store_float8<T>(v, orow, 128 * (t + u) + 8 * r, t + u < t1 ? dim : 0);
        }
      }
    }
  }
}

__device__ __forceinline__ void load_float8_any(float (&v)[8], const void *row, int c, int dim, int dtype) {
  if (dtype == RSLM_F32) load_float8<RSLM_F32>(v, row, c, dim);
  else if (dtype == RSLM_F16) load_float8<RSLM_F16>(v, row, c, dim);
  else load_float8<RSLM_BF16>(v, row, c, dim);
}

// Rotate and quantise, D >= 128: the rotation runs in registers on 16-lane
// rows (rows_dev.h), whose lanes end with 8 consecutive coordinates of each of
// their blocks, as the quantiser takes them.  Every pass is scaled as it ends,
// so the coordinates, and with them the codes, have the bits of rslm_fwht's.
template <int B, int RPV, int NBR, bool FULL>
__global__ void __launch_bounds__(256, NBR <= 4 ? 4 : 2) k_mx_quantize_rot(
    const void *__restrict__ x, int dtype, int64_t n, int64_t stride, uint8_t *__restrict__ codes,
    uint8_t *__restrict__ scales, RotParams rp) {
  constexpr int VPW = 4 / RPV;
  extern __shared__ float4 lds4[];
  __shared__ __align__(16) uint32_t s1[kSignWords];
  const int D = rp.D, steps = mx4_steps(D);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int vstride = rows_stride(D);
  float *lds = reinterpret_cast<float *>(lds4);
  uint16_t *ts = reinterpret_cast<uint16_t *>(lds + 4 * VPW * vstride);
  RowsTs<128 * RPV * NBR> tload;
  tload.load(rp);
  RowsSigns signs;
  signs.load(rp);
  tload.store(ts, rp, signs, false);
  signs.fill(s1, rp);
  __syncthreads();
  const int64_t n_groups = (n + VPW - 1) / VPW;
  for (int64_t grp = int64_t(blockIdx.x) * 4 + wid; grp < n_groups; grp += int64_t(gridDim.x) * 4) {
    int olane = lane;   // opaque: nothing derived from it is kept across the loop
    asm volatile("" : "+v"(olane));
    const RowsLane<RPV> ln(olane);
    const int64_t row = grp * VPW + ln.vslot;
    if (row >= n) continue;   // the lanes of this vector sit out; no workgroup barrier follows
    float *vb = lds + (wid * VPW + ln.vslot) * vstride;
    const char *xr = static_cast<const char *>(x) + row * stride * float_bytes(dtype);
    float z[8 * NBR];
#pragma unroll
    for (int j = 0; j < NBR; ++j) {
      float v[8];
      load_float8_any(v, xr, 128 * (j * RPV + ln.pv) + 8 * ln.r, D, dtype);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[8 * j + i] = v[i];
    }
#pragma unroll
    for (int j = 0; j < NBR; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = z[8 * j + i];
      rows_flip(v, s1, j * RPV + ln.pv, ln.r);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[8 * j + i] = v[i];
    }
    rows_forward<RPV, NBR, FULL>(z, rp, ts, vb, ln, true);
#pragma unroll
    for (int j = 0; j < NBR; ++j) {
      const int b = j * RPV + ln.pv;
      if (FULL || b < steps) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = z[8 * j + i];
        mx_put8<B>(v, codes + (row * steps + b) * (16 * B), scales + (row * steps + b) * 4, ln.r);
      }
    }
  }
}

constexpr int kDppQuadXor3 = 0x1B;

// The butterflies of the block of B < 128 coordinates 8 r + i: three stages in
// registers, three between lanes (r ^ 1, 2, 4), the last one scaled.  Coordinates
// past B keep what they have.
__device__ __forceinline__ void small_butterflies(float (&v)[8], int r, int B, float inv_sqrt_b) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = v[i];
#pragma unroll
  for (int h = 1; h < 8; h <<= 1) {
    const float scale = 2 * h == B ? inv_sqrt_b : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & h) && h < B) {
        const float a = w[i], c = w[i + h];
        w[i] = (a + c) * scale;
        w[i + h] = (a - c) * scale;
      }
  }
#pragma unroll
  for (int e = 1; e < 8; e <<= 1) {
    const float scale = 16 * e == B ? inv_sqrt_b : 1.f;
    const bool upper = r & e;
    if (8 * e < B) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float o = e == 1   ? dppf<kDppQuadXor1>(w[i])
                        : e == 2 ? dppf<kDppQuadXor2>(w[i])
                                 : dppf<kDppQuadXor3>(dppf<kDppHalfMirror>(w[i]));
        w[i] = (upper ? o - w[i] : w[i] + o) * scale;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 8 * r + i < B ? w[i] : v[i];
}

// Rotate and quantise, D < 128 (one group): 16 lanes to a vector.  B is the
// largest power of two up to D: a block, and one that ends at D where B does not
// divide it, which goes through LDS, as does the permutation between the passes.
// 284,367 x 64 float32: 38 us (2.2 TB/s), 65 at dim 100; 83 with the butterflies in
// LDS too.
template <int BITS>
__global__ void __launch_bounds__(256) k_mx_quantize_rot_small(const void *__restrict__ x, int dtype,
                                                                int64_t n, int64_t stride,
                                                                uint8_t *__restrict__ codes,
                                                                uint8_t *__restrict__ scales,
                                                                RotParams rp) {
  __shared__ __align__(16) float buf[16][132];
  const int D = rp.D, B = rp.B, r = threadIdx.x & 15;
  float *b = buf[threadIdx.x >> 4];
  float sign1[8], sign2[8];
  int from[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int o = 8 * r + i;
    sign1[i] = rp.s1[o];
    sign2[i] = o < D ? rp.s1[(o + 127) & 255] : 0.f;
    from[i] = rp.passes > 1 && o < D ? rp.tsrc[o] : o;
  }
  for (int64_t row = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); row - (threadIdx.x >> 4) < n;
       row += int64_t(gridDim.x) * 16) {
    const bool live = row < n;   // a wavefront's lanes stay together
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (live) load_float8_any(v, static_cast<const char *>(x) + row * stride * float_bytes(dtype), 8 * r, D, dtype);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= sign1[i];
    for (int pass = 0; pass < rp.passes; ++pass) {
      if (pass == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[8 * r + i] = v[i];
        wave_sync_r();
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 8 * r + i < D ? b[from[i]] * sign2[i] : 0.f;
        wave_sync_r();
      }
      small_butterflies(v, r, B, rp.inv_sqrt_b);
      if (rp.overlap) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[8 * r + i] = v[i];
        wave_sync_r();
        float u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = 8 * r + i < B ? b[D - B + 8 * r + i] : 0.f;
        wave_sync_r();
        small_butterflies(u, r, B, rp.inv_sqrt_b);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (8 * r + i < B) b[D - B + 8 * r + i] = u[i];
        wave_sync_r();
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = b[8 * r + i];
        wave_sync_r();
      }
    }
    if (live) mx_put8<BITS>(v, codes + row * (16 * BITS), scales + row * 4, r);
  }
}

// Groups of 128 coordinates of a run: the whole row where that gives the GPU
// 4,096 workgroups, at least four otherwise.
static int groups_each(int64_t n, int steps) {
  const int64_t rows = (n + 15) / 16, runs = (4096 + rows - 1) / rows;
  const int64_t each = (steps + runs - 1) / runs;
  return int(each < kFlight ? kFlight : each);
}

// Workgroups over n rows, 16 rows each; they stride over more rows than a grid
// can count.
static unsigned row_groups(int64_t n) {
  const int64_t g = (n + 15) / 16;
  return unsigned(g < (1 << 20) ? g : (1 << 20));
}

#define RSLM_MX4_TYPES(DTYPE, CALL) \
  switch (DTYPE) {                  \
    case RSLM_F32: CALL(RSLM_F32); break;   \
    case RSLM_F16: CALL(RSLM_F16); break;   \
    default: CALL(RSLM_BF16);               \
  }
struct QuantizeCall {
  const void *x;
  int dtype;
  int64_t n, stride;
  uint8_t *codes, *scales;
  hipStream_t s;
};

template <int B, int RPV, int NBR, bool FULL>
static void launch_quantize_rot_one(const rslm_plan *p, const QuantizeCall &c) {
  const size_t shm = size_t(16 / RPV) * rows_stride(p->rot.D) * 4 + 128 * RPV * NBR * 2;
  constexpr auto kernel = k_mx_quantize_rot<B, RPV, NBR, FULL>;
  const int64_t groups = (c.n + 16 / RPV - 1) / (16 / RPV);
  hipLaunchKernelGGL(kernel, dim3(rows_grid<kernel>(shm, groups)), dim3(256), shm, c.s, c.x, c.dtype,
                     c.n, c.stride, c.codes, c.scales, p->rot);
}

template <int B>
static void launch_quantize_rot(const rslm_plan *p, const QuantizeCall &c) {
  const int D = p->rot.D;
  if (!rows_ok(p->rot)) {
    const unsigned groups = row_groups(c.n);
    hipLaunchKernelGGL(k_mx_quantize_rot_small<B>, dim3(groups < 4096 ? groups : 4096), dim3(256), 0, c.s, c.x,
                       c.dtype, c.n, c.stride, c.codes, c.scales, p->rot);
    return;
  }
#define RSLM_QUANT_ROWS(RPV, NBR)                                              \
  {                                                                            \
    if (rows_only_full(RPV, NBR) || D == 128 * RPV * NBR)                      \
      launch_quantize_rot_one<B, RPV, NBR, true>(p, c);                           \
    else                                                                       \
      launch_quantize_rot_one<B, RPV, NBR, rows_only_full(RPV, NBR)>(p, c);       \
  }
  const int nbt = rows_blocks(p->rot);
  RSLM_ROWS_SWITCH(nbt, D == 384, RSLM_QUANT_ROWS)
#undef RSLM_QUANT_ROWS
}

template <int B>
static int quantize_rows(const rslm_plan *plan, const void *x, int dtype, int64_t n, int dim, int64_t stride,
                         uint8_t *codes, uint8_t *scales, void *stream) {
  if (n < 0 || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim || !float_type_ok(dtype) || stride < 0)
    return RSLM_ERR_INVALID_ARG;
  if (plan && plan->rot.D != dim) return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;
  if (!x || !codes || !scales || !aligned_to(x, float_bytes(dtype)) || !aligned_to(codes, 16) ||
      !aligned_to(scales, 4))
    return RSLM_ERR_INVALID_ARG;
  const hipStream_t s = as_stream(stream);
  if (plan && plan->rot.passes > 0) {
    launch_quantize_rot<B>(plan, QuantizeCall{x, dtype, n, stride, codes, scales, s});
    return check_launch();
  }
  const int steps = mx4_steps(dim), each = groups_each(n, steps);
  const dim3 grid(row_groups(n), unsigned((steps + each - 1) / each));
#define RSLM_QUANT(T)                                                                                             \
  hipLaunchKernelGGL((k_mx_quantize<B, T>), grid, dim3(256), 0, s, x, n, dim, stride, steps, each, codes, scales)
  RSLM_MX4_TYPES(dtype, RSLM_QUANT)
#undef RSLM_QUANT
  return check_launch();
}

template <int B>
static int dequantize_rows(const uint8_t *codes, const uint8_t *scales, int64_t n, int dim, void *out, int dtype,
                           int64_t stride, void *stream) {
  if (n < 0 || n > kMx4MaxRows || dim < 1 || dim > kMx4MaxDim || !float_type_ok(dtype) ||
      (n > 1 && stride < dim))
    return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;
  if (!out || !codes || !scales || !aligned_to(out, float_bytes(dtype)) || !aligned_to(codes, 16) ||
      !aligned_to(scales, 4))
    return RSLM_ERR_INVALID_ARG;
  const hipStream_t s = as_stream(stream);
  const int steps = mx4_steps(dim), each = groups_each(n, steps);
  const dim3 grid(row_groups(n), unsigned((steps + each - 1) / each));
#define RSLM_DEQUANT(T)                                                                                            \
  hipLaunchKernelGGL((k_mx_dequantize<B, T>), grid, dim3(256), 0, s, codes, scales, n, dim, steps, each, out, stride)
  RSLM_MX4_TYPES(dtype, RSLM_DEQUANT)
#undef RSLM_DEQUANT
  return check_launch();
}

}  // namespace rslm

using namespace rslm;

extern "C" {

int rslm_mx4_quantize(const rslm_plan *plan, const void *x, int32_t dtype, int64_t n, int32_t dim,
                      int64_t stride, uint8_t *codes, uint8_t *scales, void *stream) {
  return quantize_rows<4>(plan, x, dtype, n, dim, stride, codes, scales, stream);
}

int rslm_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t n, int32_t dim, void *out,
                        int32_t dtype, int64_t stride, void *stream) {
  return dequantize_rows<4>(codes, scales, n, dim, out, dtype, stride, stream);
}

int rslm_mx8_quantize(const rslm_plan *plan, const void *x, int32_t dtype, int64_t n, int32_t dim,
                      int64_t stride, uint8_t *codes, uint8_t *scales, void *stream) {
  return quantize_rows<8>(plan, x, dtype, n, dim, stride, codes, scales, stream);
}

int rslm_mx8_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t n, int32_t dim, void *out,
                        int32_t dtype, int64_t stride, void *stream) {
  return dequantize_rows<8>(codes, scales, n, dim, out, dtype, stride, stream);
}

}  // extern "C"
