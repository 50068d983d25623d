// Products of MX4 rows with MX4 rows (mx4_dev.h) on the scaled matrix
// instruction v_mfma_scale_f32_16x16x128_f8f6f4: 16 x 16 sums of 128 products of
// 4-bit codes, each lane's 32 products times the two scales that it gives.
//
// A lane l of an operand holds row l % 16 and the 32 coordinates 32 (l / 16)
// .. + 31 of a group of 128: 16 consecutive bytes of codes and one scale, as
// the rows are stored.  The rows of b are the instruction's first operand, so
// that a lane ends with four consecutive columns of one row of the output.
#include "mx4_dev.h"

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
// memory.
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

template <int T>
static void launch_matmul(const Mx4MatmulCall &c) {
  const dim3 grid(unsigned((c.n + 255) / 256), unsigned((c.m + 63) / 64));
  hipLaunchKernelGGL((k_mx4_matmul<T, 4, 4>), grid, dim3(256), 0, c.s, c.ac, c.as, c.m, c.bc, c.bs, c.n,
                     c.steps, c.out, c.stride);
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
