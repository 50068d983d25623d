// Verification of drafted tokens.  Of each sequence, with p_i = softmax(scale z_i) of the
// target's scores and q_i = softmax(draft_scale d_i) of the draft's (without these: all of
// it on the drafted token), drafted token x_i stands while u_i q_i(x_i) < p_i(x_i); the
// token after those that stand is drawn from max(p_i - q_i, 0), or past the last draft
// from p_i: the first j with r_0 + .. + r_j > u_K sum r.
//
// All of it is in float64: at 131,072 entries an error of 1e-7 in the sums would draw
// another token once in some hundred.  An exponential is then a table of 64 entries, a
// polynomial and a scaling.
//
// Bound by one read of the scores, where there are many rows: a first kernel sums them,
// a slice of a row to a workgroup; a second settles which drafts stand (each workgroup
// for itself) and sums r over the slices where it is not p; a third draws.
#include "mx4_dev.h"

namespace rslm {

constexpr int kVfThreads = 256;
constexpr int kVfEach = 16;                         // entries of a thread in a piece
constexpr int kVfPiece = kVfThreads * kVfEach;
constexpr int kVfMaxSlices = 64;                    // a lane of a wavefront to each
constexpr int kVfMaxDrafts = 64;
constexpr double kLn2d = 0.693147180559945309417;

// Sum of 2^(scale log2(e) (v - m)) over a slice, m its largest score; z is NaN where a
// score is NaN or +infinity.
struct VfSum {
  double z;
  float m;
};

struct VerifyArgs {
  const void *target, *draft;
  int64_t tseq, trow, dseq, drow;   // strides, in elements
  int b, k;
  int64_t n;
  const int64_t *tokens;
  const float *uniforms;
  const int32_t *counts;
  double tscale, dscale;            // times 64 log2(e)
  int slices;
  int64_t per;
  VfSum *tsums, *dsums;             // b x (k + 1) x slices, b x k x slices
  double *rsums;                    // b x slices
  int64_t *out;
  int32_t *accepted;
  float *logprob;
};

// 2^(y / 64), y <= 0.  y = i + f with |f| <= 1/2: the table has 2^((i mod 64) / 64), and
// 2^(f / 64) is its Taylor polynomial of degree 4, off by 4e-14 of itself.
__device__ __forceinline__ double exp64(double y, const double *table) {
  constexpr double l = kLn2d / 64;
  constexpr double big = 6755399441055744.0;   // 1.5 2^52: adding it rounds to a whole number
  y = fmax(y, -80000.0);                       // 2^-1250: zero
  const double t = y + big;
  const double f = y - (t - big);
  const int i = int(uint32_t(__builtin_bit_cast(uint64_t, t)));
  double p = fma(f, l * l * l * l / 24, l * l * l / 6);
  p = fma(f, p, l * l / 2);
  p = fma(f, p, l);
  const double e = table[i & 63];
  return ldexp(fma(e, f * p, e), i >> 6);
}
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 64) table[threadIdx.x] = exp2(double(threadIdx.x) / 64);
  __syncthreads();
}
// of a score v beside the largest one m; 0 for -infinity
__device__ __forceinline__ double weight64(float v, double m, double scale, const double *table) {
  return exp64((double(v) - m) * scale, table);
}

__device__ __forceinline__ VfSum vf_join(const VfSum &a, const VfSum &b, double scale, const double *table) {
  const float m = fmaxf(a.m, b.m);
  if (m == -__builtin_inff()) return VfSum{a.z + b.z, m};
  return VfSum{a.z * weight64(a.m, m, scale, table) + b.z * weight64(b.m, m, scale, table), m};
}
__device__ __forceinline__ VfSum vf_join_wave(VfSum s, double scale, const double *table) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const VfSum o{__shfl_xor(s.z, off, 64), __shfl_xor(s.m, off, 64)};
    s = vf_join(s, o, scale, table);
  }
  return s;
}

__device__ __forceinline__ int vf_count(const VerifyArgs &a, int b) {
  return a.counts ? min(max(a.counts[b], 0), a.k) : a.k;
}
template <int T>
__device__ __forceinline__ const typename FloatType<T>::type *target_row(const VerifyArgs &a, int b, int i) {
  return static_cast<const typename FloatType<T>::type *>(a.target) + b * a.tseq + i * a.trow;
}
template <int T>
__device__ __forceinline__ const typename FloatType<T>::type *draft_row(const VerifyArgs &a, int b, int i) {
  return static_cast<const typename FloatType<T>::type *>(a.draft) + b * a.dseq + i * a.drow;
}

// x[j .. j + 7], -infinity at and past end.
template <int T>
__device__ __forceinline__ void load_scores8(Raw8<T> &p, const typename FloatType<T>::type *x, int64_t j, int64_t end) {
  const int64_t left = end - j;
  load_raw8<T>(p, x + (left > 0 ? j : 0), 0, left >= 8 ? 8 : left > 0 ? int(left) : 0);
  if (left < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= left) p.v[i] = typename FloatType<T>::type(-__builtin_inff());
  }
}

template <int T>
__global__ void __launch_bounds__(kVfThreads) k_verify_sums(VerifyArgs a) {
  __shared__ double table[64];
  __shared__ VfSum parts[kVfThreads / 64];
  const int tid = threadIdx.x;
  const int slice = int(blockIdx.x) % a.slices;
  const int64_t row = int64_t(blockIdx.x) / a.slices;
  const int64_t trows = int64_t(a.b) * (a.k + 1);
  const bool draft = row >= trows;
  const int64_t at = draft ? row - trows : row;
  const int each = draft ? a.k : a.k + 1;
  const int b = int(at / each), i = int(at % each);
  // rows past the sequence's last draft are not read
  if (i >= vf_count(a, b) + (draft ? 0 : 1)) return;
  const auto *x = draft ? draft_row<T>(a, b, i) : target_row<T>(a, b, i);
  const double scale = draft ? a.dscale : a.tscale;
  const int64_t j0 = slice * a.per, j1 = min(a.n, j0 + a.per);
  fill_table(table);
  float m = -__builtin_inff();
  double z = 0;
  bool bad = false;
  for (int64_t j = j0; j < j1; j += kVfPiece) {
    Raw8<T> raw[kVfEach / 8];
#pragma unroll
    for (int u = 0; u < kVfEach / 8; ++u) load_scores8<T>(raw[u], x, j + (u * kVfThreads + tid) * 8, j1);
    float v[kVfEach];
    float top = m;
#pragma unroll
    for (int q = 0; q < kVfEach; ++q) {
      v[q] = float(raw[q / 8].v[q % 8]);
      bad |= !(v[q] < __builtin_inff());
      top = fmaxf(top, v[q]);
    }
    if (top > m) {
      if (m > -__builtin_inff()) z *= weight64(m, top, scale, table);
      m = top;
    }
    const double ref = m == -__builtin_inff() ? 0.0 : double(m);
#pragma unroll
    for (int q = 0; q < kVfEach; ++q) z += weight64(v[q], ref, scale, table);
  }
  if (bad) z = __builtin_nan("");
  VfSum s = vf_join_wave(VfSum{z, m}, scale, table);
  if ((tid & 63) == 0) parts[tid >> 6] = s;
  __syncthreads();
  if (tid) return;
#pragma unroll
  for (int w = 1; w < kVfThreads / 64; ++w) s = vf_join(s, parts[w], scale, table);
  (draft ? a.dsums + at * a.slices : a.tsums + at * a.slices)[slice] = s;
}

// What a sequence's drafts come to: how many stand, and of the rows that the next token is
// drawn from their largest scores and sums.
struct Settled {
  int accepted, count;
  VfSum p, q;
};

// By all threads of a workgroup: a wavefront joins a row's slices.
template <int T>
__device__ __forceinline__ void settle(const VerifyArgs &a, int b, const double *table, VfSum (*rows)[kVfMaxDrafts + 1],
                                       Settled &out) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int count = vf_count(a, b);
  for (int r = wid; r < 2 * count + 1; r += kVfThreads / 64) {
    const bool draft = r > count;
    if (draft && !a.draft) break;
    const int i = draft ? r - count - 1 : r;
    const VfSum *sums = draft ? a.dsums + (int64_t(b) * a.k + i) * a.slices : a.tsums + (int64_t(b) * (a.k + 1) + i) * a.slices;
    VfSum s{0.0, -__builtin_inff()};
    if (lane < a.slices) s = sums[lane];
    s = vf_join_wave(s, draft ? a.dscale : a.tscale, table);
    if (lane == 0) rows[draft][i] = s;
  }
  __syncthreads();
  if (wid == 0) {
    bool stands = false;
    if (lane < count) {
      const int64_t x = a.tokens[int64_t(b) * a.k + lane];
      if (x >= 0 && x < a.n) {
        const VfSum p = rows[0][lane], q = rows[1][lane];
        const double px = weight64(float(target_row<T>(a, b, lane)[x]), p.m, a.tscale, table) / p.z;
        const double qx = a.draft ? weight64(float(draft_row<T>(a, b, lane)[x]), q.m, a.dscale, table) / q.z : 1.0;
        stands = double(a.uniforms[int64_t(b) * (a.k + 1) + lane]) * qx < px;
      }
    }
    const int accepted = __ffsll(static_cast<unsigned long long>(~__ballot(stands))) - 1;
    if (lane == 0) {
      const int n = accepted < 0 ? count : min(accepted, count);
      out.accepted = n;
      out.count = count;
      out.p = rows[0][n];
      out.q = rows[1][n < count ? n : 0];
    }
  }
  __syncthreads();
}

// r of an entry, where a draft fell: what p has over q.
struct Over {
  bool drafted;
  int64_t x;   // without the draft's scores: its token
  double pm, pz, qm, qz, ps, qs;
  template <int T>
  __device__ __forceinline__ double of(const VerifyArgs &a, float v, float d, int64_t j, const double *table) const {
#pragma clang fp contract(off)   // of equal p and q nothing is left
    const double p = weight64(v, pm, ps, table) * pz;
    if (!drafted) return p;
    if (!a.draft) return j == x ? 0.0 : p;
    const double r = p - weight64(d, qm, qs, table) * qz;
    return r > 0 ? r : 0.0;
  }
};
__device__ __forceinline__ Over over_of(const VerifyArgs &a, int b, const Settled &s, bool drafted) {
  Over o;
  o.drafted = drafted;
  o.x = drafted && !a.draft ? a.tokens[int64_t(b) * a.k + s.accepted] : -1;
  o.pm = s.p.m, o.pz = 1.0 / s.p.z, o.ps = a.tscale;
  o.qm = s.q.m, o.qz = 1.0 / s.q.z, o.qs = a.dscale;
  return o;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Of each sequence with a draft that fell: r summed over each slice.
template <int T>
__global__ void __launch_bounds__(kVfThreads) k_verify_over(VerifyArgs a) {
  __shared__ double table[64];
  __shared__ VfSum rows[2][kVfMaxDrafts + 1];
  __shared__ Settled st;
  __shared__ double parts[kVfThreads / 64];
  const int tid = threadIdx.x;
  const int slice = int(blockIdx.x) % a.slices, b = int(blockIdx.x / a.slices);
  fill_table(table);
  settle<T>(a, b, table, rows, st);
  if (st.accepted == st.count) return;
  const Over over = over_of(a, b, st, true);
  const auto *x = target_row<T>(a, b, st.accepted);
  const auto *d = a.draft ? draft_row<T>(a, b, st.accepted) : x;
  const int64_t j0 = slice * a.per, j1 = min(a.n, j0 + a.per);
  double sum = 0;
  for (int64_t j = j0; j < j1; j += kVfPiece)
#pragma unroll
    for (int u = 0; u < kVfEach / 8; ++u) {
      const int64_t at = j + (u * kVfThreads + tid) * 8;
      Raw8<T> rp, rq;
      load_scores8<T>(rp, x, at, j1);
      load_scores8<T>(rq, d, at, j1);
#pragma unroll
      for (int q = 0; q < 8; ++q) sum += over.of<T>(a, float(rp.v[q]), float(rq.v[q]), at + q, table);
    }
  sum = wave_sum64(sum);
  if ((tid & 63) == 0) parts[tid >> 6] = sum;
  __syncthreads();
  if (tid) return;
#pragma unroll
  for (int w = 1; w < kVfThreads / 64; ++w) sum += parts[w];
  a.rsums[int64_t(b) * a.slices + slice] = sum;
}

// A workgroup to a sequence: the slice that the drawn token is in, then the token.
template <int T>
__global__ void __launch_bounds__(kVfThreads) k_verify_draw(VerifyArgs a) {
  __shared__ double table[64];
  __shared__ VfSum rows[2][kVfMaxDrafts + 1];
  __shared__ Settled st;
  __shared__ double sums[kVfMaxSlices], waves[kVfThreads / 64];
  __shared__ double want_s, base_s;
  __shared__ int slice_s, drafted_s;
  __shared__ int found_s, last_s;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, b = blockIdx.x;
  fill_table(table);
  settle<T>(a, b, table, rows, st);
  const int n = st.accepted;
  if (tid == 0) found_s = 0x7fffffff, last_s = -1;
  if (wid == 0) {
    double s = 0;
    bool drafted = n < st.count;
    if (drafted) {
      s = lane < a.slices ? a.rsums[int64_t(b) * a.slices + lane] : 0.0;
      drafted = __ballot(s > 0) != 0;   // else p and q are the same
    }
    if (!drafted) {
      s = 0;
      if (lane < a.slices) {
        const VfSum t = a.tsums[(int64_t(b) * (a.k + 1) + n) * a.slices + lane];
        s = t.m == -__builtin_inff() ? t.z : t.z * weight64(t.m, st.p.m, a.tscale, table) / st.p.z;
      }
    }
    sums[lane] = s;
    if (lane == 0) {
      double total = 0;
      for (int i = 0; i < a.slices; ++i) total += sums[i];
      const float u = a.uniforms[int64_t(b) * (a.k + 1) + a.k];
      const double want = double(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f)) * total;
      double c = 0;
      int at = -1, i = 0;
      double base = 0;
      for (; i < a.slices; ++i) {
        if (sums[i] > 0) at = i, base = c;   // the last one with any, should rounding pass them all
        c += sums[i];
        if (c > want) break;
      }
      // NaN, or nothing: no token
      slice_s = total > 0 && total < __builtin_inf() ? at : -1;
      base_s = base;
      want_s = want;
      drafted_s = drafted;
    }
  }
  __syncthreads();
  int token = -1;
  if (slice_s >= 0) {
    const Over over = over_of(a, b, st, drafted_s);
    const auto *x = target_row<T>(a, b, n);
    const auto *d = a.draft && drafted_s ? draft_row<T>(a, b, n) : x;
    const int64_t j0 = slice_s * a.per, j1 = min(a.n, j0 + a.per);
    double base = base_s;
    for (int64_t j = j0; j < j1; j += kVfPiece) {
      // 16 consecutive entries of a thread
      const int64_t at = j + tid * kVfEach;
      double r[kVfEach];
      double sum = 0;
#pragma unroll
      for (int u = 0; u < kVfEach / 8; ++u) {
        Raw8<T> rp, rq;
        load_scores8<T>(rp, x, at + 8 * u, j1);
        load_scores8<T>(rq, d, at + 8 * u, j1);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          r[8 * u + q] = over.of<T>(a, float(rp.v[q]), float(rq.v[q]), at + 8 * u + q, table);
          sum += r[8 * u + q];
        }
      }
      double upto = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(upto, off, 64);
        if (lane >= off) upto += o;
      }
      if (lane == 63) waves[wid] = upto;
      __syncthreads();
      double c = base + (upto - sum);
      for (int w = 0; w < wid; ++w) c += waves[w];
      int found = 0x7fffffff, last = -1;
#pragma unroll
      for (int q = 0; q < kVfEach; ++q) {
        c += r[q];
        if (r[q] > 0) last = int(at) + q;
        if (c > want_s && r[q] > 0 && found == 0x7fffffff) found = int(at) + q;
      }
      if (found != 0x7fffffff) atomicMin(&found_s, found);
      if (last >= 0) atomicMax(&last_s, last);
      __syncthreads();
      if (found_s != 0x7fffffff) break;
      for (int w = 0; w < kVfThreads / 64; ++w) base += waves[w];
      __syncthreads();
    }
    token = found_s != 0x7fffffff ? found_s : last_s;
  }
  for (int i = tid; i <= a.k; i += kVfThreads) {
    const int64_t o = int64_t(b) * (a.k + 1) + i;
    const int64_t t = i < n ? a.tokens[int64_t(b) * a.k + i] : i == n ? int64_t(token) : -1;
    a.out[o] = t;
    if (a.logprob) {
      double lp = 0;
      if (t >= 0) {
        const VfSum p = rows[0][i];
        lp = (double(float(target_row<T>(a, b, i)[t])) - double(p.m)) * (a.tscale * (kLn2d / 64)) - log(p.z);
      }
      a.logprob[o] = float(lp);
    }
  }
  if (tid == 0) a.accepted[b] = n;
}

// Workgroups to fill the GPU, a piece each at least.
static int verify_slices(int64_t rows, int64_t n) {
  const int64_t most = (n + kVfPiece - 1) / kVfPiece;
  int64_t s = (4096 + rows - 1) / rows;
  if (s > most) s = most;
  return int(s < 1 ? 1 : s > kVfMaxSlices ? kVfMaxSlices : s);
}
static int64_t verify_rows(int b, int k, bool draft) { return int64_t(b) * (k + 1 + (draft ? k : 0)); }

static bool verify_sizes_ok(int64_t b, int k, int64_t n) {
  return b >= 0 && k >= 0 && k <= kVfMaxDrafts && n >= 1 && n <= 0x7fffffff - 2 * kVfPiece &&
         b * (2 * k + 1) <= 0x7fffffff / kVfThreads;   // a grid counts its threads in 32 bits
}

static size_t verify_bytes(int64_t b, int k, bool draft, int slices) {
  return size_t(verify_rows(int(b), k, draft)) * slices * sizeof(VfSum) + size_t(b) * slices * sizeof(double);
}

template <int T>
static void launch_verify(const VerifyArgs &a, hipStream_t s) {
  const dim3 threads(kVfThreads);
  hipLaunchKernelGGL(k_verify_sums<T>, dim3(unsigned(verify_rows(a.b, a.k, a.draft != nullptr) * a.slices)), threads, 0,
                     s, a);
  if (a.k > 0) hipLaunchKernelGGL(k_verify_over<T>, dim3(unsigned(a.b) * a.slices), threads, 0, s, a);
  hipLaunchKernelGGL(k_verify_draw<T>, dim3(unsigned(a.b)), threads, 0, s, a);
}

}  // namespace rslm

using namespace rslm;

extern "C" {

size_t rslm_verify_workspace(int64_t b, int32_t k, int64_t n, int32_t draft) {
  if (!verify_sizes_ok(b, k, n) || b == 0) return 0;
  return verify_bytes(b, k, draft != 0, verify_slices(verify_rows(int(b), k, draft != 0), n));
}

int rslm_verify(const void *target, int32_t dtype, int64_t b, int32_t k, int64_t n, int64_t target_seq_stride,
                int64_t target_stride, float scale, const void *draft, int64_t draft_seq_stride, int64_t draft_stride,
                float draft_scale, const int64_t *tokens, const float *uniforms, const int32_t *counts,
                int64_t *out_tokens, int32_t *accepted, float *logprob, void *ws, size_t ws_bytes, void *stream) {
  if (!verify_sizes_ok(b, k, n) || !float_type_ok(dtype) || target_seq_stride < 0 || target_stride < 0 ||
      !(scale > 0.f && scale <= 0x1p127f) ||
      (draft && (draft_seq_stride < 0 || draft_stride < 0 || !(draft_scale > 0.f && draft_scale <= 0x1p127f))))
    return RSLM_ERR_INVALID_ARG;
  if (b == 0) return RSLM_OK;
  const int e = float_bytes(dtype);
  if (!target || !uniforms || !out_tokens || !accepted || (k > 0 && !tokens) || !aligned_to(target, e) ||
      !aligned_to(draft, e) || !aligned_to(tokens, 8) || !aligned_to(uniforms, 4) || !aligned_to(counts, 4) ||
      !aligned_to(out_tokens, 8) || !aligned_to(accepted, 4) || !aligned_to(logprob, 4))
    return RSLM_ERR_INVALID_ARG;
  if (k == 0) draft = nullptr;
  const bool with = draft != nullptr;
  if (ws_bytes < rslm_verify_workspace(b, k, n, with)) return RSLM_ERR_WORKSPACE;
  if (!ws || !aligned_to(ws, 16)) return RSLM_ERR_INVALID_ARG;
  const double unit = 64 * 1.442695040888963407360;
  VerifyArgs a{target, draft,  target_seq_stride, target_stride,  draft_seq_stride,
               draft_stride, int(b), k, n, tokens, uniforms, counts, double(scale) * unit,
               with ? double(draft_scale) * unit : 1.0};
  a.slices = verify_slices(verify_rows(a.b, k, with), n);
  a.per = (n + int64_t(a.slices) * kVfPiece - 1) / (int64_t(a.slices) * kVfPiece) * kVfPiece;
  a.tsums = static_cast<VfSum *>(ws);
  a.dsums = a.tsums + size_t(b) * (k + 1) * a.slices;
  a.rsums = reinterpret_cast<double *>(a.tsums + size_t(verify_rows(a.b, k, with)) * a.slices);
  a.out = out_tokens;
  a.accepted = accepted;
  a.logprob = logprob;
  const hipStream_t s = as_stream(stream);
  if (dtype == RSLM_F32) launch_verify<RSLM_F32>(a, s);
  else if (dtype == RSLM_F16) launch_verify<RSLM_F16>(a, s);
  else launch_verify<RSLM_BF16>(a, s);
  return check_launch();
}

}  // extern "C"
