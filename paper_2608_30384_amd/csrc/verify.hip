// Verification of drafted tokens.  Of each sequence, with p_i = softmax(scale z_i) of the
// target's scores and q_i = softmax(draft_scale d_i) of the draft's (without these: all of
// it on the drafted token), drafted token x_i stands while u_i q_i(x_i) < p_i(x_i); the
// token after those that stand is drawn from max(p_i - q_i, 0), or past the last draft
// from p_i: the first j with r_0 + .. + r_j > u_K sum r.
//
// All of it is in float64: at 131,072 entries an error of 1e-7 in the sums would draw
// another token once in some hundred.  An exponential is then a table of 256 entries, a
// polynomial of degree 3 and a scaling, some 16 instructions, which bound the first kernel
// where there are many rows.
//
// Two kernels.  The first sums the exponentials of every row, a slice of 1,024 entries (more
// where a row has over 262,144) at a time to a wavefront.  In the second each workgroup of a
// sequence settles which drafts stand, and where one falls sums r over its slices; the last
// one to have done so draws.  64 sequences of 4 drafts by 131,072 bfloat16 scores: 35 and 26
// us (a kernel of its own for the draw: 17 and 9); one, of float32: 4.8 and 11.6 (5.4 and 8.3,
// and a launch), chains of dependent reads.
#include "mx4_dev.h"

namespace rslm {

constexpr int kVfThreads = 256;
constexpr int kVfWaves = kVfThreads / 64;
constexpr int kVfEach = 16;                         // entries of a lane in a block
constexpr int kVfBlock = 64 * kVfEach;
constexpr int kVfMaxSlices = 256;
constexpr int kVfMaxDrafts = 64;
constexpr double kLn2d = 0.693147180559945309417;

// 2^(i / 256).
struct VfTable {
  double v[256];
};
constexpr VfTable vf_table() {
  VfTable t{};
  for (int i = 0; i < 256; ++i) {
    const double x = kLn2d * i / 256;
    double e = 1;
    for (int k = 24; k > 0; --k) e = 1 + e * x / k;   // the exponential's series
    t.v[i] = e;
  }
  return t;
}
__device__ const VfTable kVfTable = vf_table();

// A sum of weights 2^((v - top) scale / 256) of scores v, `top` the largest; z is NaN where
// a score is NaN or +infinity.  (With v scale - top scale in one fused step a score of 1e20
// and more would not be 0 beside itself.)
struct VfSum {
  double z, top;
};

// What a sequence's drafts come to: how many stand, and of the rows that the next token is
// drawn from their sums.
struct Settled {
  int accepted, count;
  VfSum p, q;
};

struct VerifyArgs {
  const void *target, *draft;
  int64_t tseq, trow, dseq, drow;   // strides, in elements
  int b, k;
  int64_t n;
  const int64_t *tokens;
  const float *uniforms;
  const int32_t *counts;
  double tscale, dscale;            // times 256 log2(e)
  int slices, blocks;               // of a row; blocks of a slice
  int each, groups;                 // slices of a wavefront, workgroups of a row, in the first kernel
  int oeach, ogroups;               // and of a sequence in the second
  VfSum *tsums, *dsums;             // b x (k + 1) x slices, b x k x slices
  double *rsums;                    // b x slices
  int *done;                        // b: workgroups that have written their rsums
  int64_t *out;
  int32_t *accepted;
  float *logprob;
};

// 2^(y / 256), y <= 0, as a product.  y = i + f with |f| <= 1/2: the table has
// 2^((i mod 256) / 256), and 2^(f / 256) is its Taylor polynomial of degree 3, off by 1.4e-13
// of itself.  0 for -infinity (and NaN).
struct Factors {
  double e, q;
};
__device__ __forceinline__ Factors factors256(double y, const double *table) {
  constexpr double l = kLn2d / 256;
  constexpr double big = 6755399441055744.0;   // 1.5 2^52: adding it rounds to a whole number
  y = fmax(y, -320000.0);                      // 2^-1250: zero
  const double t = y + big;
  const double f = y - (t - big);
  const int i = int(uint32_t(__builtin_bit_cast(uint64_t, t)));
  return Factors{ldexp(table[i & 255], i >> 8), fma(f, fma(f, fma(f, l * l * l / 6, l * l / 2), l), 1.0)};
}
__device__ __forceinline__ double exp256(double y, const double *table) {
  const Factors p = factors256(y, table);
  return p.e * p.q;
}
__device__ __forceinline__ double weight64(float v, double top, double scale, const double *table) {
  return exp256((double(v) - top) * scale, table);
}
// Without a barrier: that is the caller's.
__device__ __forceinline__ void fill_table(double *table) { table[threadIdx.x] = kVfTable.v[threadIdx.x]; }

// v of the lane R behind, round each 16 lanes.
template <int R>
__device__ __forceinline__ float row_turn(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x120 + R, 0xf, 0xf, true));   // row_ror
}
template <int R>
__device__ __forceinline__ double row_turn(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_mov_dpp(int(uint32_t(u)), 0x120 + R, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp(int(uint32_t(u >> 32)), 0x120 + R, 0xf, 0xf, true);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_sum64(double v) {
  v += row_turn<8>(v);
  v += row_turn<4>(v);
  v += row_turn<2>(v);
  v += row_turn<1>(v);
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
__device__ __forceinline__ float wave_max32(float v) {
  v = fmaxf(v, row_turn<8>(v));
  v = fmaxf(v, row_turn<4>(v));
  v = fmaxf(v, row_turn<2>(v));
  v = fmaxf(v, row_turn<1>(v));
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmax(v, __shfl_xor(v, off, 64));
  return v;
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

// A lane's entries of the block at j, as they are stored: 8 at 8 lane, 8 at 512 + 8 lane;
// -infinity at and past end, which the block may be behind.
template <int T>
struct VfRaw {
  Raw8<T> v[kVfEach / 8];
};
template <int T>
__device__ __forceinline__ void load_block(VfRaw<T> &p, const typename FloatType<T>::type *x, int64_t j, int64_t end) {
  typedef typename FloatType<T>::type F;
  const int lane = threadIdx.x & 63;
  if (j + kVfBlock <= end) {   // the same for all lanes: no branch keeps the loads apart
#pragma unroll
    for (int u = 0; u < kVfEach / 8; ++u) load_raw8<T>(p.v[u], x + j + u * 512 + 8 * lane, 0, 8);
  } else {
#pragma unroll
    for (int u = 0; u < kVfEach / 8; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t at = j + u * 512 + 8 * lane + i;
        const F e = x[min(at, end - 1)];
        p.v[u].v[i] = at < end ? e : F(-__builtin_inff());
      }
  }
}

template <int T>
__global__ void __launch_bounds__(kVfThreads) k_verify_sums(VerifyArgs a) {
  __shared__ double table[256];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = int64_t(blockIdx.x) / a.groups, trows = int64_t(a.b) * (a.k + 1);
  const bool draft = row >= trows;
  const int64_t at = draft ? row - trows : row;
  const int b = int(at / (draft ? a.k : a.k + 1)), i = int(at - int64_t(b) * (draft ? a.k : a.k + 1));
  if (at == int64_t(b) * (a.k + 1) && !draft && int(blockIdx.x) % a.groups == 0 && threadIdx.x == 0) a.done[b] = 0;
  // rows past the sequence's last draft are not read
  if (i >= vf_count(a, b) + (draft ? 0 : 1)) return;
  const auto *x = draft ? draft_row<T>(a, b, i) : target_row<T>(a, b, i);
  const double scale = draft ? a.dscale : a.tscale;
  // slices s0, s0 + 4, ..
  const int s0 = (int(blockIdx.x) % a.groups) * (kVfWaves * a.each) + wid;
  const int mine = min(a.each, (a.slices - s0 + kVfWaves - 1) / kVfWaves);
  auto place = [&](int t) {   // of the wavefront's block t
    const int s = s0 + kVfWaves * (t / a.blocks);
    return (int64_t(s) * a.blocks + t % a.blocks) * kVfBlock;
  };
  VfRaw<T> next;
  if (mine > 0) load_block<T>(next, x, place(0), a.n);
  fill_table(table);
  __syncthreads();
  VfSum s{0.0, -__builtin_inf()};
  bool bad = false;
  for (int t = 0; t < mine * a.blocks; ++t) {
    float v[kVfEach];
#pragma unroll
    for (int q = 0; q < kVfEach; ++q) {
      v[q] = float(next.v[q / 8].v[q % 8]);
      asm("" : "+v"(v[q]));   // else the maxima are rounded to 16 bits one by one
    }
    if (t + 1 < mine * a.blocks) load_block<T>(next, x, place(t + 1), a.n);
    float m = v[0];
#pragma unroll
    for (int q = 0; q < kVfEach; ++q) {
      bad |= !(v[q] < __builtin_inff());
      m = fmaxf(m, v[q]);
    }
    const double top = fmax(s.top, double(wave_max32(m)));
    if (a.blocks > 1) s.z *= exp256((s.top - top) * scale, table);
    s.top = top;
#pragma unroll
    for (int q = 0; q < kVfEach; ++q) {
      const Factors p = factors256((double(v[q]) - top) * scale, table);
      s.z = fma(p.e, p.q, s.z);
      if (q % 2 == 1) {   // two at a time: all at once take 138 registers and not 91, 54 us and not 45
        asm volatile("" : "+v"(s.z));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (a.blocks == 1 || t % a.blocks == a.blocks - 1) {
      s.z = __ballot(bad) ? __builtin_nan("") : wave_sum64(s.z);
      if (lane == 0) (draft ? a.dsums : a.tsums)[at * a.slices + s0 + kVfWaves * (t / a.blocks)] = s;
      s = VfSum{0.0, -__builtin_inf()};
      bad = false;
    }
  }
}

// The slices' sums of a row, by a wavefront.
__device__ __forceinline__ VfSum join_slices(const VfSum *sums, int slices, double scale, const double *table) {
  const int lane = threadIdx.x & 63;
  VfSum v[kVfMaxSlices / 64];
  double top = -__builtin_inf();
#pragma unroll
  for (int u = 0; u < kVfMaxSlices / 64; ++u) {
    v[u] = VfSum{0.0, -__builtin_inf()};
    if (64 * u + lane < slices) v[u] = sums[64 * u + lane];
    top = fmax(top, v[u].top);
  }
  top = wave_max64(top);
  double z = 0;
#pragma unroll
  for (int u = 0; u < kVfMaxSlices / 64; ++u)
    if (64 * u < slices) z += v[u].z * exp256((v[u].top - top) * scale, table);
  return VfSum{wave_sum64(z), top};
}

// A drafted token and its score, by the lane of the first wavefront that has it.
struct Drafted {
  int64_t x;
  float score;
};

// Log probability of an entry.
__device__ __forceinline__ float log_of(float v, const VfSum &p, double scale) {
  return float((double(v) - p.top) * (scale * (kLn2d / 256)) - log(p.z));
}

// By all threads of a workgroup: a wavefront joins a row's slices.
template <int T>
__device__ __forceinline__ Drafted settle(const VerifyArgs &a, int b, const double *table,
                                          VfSum (*rows)[kVfMaxDrafts + 1], Settled &out) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int count = vf_count(a, b);
  // asked for first: two reads, one after the other
  bool inside = false;
  int64_t x = -1;
  float px = 0.f, qx = 0.f, u = 0.f;
  if (wid == 0 && lane < count) {
    x = a.tokens[int64_t(b) * a.k + lane];
    u = a.uniforms[int64_t(b) * (a.k + 1) + lane];
    inside = x >= 0 && x < a.n;
    if (inside) {
      px = float(target_row<T>(a, b, lane)[x]);
      if (a.draft) qx = float(draft_row<T>(a, b, lane)[x]);
    }
  }
  for (int r = wid; r < (a.draft ? 2 * count + 1 : count + 1); r += kVfWaves) {
    const bool draft = r > count;
    const int i = draft ? r - count - 1 : r;
    const VfSum s = join_slices(draft ? a.dsums + (int64_t(b) * a.k + i) * a.slices
                                      : a.tsums + (int64_t(b) * (a.k + 1) + i) * a.slices, a.slices,
                                draft ? a.dscale : a.tscale, table);
    if (lane == 0) rows[draft][i] = s;
  }
  __syncthreads();
  if (wid == 0) {
    bool stands = false;
    if (inside) {
      const VfSum p = rows[0][lane], q = rows[1][lane];
      const double is = weight64(px, p.top, a.tscale, table) / p.z;
      const double was = a.draft ? weight64(qx, q.top, a.dscale, table) / q.z : 1.0;
      stands = double(u) * was < is;
    }
    const int fallen = __ffsll(static_cast<unsigned long long>(~__ballot(stands))) - 1;   // -1: none of 64
    if (lane == 0) {
      const int n = fallen < 0 ? count : min(fallen, count);
      out.accepted = n;
      out.count = count;
      out.p = rows[0][n];
      out.q = rows[1][n < count ? n : 0];
    }
  }
  __syncthreads();
  return Drafted{x, px};
}

// The weight r of an entry: p, or where a draft fell what p has over q.
struct Over {
  bool drafted;
  int64_t x;   // without the draft's scores: its token
  VfSum p, q;  // z: the sums' reciprocals
  double ps, qs;
  bool with;
  __device__ __forceinline__ double of(float v, float d, int64_t j, const double *table) const {
#pragma clang fp contract(off)   // of equal p and q nothing is left
    const double is = weight64(v, p.top, ps, table) * p.z;
    if (!drafted) return is;
    if (!with) return j == x ? 0.0 : is;
    const double r = is - weight64(d, q.top, qs, table) * q.z;
    return r > 0 ? r : 0.0;
  }
};
__device__ __forceinline__ Over over_of(const VerifyArgs &a, int b, const Settled &s, bool drafted) {
  Over o;
  o.drafted = drafted;
  o.with = drafted && a.draft;
  o.x = drafted && !a.draft ? a.tokens[int64_t(b) * a.k + s.accepted] : -1;
  o.p = VfSum{1.0 / s.p.z, s.p.top}, o.ps = a.tscale;
  o.q = VfSum{1.0 / s.q.z, s.q.top}, o.qs = a.dscale;
  return o;
}

// r summed over the slices of a workgroup, one at a time to a wavefront.
template <int T>
__device__ __forceinline__ void sum_over(const VerifyArgs &a, int b, int group, const Settled &st, const double *table) {
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Over over = over_of(a, b, st, true);
  const auto *x = target_row<T>(a, b, st.accepted);
  const auto *d = a.draft ? draft_row<T>(a, b, st.accepted) : x;
  for (int t = 0; t < a.oeach; ++t) {
    const int s = group * (kVfWaves * a.oeach) + kVfWaves * t + wid;
    if (s >= a.slices) break;
    double sum = 0;
    for (int64_t j = int64_t(s) * a.blocks * kVfBlock, e = j + int64_t(a.blocks) * kVfBlock; j < min(e, a.n); j += kVfBlock) {
      VfRaw<T> rp, rq;
      load_block<T>(rp, x, j, a.n);
      load_block<T>(rq, d, j, a.n);
#pragma unroll
      for (int q = 0; q < kVfEach; ++q)
        sum += over.of(float(rp.v[q / 8].v[q % 8]), float(rq.v[q / 8].v[q % 8]), j + (q >> 3) * 512 + 8 * lane + (q & 7), table);
    }
    sum = wave_sum64(sum);
    if (lane == 0) __hip_atomic_store(&a.rsums[int64_t(b) * a.slices + s], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

__device__ __forceinline__ double wave_upto64(double v) {   // the sum of lanes up to this one
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(v, off, 64);
    if (lane >= off) v += o;
  }
  return v;
}

// Of each sequence: which drafts stand, by each of its workgroups; where one fell, r summed
// over each slice; then, by the last workgroup to do so (else the first), the drawn token: the
// slice that it is in, then the token.
template <int T>
__global__ void __launch_bounds__(kVfThreads) k_verify_draw(VerifyArgs a) {
  __shared__ double table[256];
  __shared__ VfSum rows[2][kVfMaxDrafts + 1];
  __shared__ Settled st;
  __shared__ double waves[kVfWaves];
  __shared__ double want_s, base_s;
  __shared__ int slice_s, drafted_s, found_s, last_s, draws_s;
  __shared__ float score_s;
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = int(blockIdx.x) / a.ogroups, group = int(blockIdx.x) % a.ogroups;
  const float u = a.uniforms[int64_t(b) * (a.k + 1) + a.k];
  fill_table(table);
  __syncthreads();
  const Drafted drafts = settle<T>(a, b, table, rows, st);
  const int n = st.accepted;
  if (group == 0) {   // all but the drawn token
    if (tid < n) {
      a.out[int64_t(b) * (a.k + 1) + tid] = drafts.x;
      if (a.logprob) a.logprob[int64_t(b) * (a.k + 1) + tid] = log_of(drafts.score, rows[0][tid], a.tscale);
    } else if (tid > n && tid <= a.k) {
      a.out[int64_t(b) * (a.k + 1) + tid] = -1;
      if (a.logprob) a.logprob[int64_t(b) * (a.k + 1) + tid] = 0.f;
    }
    if (tid == 0) a.accepted[b] = n;
  }
  if (n < st.count) {
    // The sums are written and read past the caches that other workgroups do not share, and
    // have arrived before the workgroup counts itself: the last one reads all of them.  (With
    // fences, which write back and empty those caches, 64 sequences took 44 us and not 26.)
    // All these accesses are relaxed: their order is gfx950's and not the language's.  There
    // stores and loads of agent scope go to memory that all XCDs see, the wait ends when a
    // wavefront's stores are there, and the barrier comes behind every wavefront's.
    sum_over<T>(a, b, group, st, table);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0)
      draws_s = __hip_atomic_fetch_add(&a.done[b], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.ogroups - 1;
    __syncthreads();
    if (!draws_s) return;
  } else if (group > 0) {
    return;
  }
  if (tid == 0) found_s = 0x7fffffff, last_s = -1;
  if (wid == 0) {
    constexpr int each = kVfMaxSlices / 64;   // neighbouring slices of a lane
    double r[each] = {};
    bool drafted = n < st.count;
    if (drafted) {
#pragma unroll
      for (int i = 0; i < each; ++i)
        if (each * lane + i < a.slices)
          r[i] = __hip_atomic_load(&a.rsums[int64_t(b) * a.slices + each * lane + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      drafted = __ballot(r[0] > 0 || r[1] > 0 || r[2] > 0 || r[3] > 0) != 0;   // else p and q are the same
    }
    if (!drafted) {
      const VfSum *t = a.tsums + (int64_t(b) * (a.k + 1) + n) * a.slices;
#pragma unroll
      for (int i = 0; i < each; ++i) {
        r[i] = 0;
        if (each * lane + i < a.slices) {
          const VfSum v = t[each * lane + i];
          r[i] = v.z * exp256((v.top - st.p.top) * a.tscale, table) / st.p.z;
        }
      }
    }
    double mine = 0;
#pragma unroll
    for (int i = 0; i < each; ++i) mine += r[i];
    const double upto = wave_upto64(mine), total = __shfl(upto, 63, 64);
    const double want = double(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f)) * total;
    // the first lane past `want`, or the last one with any, should rounding pass them all
    const uint64_t past = __ballot(upto > want && mine > 0), any = __ballot(mine > 0);
    const int in = past ? __ffsll(static_cast<unsigned long long>(past)) - 1 : 63 - __clzll(static_cast<long long>(any));
    if (lane == in) {
      double c = upto - mine, base = c;
      int at = -1;
#pragma unroll
      for (int i = 0; i < each; ++i) {
        if (r[i] > 0 && (at < 0 || !(c > want))) at = each * lane + i, base = c;
        c += r[i];
      }
      slice_s = at;
      base_s = base;
      want_s = want;
      drafted_s = drafted;
    }
    if (lane == 0 && !(total > 0 && total < __builtin_inf())) slice_s = -1;   // NaN, or nothing: no token
  }
  __syncthreads();
  int token = -1;
  if (slice_s >= 0) {
    constexpr int E = kVfBlock / kVfThreads;   // consecutive entries of a thread
    const Over over = over_of(a, b, st, drafted_s);
    const auto *x = target_row<T>(a, b, n);
    const auto *d = over.with ? draft_row<T>(a, b, n) : x;
    const int64_t j0 = int64_t(slice_s) * a.blocks * kVfBlock, j1 = min(a.n, j0 + int64_t(a.blocks) * kVfBlock);
    double base = base_s;
    for (int64_t j = j0; j < j1; j += kVfBlock) {
      const int64_t at = j + tid * E;
      float v[E], w[E];
#pragma unroll
      for (int q = 0; q < E; ++q) v[q] = float(x[min(at + q, j1 - 1)]), w[q] = float(d[min(at + q, j1 - 1)]);
      double r[E], sum = 0;
#pragma unroll
      for (int q = 0; q < E; ++q) {
        r[q] = at + q < j1 ? over.of(v[q], w[q], at + q, table) : 0.0;
        sum += r[q];
      }
      const double upto = wave_upto64(sum);
      if (lane == 63) waves[wid] = upto;
      __syncthreads();
      double c = base + (upto - sum);
      for (int k = 0; k < wid; ++k) c += waves[k];
      int found = 0x7fffffff, last = -1;
#pragma unroll
      for (int q = 0; q < E; ++q) {
        c += r[q];
        if (r[q] > 0) last = int(at) + q;
        if (c > want_s && r[q] > 0 && found == 0x7fffffff) found = int(at) + q;
      }
      if (found != 0x7fffffff) atomicMin(&found_s, found);
      if (last >= 0) atomicMax(&last_s, last);
      __syncthreads();
      // the token so far, and its score
      token = found_s != 0x7fffffff ? found_s : last_s;
#pragma unroll
      for (int q = 0; q < E; ++q)
        if (at + q == token) score_s = v[q];
      if (found_s != 0x7fffffff) break;
      for (int k = 0; k < kVfWaves; ++k) base += waves[k];
      __syncthreads();
    }
    __syncthreads();
  }
  if (tid) return;
  a.out[int64_t(b) * (a.k + 1) + n] = token;
  if (a.logprob) a.logprob[int64_t(b) * (a.k + 1) + n] = token < 0 ? 0.f : log_of(score_s, st.p, a.tscale);
}

static int64_t verify_rows(int64_t b, int k, bool draft) { return b * (k + 1 + (draft ? k : 0)); }

// Blocks of a slice, and slices of a row.
static int verify_blocks(int64_t n) { return int((n + int64_t(kVfBlock) * kVfMaxSlices - 1) / (int64_t(kVfBlock) * kVfMaxSlices)); }
static int verify_slices(int64_t n) {
  const int64_t slice = int64_t(kVfBlock) * verify_blocks(n);
  return int((n + slice - 1) / slice);
}
// Slices of a wavefront: one where that is no more than `most` workgroups (of the sums of 64
// sequences with 6,144 of them 40 us, 43 with 4,096 or 8,192; of the second kernel with 1,024
// 17, 19 with 2,048, as each settles first).
static int verify_each(int64_t rows, int slices, int64_t most) {
  const int64_t each = rows * slices / (kVfWaves * most), all = (slices + kVfWaves - 1) / kVfWaves;
  return int(each < 1 ? 1 : each > all ? all : each);
}

static bool verify_sizes_ok(int64_t b, int k, int64_t n) {
  return b >= 0 && k >= 0 && k <= kVfMaxDrafts && n >= 1 && n <= 0x7fffffff - 2 * 4096 &&
         b <= 0x7fffffff / kVfThreads / (2 * k + 1);   // a grid counts its threads in 32 bits
}

static size_t verify_bytes(int64_t b, int k, bool draft, int slices) {
  return size_t(verify_rows(b, k, draft)) * slices * sizeof(VfSum) +
         size_t(b) * (slices * sizeof(double) + sizeof(int));
}

template <int T>
static void launch_verify(const VerifyArgs &a, hipStream_t s) {
  const dim3 threads(kVfThreads);
  hipLaunchKernelGGL(k_verify_sums<T>, dim3(unsigned(verify_rows(a.b, a.k, a.draft != nullptr) * a.groups)), threads, 0,
                     s, a);
  hipLaunchKernelGGL(k_verify_draw<T>, dim3(unsigned(int64_t(a.b) * a.ogroups)), threads, 0, s, a);
}

}  // namespace rslm

using namespace rslm;

extern "C" {

size_t rslm_verify_workspace(int64_t b, int32_t k, int64_t n, int32_t draft) {
  if (!verify_sizes_ok(b, k, n) || b == 0) return 0;
  return verify_bytes(b, k, draft != 0, verify_slices(n));
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
  const double unit = 256 * 1.442695040888963407360;
  VerifyArgs a{target, draft,  target_seq_stride, target_stride,  draft_seq_stride,
               draft_stride, int(b), k, n, tokens, uniforms, counts, double(scale) * unit,
               with ? double(draft_scale) * unit : 1.0};
  a.slices = verify_slices(n);
  a.blocks = verify_blocks(n);
  a.each = verify_each(verify_rows(b, k, with), a.slices, 6144);
  a.groups = (a.slices + kVfWaves * a.each - 1) / (kVfWaves * a.each);
  a.oeach = verify_each(b, a.slices, 1024);
  a.ogroups = k > 0 ? (a.slices + kVfWaves * a.oeach - 1) / (kVfWaves * a.oeach) : 1;
  a.tsums = static_cast<VfSum *>(ws);
  a.dsums = a.tsums + size_t(b) * (k + 1) * a.slices;
  a.rsums = reinterpret_cast<double *>(a.tsums + size_t(verify_rows(a.b, k, with)) * a.slices);
  a.done = reinterpret_cast<int *>(a.rsums + size_t(b) * a.slices);
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
