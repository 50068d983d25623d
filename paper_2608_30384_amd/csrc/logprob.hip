// Log probabilities over rows of scores, z = scale * score:
//   lse = log sum_j e^{z_j},  log probability of an entry z_j - lse,
//   entropy = lse - sum_j p_j z_j,  and the k largest entries;
// and the gradient  dz_j = dlp (1[j = target] - p_j) - dH p_j (z_j - lse + H).
//
// Forward: one pass over a row.  A thread keeps a running maximum and two sums
// of the entries it reads, Z = sum w and W = sum w y with y = (score - maximum)
// scale log2(e) and w = 2^y, and rescales them when its maximum rises; the
// threads' are joined at the end (lse = maximum scale + ln Z, entropy = ln Z - ln2 W / Z).
// The k largest come from the same pass.  The k-th largest of the threads' running
// maxima is a value that at least k entries reach; a
// thread whose piece of 16 entries reaches the one known so far notes the piece
// in LDS.  At the end the noted pieces are read again (from the cache) for the
// entries at or above the last such value, about k, which are ranked.  A row
// that overflows the notes is gone through once more, a few entries at a time: one that
// ascends, say, and most long rows for k of about 200 and more, as the bound is weak
// where k nears the 256 threads and there is none past them.  Few rows are cut into
// slices, joined by a second kernel; the slices' candidates, up to 2 k each, share
// its 2,048 places, so that a row has 51 slices at most at k = 20, 10 at k = 100, 2
// at k = 1,024.
// us a call, repeated by itself: 4,096 x 32,768 bfloat16 55 without alternatives (4.9
// TB/s), 69 with k = 10 (VALU 72 % busy), 87 with 100, 374 with 200, 600 with 256, 4,400
// with 1,024; one row of 1,000,000 float32 17, 20, 39, 227, 279, 16,200.  Of the
// arrangements for k = 10 (73 then): 97 where the bound came of ranking 64 parts' maxima,
// lane by lane, and 104 where every entry at or above the first piece's bound went to
// the candidates at once.  1 x 131,072 float32, k = 20: 7.1 us in 32 slices and 6.4 for
// the join, both the latency of their barriers and reads.  Backward, 4,096 x 32,768
// bfloat16: 106 us behind the forward pass (5.1 TB/s read and written), 127 by itself;
// VALU 94 % busy, so that neither memory nor the arithmetic has much room.
//
// An entry of -infinity (or one that scale makes so) is masked: probability 0,
// no alternative, gradient 0.  A row of nothing else has lse -infinity and
// entropy 0.  Floors: one read forward, a read and a write backward.
#include "mx4_dev.h"
#include "select_dev.h"

namespace rslm {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kLpThreads = 256;
constexpr int kLpEach = 16;                          // entries of a thread in a piece
constexpr int kLpPiece = kLpThreads * kLpEach;
constexpr int kLpMaxSlices = 256;
constexpr int kLpNotes = 1024;

// A difference of scores times scale, as (v part - m part) times rest, part a power
// of two and the first of them one fused step: two scores may lie further apart than
// float32's largest value, which at scales up to 1 is still a z of interest and
// takes halves.  At larger ones such a z - lse is below float32's range anyway.
struct ScoreStep {
  float part, rest, c;   // c: rest log2(e)
  __device__ __forceinline__ explicit ScoreStep(float scale)
      : part(scale <= 1.f ? 0.5f : 1.f), rest(scale <= 1.f ? 2.f * scale : scale), c(rest * kLog2e) {}
  __device__ __forceinline__ float apart(float v, float m) const { return fmaf(v, part, -(m * part)); }
};

// Running maximum (of the scores) and sums of part of a row.
struct SoftSum {
  float m, z, w;
};

// The sums of a and b together.
__device__ __forceinline__ SoftSum soft_join(const SoftSum &a, const SoftSum &b, const ScoreStep &u) {
  const float m = fmaxf(a.m, b.m);
  if (m == -__builtin_inff()) {
    // nothing but masked entries, or NaN
    return SoftSum{m, a.z + b.z, a.w + b.w};
  }
  SoftSum r{m, 0.f, 0.f};
  const float da = u.apart(a.m, m) * u.c, db = u.apart(b.m, m) * u.c;
  // a part that is empty keeps what it has (0, or NaN): e^-inf times it
  const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
  r.z = a.z * ea + b.z * eb;
  r.w = ea * (a.w + fmaxf(da, -200.f) * a.z) + eb * (b.w + fmaxf(db, -200.f) * b.z);
  return r;
}

__device__ __forceinline__ SoftSum soft_join_wave(SoftSum s, const ScoreStep &u) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const SoftSum o{__shfl_xor(s.m, off, 64), __shfl_xor(s.z, off, 64), __shfl_xor(s.w, off, 64)};
    s = soft_join(s, o, u);
  }
  return s;
}

struct LogprobArgs {
  const void *scores;
  int64_t m, n, stride;
  float scale;
  const int64_t *target;
  int k;
  float *logprob, *lse, *entropy, *stats, *top_logprob;
  int32_t *top_ids;
  int slices;
  int64_t per;          // entries of a slice, a multiple of kLpPiece
  int room;             // entries that a slice may leave, at least k
  SoftSum *sums;        // m x slices
  uint64_t *cands;      // m x kSelCap: slices x room of them used
  int32_t *counts;      // m x slices
};

// z - lse of a score, from the row's largest and ln Z: exact to the last places
// where z itself is large, and -infinity for a masked entry.
__device__ __forceinline__ float log_of(float v, float m, float lz, float scale) {
  const ScoreStep u(scale);
  return v * scale == -__builtin_inff() ? -__builtin_inff() : fmaf(u.apart(v, m), u.rest, -lz);
}

// The score of the row's target, asked for early: two reads, one after the other.
struct Target {
  bool in;
  float score;
};
template <int T>
__device__ __forceinline__ Target target_of(const LogprobArgs &a, int64_t row) {
  const int64_t t = a.logprob ? a.target[row] : -1;
  Target r{t >= 0 && t < a.n, 0.f};
  if (r.in) r.score = load_float<T>(a.scores, row * a.stride + t);
  return r;
}

// The row's numbers from its sums, by one thread; ln Z.
__device__ __forceinline__ float emit_row(const LogprobArgs &a, int64_t row, const SoftSum &s, const Target &target) {
  float lz = logf(s.z), lse = fmaf(s.m, a.scale, lz), h = fmaf(-kLn2, s.w / s.z, lz);
  if (s.z != s.z) {
    lz = lse = h = s.z;
  } else if (s.m * a.scale == -__builtin_inff()) {
    lse = -__builtin_inff();
    h = 0.f;
  }
  if (a.lse) a.lse[row] = lse;
  if (a.entropy) a.entropy[row] = h;
  a.stats[2 * row] = s.m;
  a.stats[2 * row + 1] = lz;
  if (a.logprob) a.logprob[row] = target.in ? log_of(target.score, s.m, lz, a.scale) : 0.f;
  return lz;
}

// The k best of the cnt composites in sm.buf, in order, as log probabilities.
// Up to 1,024 entries, an entry's place is the number of larger ones (no two are
// equal): one read of all by every thread, instead of a sort's barriers.
__device__ __forceinline__ void emit_top(const LogprobArgs &a, int64_t row, SelectSmem &sm, int cnt, float m, float lz) {
  const int t = threadIdx.x, k = a.k;
  float *os = a.top_logprob + row * k;
  int32_t *oi = a.top_ids + row * k;
  auto put = [&](int r, uint64_t e) {
    const float v = key_to_float(uint32_t(e >> 32));
    os[r] = log_of(v, m, lz, a.scale);
    oi[r] = v * a.scale == -__builtin_inff() ? -1 : int32_t(0xffffffffu - uint32_t(e & 0xffffffffu));
  };
  if (cnt <= 4 * kLpThreads) {
    uint64_t e[4];
    int r[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = t + i * kLpThreads < cnt ? sm.buf[t + i * kLpThreads] : 0ull;
    if (cnt <= kLpThreads) {
#pragma unroll 8
      for (int j = 0; j < cnt; ++j) r[0] += sm.buf[j] > e[0];
    } else {
#pragma unroll 4
      for (int j = 0; j < cnt; ++j) {
        const uint64_t o = sm.buf[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] += o > e[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t + i * kLpThreads < cnt && r[i] < k) put(r[i], e[i]);
  } else {
    sort_desc(sm, cnt);
    for (int j = t; j < min(cnt, k); j += kLpThreads) put(j, sm.buf[j]);
  }
  for (int j = cnt + t; j < k; j += kLpThreads) {
    os[j] = -__builtin_inff();
    oi[j] = -1;
  }
}

// A thread's entries of a piece, as they are stored; -infinity past the end.
template <int T>
struct PieceRaw {
  typename FloatType<T>::type v[kLpEach];
};
template <int T>
__device__ __forceinline__ void load_piece(PieceRaw<T> &p, const typename FloatType<T>::type *x, int64_t j, int64_t end) {
  typedef typename FloatType<T>::type F;
#pragma unroll
  for (int u = 0; u < kLpEach / 8; ++u) {
    const int64_t at = j + (u * kLpThreads + int(threadIdx.x)) * 8, left = end - at;
    if (left >= 8) {
      if constexpr (T == RSLM_F32) {
        const F32x8u e = *reinterpret_cast<const F32x8u *>(x + at);
        __builtin_memcpy(&p.v[8 * u], &e, sizeof(e));
      } else {
        const H16x8u e = *reinterpret_cast<const H16x8u *>(x + at);
        __builtin_memcpy(&p.v[8 * u], &e, sizeof(e));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p.v[8 * u + i] = i < left ? x[at + i] : F(-__builtin_inff());
    }
  }
}
template <int T>
__device__ __forceinline__ float piece_values(float (&v)[kLpEach], const PieceRaw<T> &p) {
#pragma unroll
  for (int i = 0; i < kLpEach; ++i) v[i] = float(p.v[i]);
  float top = v[0];
#pragma unroll
  for (int i = 1; i < kLpEach; ++i) top = fmaxf(top, v[i]);
  return top == top ? top : -__builtin_inff();
}
// index in the row of a thread's entry i of the piece at j
__device__ __forceinline__ int32_t piece_index(int64_t j, int i) {
  return int32_t(j + ((i >> 3) * kLpThreads + int(threadIdx.x)) * 8 + (i & 7));
}

// A value that at least k of the threads' `top` reach, the k-th largest cut to
// its upper 16 bits (as ordered integers): found bit by bit, a step being four
// compares and counts of lanes.  -infinity where k is more than the threads.
__device__ __forceinline__ float top_bound(float top, int k, uint32_t *tops) {
  if (k > kLpThreads) return -__builtin_inff();
  tops[threadIdx.x] = order_key(top + 0.f);
  __syncthreads();
  const uint4 v = reinterpret_cast<const uint4 *>(tops)[threadIdx.x & 63];
  __syncthreads();
  uint32_t bound = 0u;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t up = bound | 1u << bit;
    const int reach = __popcll(__ballot(v.x >= up)) + __popcll(__ballot(v.y >= up)) + __popcll(__ballot(v.z >= up)) +
                      __popcll(__ballot(v.w >= up));
    if (reach >= k) bound = up;
  }
  return bound < 0x00800000u ? -__builtin_inff() : key_to_float(bound);   // that of the lowest float
}

// Entries of a thread's piece at or above thr, to the buffer while it has room
// (sm.count counts on).
__device__ __forceinline__ void push(SelectSmem &sm, const float (&v)[kLpEach], float top, float thr, int64_t j, int i0,
                                     int i1) {
  if (!(top >= thr)) return;
#pragma unroll
  for (int i = 0; i < kLpEach; ++i) {
    if (i >= i0 && i < i1 && v[i] >= thr && v[i] > -__builtin_inff()) {
      const uint32_t pos = atomicAdd(&sm.count, 1u);
      if (pos < uint32_t(kSelCap)) sm.buf[pos] = composite(order_key(v[i] + 0.f), piece_index(j, i));
    }
  }
}

// The buffer's k best of `count` (a barrier ahead of it is the caller's): their
// number, and the k-th as the threshold.
__device__ __forceinline__ int cut(SelectSmem &sm, int count, int k, float &thr) {
  sort_desc(sm, count);
  __syncthreads();
  if (count < k) return count;
  thr = fmaxf(thr, key_to_float(uint32_t(sm.buf[k - 1] >> 32)));
  return k;
}

// The candidates of [j0, j1) again, where they overflowed: 1,024 entries at a
// time, which always fit beside the k <= 1,024 that the buffer is cut to when
// it has no room for more.  Returns their number.
template <int T>
__device__ __noinline__ int collect_again(SelectSmem &sm, const typename FloatType<T>::type *x, int64_t j0, int64_t j1,
                                          int k) {
  int count = 0;
  float thr = -__builtin_inff();
  for (int64_t j = j0; j < j1; j += kLpPiece) {
    PieceRaw<T> raw;
    float v[kLpEach];
    load_piece<T>(raw, x, j, j1);
    const float top = piece_values<T>(v, raw);
    if (!__syncthreads_or(top >= thr && top > -__builtin_inff())) continue;
    bool full = false;   // the buffer has been cut to k, and nothing added
    for (int i = 0; i < kLpEach; i += 4) {
      if (threadIdx.x == 0) sm.count = uint32_t(count);
      __syncthreads();
      push(sm, v, top, thr, j, i, i + 4);
      __syncthreads();
      const int now = int(sm.count);
      __syncthreads();
      full = full && now == count;
      count = now;
      if (count > kSelCap - 1024 && count > k) {
        count = cut(sm, count, k, thr);
        full = count == k;
      }
    }
    // later entries have higher indices and lose to equal ones
    if (full) thr = key_to_float(order_key(thr + 0.f) + 1u);
  }
  return count;
}

template <int T, bool TOP>
__global__ void __launch_bounds__(kLpThreads) k_logprob(LogprobArgs a) {
  __shared__ SelectSmem sm;
  __shared__ SoftSum parts[kLpThreads / 64];
  __shared__ __align__(16) uint32_t tops[kLpThreads];
  __shared__ uint32_t notes[TOP ? kLpNotes : 1];   // piece * 256 + thread
  __shared__ float lz_s;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t row = blockIdx.x / a.slices;
  const int slice = int(blockIdx.x % a.slices);
  const int64_t j0 = int64_t(slice) * a.per, j1 = min(a.n, j0 + a.per);
  const typename FloatType<T>::type *x = static_cast<const typename FloatType<T>::type *>(a.scores) + row * a.stride;
  const ScoreStep step(a.scale);
  const float ninf = -__builtin_inff();
  SoftSum s{ninf, 0.f, 0.f};
  float thr = ninf;     // at least k entries reach it
  if (TOP && tid == 0) sm.count = 0u;
  if (TOP) __syncthreads();
  PieceRaw<T> next;
  if (j0 < j1) load_piece<T>(next, x, j0, j1);
  Target target{};
  if (a.slices == 1 && tid == 0) target = target_of<T>(a, row);
  int piece = 0, look = 0;
  for (int64_t j = j0; j < j1; j += kLpPiece, ++piece) {
    float v[kLpEach];
    const float top = piece_values<T>(v, next);
    if (j + kLpPiece < j1) load_piece<T>(next, x, j + kLpPiece, j1);
    if (top > s.m) {
      if (s.m > ninf) {
        const float d = step.apart(s.m, top) * step.c, e = __builtin_amdgcn_exp2f(d);
        s.w = e * (s.w + fmaxf(d, -200.f) * s.z);
        s.z *= e;
      }
      s.m = top;
    }
    const float ref = s.m == ninf ? 0.f : s.m;
#pragma unroll
    for (int i = 0; i < kLpEach; ++i) {
      const float y = step.apart(v[i], ref) * step.c;
      const float w = __builtin_amdgcn_exp2f(y);
      s.z += w;
      s.w = fmaf(w, fmaxf(y, -200.f), s.w);   // masked: w = 0 times -200
    }
    if constexpr (TOP) {
      if (piece == look && j + kLpPiece < j1) {   // pieces 0, 3, 15, 63, ...
        thr = fmaxf(thr, top_bound(s.m, a.k, tops));
        look = 4 * look + 3;
      }
      if (top >= thr && top > ninf) {
        const uint32_t pos = atomicAdd(&sm.count, 1u);
        if (pos < uint32_t(kLpNotes)) notes[pos] = uint32_t(piece * kLpThreads + tid);
      }
    }
  }
  int count = 0;
  if constexpr (TOP) {
    thr = fmaxf(thr, top_bound(s.m, a.k, tops));
    __syncthreads();
    const int noted = int(sm.count);
    __syncthreads();
    if (tid == 0) sm.count = 0u;
    __syncthreads();
    bool again = noted > kLpNotes;
    if (!again) {
      for (int i = tid; i < noted; i += kLpThreads) {
        const uint32_t at = notes[i];
        const int64_t j = j0 + int64_t(at / kLpThreads) * kLpPiece;
#pragma unroll
        for (int u = 0; u < kLpEach / 8; ++u) {
          const int64_t j8 = j + (u * kLpThreads + int(at % kLpThreads)) * 8;
          const int left = int(j1 - j8 < 8 ? (j1 - j8 < 0 ? 0 : j1 - j8) : 8);
          float e[8];
          load_float8<T>(e, x + j8, 0, left);
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (q < left && e[q] >= thr && e[q] > ninf) {
              const uint32_t pos = atomicAdd(&sm.count, 1u);
              if (pos < uint32_t(kSelCap)) sm.buf[pos] = composite(order_key(e[q] + 0.f), int32_t(j8 + q));
            }
        }
      }
      __syncthreads();
      count = int(sm.count);
      __syncthreads();
      again = count > kSelCap;
    }
    if (again) {
      count = collect_again<T>(sm, x, j0, j1, a.k);
      __syncthreads();
    }
  }
  s = soft_join_wave(s, step);
  if (lane == 0) parts[wid] = s;
  __syncthreads();
  s = parts[0];
#pragma unroll
  for (int i = 1; i < kLpThreads / 64; ++i) s = soft_join(s, parts[i], step);
  if (a.slices == 1) {
    if (tid == 0) lz_s = emit_row(a, row, s, target);
    __syncthreads();
    if constexpr (TOP) emit_top(a, row, sm, count, s.m, lz_s);
  } else {
    if (tid == 0) a.sums[blockIdx.x] = s;
    if constexpr (TOP) {
      if (count > a.room) {
        float none = ninf;
        count = cut(sm, count, a.k, none);
      }
      if (tid == 0) a.counts[blockIdx.x] = count;
      for (int i = tid; i < count; i += kLpThreads) a.cands[row * kSelCap + slice * a.room + i] = sm.buf[i];
    }
  }
}

// Joins the slices of a row.  Of their candidates, those that can be among the k
// largest (top_bound again) are ranked.
template <int T, bool TOP>
__global__ void __launch_bounds__(kLpThreads) k_logprob_join(LogprobArgs a) {
  __shared__ SelectSmem sm;
  __shared__ SoftSum parts[kLpThreads / 64];
  __shared__ __align__(16) uint32_t tops[kLpThreads];
  __shared__ float lz_s;
  constexpr int kHeld = kSelCap / kLpThreads;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t row = blockIdx.x;
  const ScoreStep step(a.scale);
  SoftSum s{-__builtin_inff(), 0.f, 0.f};
  if (tid < a.slices) s = a.sums[row * a.slices + tid];
  Target target{};
  uint64_t e[kHeld];
  float top = -__builtin_inff();
  if constexpr (TOP) {
    if (tid == 0) sm.count = 0u;
    // room for all is there: candidates and their numbers are read at once
    int have[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int at = i * kLpThreads + tid;
      e[i] = a.cands[row * kSelCap + at];
      have[i] = a.counts[row * a.slices + min(at / a.room, a.slices - 1)];
    }
    if (tid == 0) target = target_of<T>(a, row);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int at = i * kLpThreads + tid, slice = at / a.room;
      const bool in = slice < a.slices && at - slice * a.room < have[i];
      if (!in) e[i] = 0ull;   // no composite is 0
      if (in) top = fmaxf(top, key_to_float(uint32_t(e[i] >> 32)));
    }
  } else if (tid == 0) {
    target = target_of<T>(a, row);
  }
  s = soft_join_wave(s, step);
  if (lane == 0) parts[wid] = s;
  __syncthreads();
  s = parts[0];
#pragma unroll
  for (int i = 1; i < kLpThreads / 64; ++i) s = soft_join(s, parts[i], step);
  if (tid == 0) lz_s = emit_row(a, row, s, target);
  if constexpr (TOP) {
    const float bound = top_bound(top, a.k, tops);
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (e[i] && key_to_float(uint32_t(e[i] >> 32)) >= bound) sm.buf[atomicAdd(&sm.count, 1u)] = e[i];
    __syncthreads();
    emit_top(a, row, sm, int(sm.count), s.m, lz_s);
  }
}

template <int T>
__global__ void __launch_bounds__(256) k_logprob_backward(const void *scores, int64_t rows, int64_t n, int64_t stride,
                                                          float scale, const int64_t *__restrict__ target,
                                                          const float *__restrict__ stats,
                                                          const float *__restrict__ entropy,
                                                          const float *__restrict__ dlogprob,
                                                          const float *__restrict__ dentropy, void *out,
                                                          int64_t ostride, int64_t pieces) {
  for (int64_t at = blockIdx.x; at < rows * pieces; at += gridDim.x) {
    const int64_t row = at / pieces;
    const int64_t j0 = ((at - row * pieces) * 256 + threadIdx.x) * 8;
    if (j0 >= n) continue;
    const typename FloatType<T>::type *x = static_cast<const typename FloatType<T>::type *>(scores) + row * stride;
    const int left = int(n - j0 < 8 ? n - j0 : 8);
    float v[8];
    load_float8<T>(v, x + j0, 0, left);
    const int64_t t = target ? target[row] : -1;
    const float m = stats[2 * row], lz = stats[2 * row + 1];
    const float dl = dlogprob && t >= 0 && t < n ? dlogprob[row] : 0.f;
    const float dh = dentropy ? dentropy[row] : 0.f, h = dentropy ? entropy[row] : 0.f;
    const float a = dl * scale, b = dh * scale;   // here: a use beside its load would wait for it
    // Of 2^24 p, so that a p below float32's normal range keeps its digits, the
    // 2^-24 is taken off a and b, or where these are small themselves off the product.
    const bool small = fmaxf(fabsf(a), fabsf(b)) < 0x1p-60f;
    const float as = small ? a : a * 0x1p-24f, bs = small ? b : b * 0x1p-24f, rest = small ? -0x1p-24f : -1.f;
    const ScoreStep u(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float lp = fmaf(u.apart(v[i], m), u.rest, -lz);
      const float p = __builtin_amdgcn_exp2f(fmaf(lp, kLog2e, 24.f));
      const float d = fmaf(p * fmaf(bs, fmaxf(lp, -1e4f) + h, as), rest, j0 + i == t ? a : 0.f);
      v[i] = v[i] * scale == -__builtin_inff() ? 0.f : d;
    }
    store_float8<T>(v, static_cast<typename FloatType<T>::type *>(out) + row * ostride + j0, 0, left);
  }
}

// Slices of a row: enough workgroups for the GPU where there are few rows, a
// piece each at least, and no more candidates than the join's buffer holds.
static int logprob_slices(int64_t m, int64_t n, int k) {
  int64_t s = (1024 + m - 1) / m;
  const int64_t most = (n + kLpPiece - 1) / kLpPiece;
  if (s > most) s = most;
  if (s > kLpMaxSlices) s = kLpMaxSlices;
  // twice the k best of a slice, which it mostly need not cut to them
  const int room = k <= kSelCap / 16 ? 2 * k : k;
  if (k > 0 && s > kSelCap / room) s = kSelCap / room;
  return int(s < 1 ? 1 : s);
}
static size_t logprob_sums_bytes(int64_t m, int slices) {
  return (size_t(m) * slices * sizeof(SoftSum) + 255) / 256 * 256;
}

template <int T>
static void launch_logprob(const LogprobArgs &a, hipStream_t s) {
  const dim3 grid(unsigned(a.m * a.slices)), rows(unsigned(a.m)), threads(kLpThreads);
  if (a.k > 0) {
    hipLaunchKernelGGL((k_logprob<T, true>), grid, threads, 0, s, a);
    if (a.slices > 1) hipLaunchKernelGGL((k_logprob_join<T, true>), rows, threads, 0, s, a);
  } else {
    hipLaunchKernelGGL((k_logprob<T, false>), grid, threads, 0, s, a);
    if (a.slices > 1) hipLaunchKernelGGL((k_logprob_join<T, false>), rows, threads, 0, s, a);
  }
}

static bool logprob_sizes_ok(int64_t m, int64_t n, int k) {
  return m >= 0 && n >= 1 && m <= 0x7fffffff / kLpMaxSlices && n <= 0x7fffffff && k >= 0 && k <= kMaxK;
}
// Up to 2^127: times log2(e) it has to stay within float32.
static bool scale_ok(float scale) { return scale > 0.f && scale <= 0x1p127f; }

}  // namespace rslm

using namespace rslm;

extern "C" {

size_t rslm_logprob_workspace(int64_t m, int64_t n, int32_t k) {
  if (!logprob_sizes_ok(m, n, k) || m == 0) return 0;
  const int s = logprob_slices(m, n, k);
  return s > 1 ? logprob_sums_bytes(m, s) + size_t(m) * (k > 0 ? kSelCap * sizeof(uint64_t) + s * sizeof(int32_t) : 0)
               : 0;
}

int rslm_logprob(const void *scores, int32_t dtype, int64_t m, int64_t n, int64_t stride, float scale,
                 const int64_t *target, int32_t k, float *logprob, float *lse, float *entropy, float *stats,
                 float *top_logprob, int32_t *top_ids, void *ws, size_t ws_bytes, void *stream) {
  if (!logprob_sizes_ok(m, n, k) || !float_type_ok(dtype) || stride < 0 || !scale_ok(scale))
    return RSLM_ERR_INVALID_ARG;
  if (m == 0) return RSLM_OK;
  if (!scores || !stats || (logprob && !target) || (k > 0 && (!top_logprob || !top_ids)) ||
      !aligned_to(scores, float_bytes(dtype)) || !aligned_to(target, 8) || !aligned_to(logprob, 4) ||
      !aligned_to(lse, 4) || !aligned_to(entropy, 4) || !aligned_to(stats, 4) || !aligned_to(top_logprob, 4) || !aligned_to(top_ids, 4))
    return RSLM_ERR_INVALID_ARG;
  LogprobArgs a{scores, m, n, stride, scale, target, k, logprob, lse, entropy, stats, top_logprob, top_ids};
  a.slices = logprob_slices(m, n, k);
  if (ws_bytes < rslm_logprob_workspace(m, n, k)) return RSLM_ERR_WORKSPACE;
  if (a.slices > 1) {
    if (!ws || !aligned_to(ws, 16)) return RSLM_ERR_INVALID_ARG;
    a.sums = static_cast<SoftSum *>(ws);
    a.room = kSelCap / a.slices;
    a.cands = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + logprob_sums_bytes(m, a.slices));
    a.counts = reinterpret_cast<int32_t *>(a.cands + size_t(m) * kSelCap);
  }
  a.per = (n + int64_t(a.slices) * kLpPiece - 1) / (int64_t(a.slices) * kLpPiece) * kLpPiece;
  const hipStream_t s = as_stream(stream);
  if (dtype == RSLM_F32) launch_logprob<RSLM_F32>(a, s);
  else if (dtype == RSLM_F16) launch_logprob<RSLM_F16>(a, s);
  else launch_logprob<RSLM_BF16>(a, s);
  return check_launch();
}

int rslm_logprob_backward(const void *scores, int32_t dtype, int64_t m, int64_t n, int64_t stride, float scale,
                          const int64_t *target, const float *stats, const float *entropy, const float *dlogprob,
                          const float *dentropy, void *dscores, int64_t dstride, void *stream) {
  if (!logprob_sizes_ok(m, n, 0) || !float_type_ok(dtype) || stride < 0 || (m > 1 && dstride < n) ||
      !scale_ok(scale))
    return RSLM_ERR_INVALID_ARG;
  if (m == 0) return RSLM_OK;
  if (!scores || !stats || !dscores || (dlogprob && !target) || (dentropy && !entropy) ||
      !aligned_to(scores, float_bytes(dtype)) || !aligned_to(dscores, float_bytes(dtype)) || !aligned_to(target, 8) ||
      !aligned_to(stats, 4) || !aligned_to(entropy, 4) || !aligned_to(dlogprob, 4) || !aligned_to(dentropy, 4))
    return RSLM_ERR_INVALID_ARG;
  const int64_t pieces = (n + 2047) / 2048;
  const dim3 grid(unsigned(m * pieces < (1 << 22) ? m * pieces : (1 << 22)));
  const hipStream_t s = as_stream(stream);
#define RSLM_LOGPROB_BACKWARD(T)                                                                                  \
  hipLaunchKernelGGL(k_logprob_backward<T>, grid, dim3(256), 0, s, scores, m, n, stride, scale, target, stats,    \
                     entropy, dlogprob, dentropy, dscores, dstride, pieces)
  if (dtype == RSLM_F32) RSLM_LOGPROB_BACKWARD(RSLM_F32);
  else if (dtype == RSLM_F16) RSLM_LOGPROB_BACKWARD(RSLM_F16);
  else RSLM_LOGPROB_BACKWARD(RSLM_BF16);
#undef RSLM_LOGPROB_BACKWARD
  return check_launch();
}

}  // extern "C"
