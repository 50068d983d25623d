// Rows of a table for given tokens, out_i = scale table[id_i] (0 for a token outside the
// table), and the gradient of a float table, dtable_v = scale sum over i with id_i = v of
// dout_i.
//
// Forward: bound by memory, a row read and written for each token: 65,536 x 768 bfloat16 of a
// table that the last-level cache holds 39 us (5.2 TB/s), 256 tokens of MX4 rows 3.7.
//
// Gradient: the tokens are sorted by their ids, a stable counting sort of a digit at a
// time, so that a table row's tokens lie side by side in the order in which they came;
// runs of them are summed in float32, always in that order, so that results do not
// change from call to call.  Bound by memory: dout read once, dtable written once.
#include "mx4_dev.h"

namespace rslm {

// ---- forward

struct EmbedArgs {
  const void *table;       // floats, or codes of MX4 rows
  const uint8_t *scales;
  int64_t rows, stride;
  const void *ids;
  int wide;                // ids: 64-bit, else 32
  int64_t n;
  int dim, steps, each;
  float scale;
  void *out;
  int64_t ostride;
};

__device__ __forceinline__ int64_t id_at(const void *ids, int wide, int64_t i) {
  return wide ? static_cast<const int64_t *>(ids)[i] : int64_t(static_cast<const int32_t *>(ids)[i]);
}

constexpr int kMx4Table = 3;   // beside RSLM_F32, ...
constexpr int kEmbedFlight = 4;

// 16 lanes to a token, 8 coordinates each of a group of 128, four groups in flight.
template <int S, int T>
__global__ void __launch_bounds__(256) k_embed(EmbedArgs a) {
  const int r = threadIdx.x & 15;
  const int t0 = blockIdx.y * a.each, t1 = min(a.steps, t0 + a.each);
  for (int64_t i = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); i < a.n; i += int64_t(gridDim.x) * 16) {
    const int64_t id = id_at(a.ids, a.wide, i);
    const bool in = id >= 0 && id < a.rows;
    typename FloatType<T>::type *o = static_cast<typename FloatType<T>::type *>(a.out) + i * a.ostride;
    for (int t = t0; t < t1; t += kEmbedFlight) {
      float v[kEmbedFlight][8];
      if constexpr (S == kMx4Table) {
        uint32_t w[kEmbedFlight], s[kEmbedFlight];
#pragma unroll
        for (int u = 0; u < kEmbedFlight; ++u) {
          const int64_t g = id * a.steps + min(t + u, t1 - 1);
          w[u] = in ? *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(a.table) + g * 64 + 4 * r) : 0u;
          s[u] = in ? a.scales[g * 4 + (r >> 2)] : 0u;
        }
#pragma unroll
        for (int u = 0; u < kEmbedFlight; ++u) mx4_values8(v[u], w[u], s[u]);
      } else {
        Raw8<S> raw[kEmbedFlight];
        const auto *x = static_cast<const typename FloatType<S>::type *>(a.table) + (in ? id : 0) * a.stride;
#pragma unroll
        for (int u = 0; u < kEmbedFlight; ++u)
          load_raw8<S>(raw[u], x, 128 * (t + u) + 8 * r, in && t + u < t1 ? a.dim : 0);
#pragma unroll
        for (int u = 0; u < kEmbedFlight; ++u) raw_values<S>(v[u], raw[u]);
      }
#pragma unroll
      for (int u = 0; u < kEmbedFlight; ++u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[u][j] = in ? v[u][j] * a.scale : 0.f;
          // a float32 product for float16 results too, which else are rounded from the exact one
          if constexpr (T == RSLM_F16) asm("" : "+v"(v[u][j]));
        }
        store_float8<T>(v[u], o, 128 * (t + u) + 8 * r, t + u < t1 ? a.dim : 0);
      }
    }
  }
}

// ---- the sort
//
// Of 65,536 entries two passes, each a kernel of 5 us that counts and one of 11 that moves,
// bound by their chains of reads, barriers and votes; beside the latter the table is filled
// with zeros, by workgroups of their own.  Up to 8,192 entries take one kernel, of one
// workgroup, its entries and counts in LDS: whole gradients of 131,072 x 96 with 4,096 entries
// in 24 us, 37 with two kernels a pass; with 8,192 in 31, 38.

// A token of the sort: its id (the number of rows: none) and its place.
typedef uint2 Entry;   // x: id, y: place

constexpr int kSortThreads = 256;
constexpr int kSortEach = 8;                                 // entries of a thread
constexpr int kSortRound = kSortThreads * kSortEach;         // entries of a workgroup's round
constexpr int kSortMaxBits = 9;
constexpr int kSortMaxBins = 1 << kSortMaxBits;
constexpr int kSortMaxTiles = 256;
constexpr int kSortSmall = 1024 * kSortEach;                 // entries that one workgroup sorts

// A part of the table's rows, to be filled with zeros by the workgroups past `from`.
struct Fill {
  void *table;
  int64_t row0, row1, stride;
  int dim, type, from;
};

__device__ __forceinline__ void fill_rows(const Fill &f) {
  const float zero[8] = {};
  const int pieces = (f.dim + 7) / 8;
  const int64_t n = (f.row1 - f.row0) * pieces, step = int64_t(gridDim.x - f.from) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x - f.from) * blockDim.x + threadIdx.x; i < n; i += step) {
    const int64_t row = i / pieces;
    const int c = int(i - row * pieces) * 8;
    if (f.type == RSLM_F32)
      store_float8<RSLM_F32>(zero, static_cast<float *>(f.table) + (f.row0 + row) * f.stride, c, f.dim);
    else
      store_float8<RSLM_F16>(zero, static_cast<uint16_t *>(f.table) + (f.row0 + row) * f.stride, c, f.dim);
  }
}

__global__ void __launch_bounds__(256) k_embed_fill(Fill f) { fill_rows(f); }

struct SortArgs {
  const void *ids;         // of the first pass; null: entries
  int wide;
  int64_t rows;
  const Entry *in;
  Entry *out;
  int64_t n, per;          // per: entries of a workgroup, a multiple of kSortRound
  int shift, bits, tiles;
  uint32_t *counts;        // tiles x bins
  Fill fill;
};

__device__ __forceinline__ Entry id_entry(const SortArgs &a, int64_t i) {
  const int64_t id = id_at(a.ids, a.wide, i);
  return make_uint2(id >= 0 && id < a.rows ? uint32_t(id) : uint32_t(a.rows), uint32_t(i));
}
__device__ __forceinline__ Entry sort_entry(const SortArgs &a, int64_t i) { return a.ids ? id_entry(a, i) : a.in[i]; }

// How many entries of a workgroup's run have each digit.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs a) {
  __shared__ uint32_t bins[kSortMaxBins];
  const int nb = 1 << a.bits;
  for (int b = threadIdx.x; b < nb; b += kSortThreads) bins[b] = 0u;
  __syncthreads();
  const int64_t i0 = int64_t(blockIdx.x) * a.per, i1 = min(a.n, i0 + a.per);
  for (int64_t r0 = i0; r0 < i1; r0 += kSortRound) {
    Entry e[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const int64_t i = r0 + k * kSortThreads + threadIdx.x;
      e[k] = i < i1 ? sort_entry(a, i) : make_uint2(0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      if (r0 + k * kSortThreads + threadIdx.x < i1) atomicAdd(&bins[(e[k].x >> a.shift) & (nb - 1)], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < nb; b += kSortThreads) a.counts[int64_t(blockIdx.x) * nb + b] = bins[b];
}

template <int THREADS>
struct SortSmem {
  uint32_t start[kSortMaxBins];                // of this workgroup's next entry of a digit
  uint32_t own[THREADS / 64][kSortMaxBins];    // counts, then places, of a wavefront's entries
  uint32_t sums[THREADS / 64];
};

// sm.start: the sum of total over the lower digits, plus before.  Thread t has the digits
// 2 t and 2 t + 1 (`each` 2), or t.
template <int THREADS>
__device__ __forceinline__ void sort_starts(SortSmem<THREADS> &sm, const uint32_t (&total)[2], const uint32_t (&before)[2],
                                            int each, int nb) {
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t mine = total[0] + total[1];
  uint32_t upto = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(upto, off, 64);
    upto += lane >= off ? o : 0u;
  }
  if (lane == 63) sm.sums[tid >> 6] = upto;
  __syncthreads();
  uint32_t at = upto - mine;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) at += w < (tid >> 6) ? sm.sums[w] : 0u;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int b = tid * each + q;
    if (q < each && b < nb) sm.start[b] = at + before[q];
    at += total[q];
  }
}

// A round's `count` entries e to their places.  A wavefront has 64 kSortEach consecutive
// ones, 64 at a time; lanes with the same digit are found by a vote on each of its bits.
// sm.start moves on.
template <int THREADS, class Out>
__device__ __forceinline__ void sort_round(SortSmem<THREADS> &sm, const Entry (&e)[kSortEach], int count, int shift, int bits,
                                           Out &&out) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, nb = 1 << bits;
  for (int b = tid; b < nb; b += THREADS)
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) sm.own[w][b] = 0u;
  __syncthreads();
  const int first = wid * (64 * kSortEach) + lane;
#pragma unroll
  for (int k = 0; k < kSortEach; ++k)
    if (first + 64 * k < count) atomicAdd(&sm.own[wid][(e[k].x >> shift) & (nb - 1)], 1u);
  __syncthreads();
  for (int b = tid; b < nb; b += THREADS) {
    uint32_t p = sm.start[b];
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      const uint32_t c = sm.own[w][b];
      sm.own[w][b] = p;
      p += c;
    }
    sm.start[b] = p;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) {
    const bool on = first + 64 * k < count;
    const uint32_t d = (e[k].x >> shift) & (nb - 1);
    uint64_t same = __ballot(on);
#pragma unroll
    for (int bit = 0; bit < kSortMaxBits; ++bit)
      if (bit < bits) {
        const uint64_t set = __ballot(d >> bit & 1);   // that of lanes without an entry does not matter
        same &= (d >> bit & 1) ? set : ~set;
      }
    if (on) {
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const uint32_t p = sm.own[wid][d] + rank;
      out(p, e[k]);
      // the wavefront's reads of this step come before the write, its next ones after
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (rank == 0) sm.own[wid][d] = p + __popcll(same);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();
}

// Entries to their places: behind those of lower digits, those of the same digit in the
// workgroups before this one, and those of the same digit before it here.
__global__ void __launch_bounds__(kSortThreads) k_sort_move(SortArgs a) {
  if (int(blockIdx.x) >= a.tiles) return fill_rows(a.fill);
  __shared__ SortSmem<kSortThreads> sm;
  const int nb = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t i0 = int64_t(blockIdx.x) * a.per, i1 = min(a.n, i0 + a.per);
  Entry e[kSortEach];
  auto read = [&](int64_t r0) {
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const int64_t i = r0 + wid * (64 * kSortEach) + lane + 64 * k;
      e[k] = i < i1 ? sort_entry(a, i) : make_uint2(0u, 0u);
    }
  };
  read(i0);
  const int each = nb > kSortThreads ? 2 : 1;   // neighbouring digits of a thread
  uint32_t total[2] = {}, before[2] = {};
  if (tid * each < nb) {
    const uint32_t *c = a.counts + tid * each;
    constexpr int U = 32;   // tiles' counts asked for at once
    for (int t0 = 0; t0 < a.tiles; t0 += U) {
      uint32_t v[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = int64_t(min(t0 + u, a.tiles - 1)) * nb;
        v[u][0] = c[at];
        v[u][1] = c[at + each - 1];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint32_t w = t0 + u < a.tiles && q < each ? v[u][q] : 0u;
          total[q] += w;
          before[q] += t0 + u < int(blockIdx.x) ? w : 0u;
        }
    }
  }
  sort_starts(sm, total, before, each, nb);
  for (int64_t r0 = i0; r0 < i1; r0 += kSortRound) {
    if (r0 > i0) read(r0);
    sort_round(sm, e, int(i1 - r0 < kSortRound ? i1 - r0 : kSortRound), a.shift, a.bits,
               [&](uint32_t p, const Entry &v) { a.out[p] = v; });
  }
}

// All passes over one round's entries, in LDS.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_sort_small(SortArgs a, int passes) {
  if (int(blockIdx.x) >= 1) return fill_rows(a.fill);
  __shared__ SortSmem<THREADS> sm;
  __shared__ Entry held[THREADS * kSortEach];
  const int nb = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = int(a.n);
  const int first = wid * (64 * kSortEach) + lane;
  Entry e[kSortEach];
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) e[k] = first + 64 * k < n ? id_entry(a, first + 64 * k) : make_uint2(0u, 0u);
  const int each = nb > THREADS ? 2 : 1;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * a.bits;
    for (int b = tid; b < nb; b += THREADS) sm.start[b] = 0u;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      if (first + 64 * k < n) atomicAdd(&sm.start[(e[k].x >> shift) & (nb - 1)], 1u);
    __syncthreads();
    uint32_t total[2] = {}, before[2] = {};
#pragma unroll
    for (int q = 0; q < 2; ++q)
      if (q < each && tid * each + q < nb) total[q] = sm.start[tid * each + q];
    sort_starts(sm, total, before, each, nb);   // a barrier between these reads and its writes
    if (pass + 1 < passes) {
      sort_round(sm, e, n, shift, a.bits, [&](uint32_t p, const Entry &v) { held[p] = v; });
#pragma unroll
      for (int k = 0; k < kSortEach; ++k)
        if (first + 64 * k < n) e[k] = held[first + 64 * k];
    } else {
      sort_round(sm, e, n, shift, a.bits, [&](uint32_t p, const Entry &v) { a.out[p] = v; });
    }
  }
}

// ---- sums over runs

struct EmbedSumArgs {
  const Entry *sorted;
  int64_t n;
  uint32_t rows;
  int chunk;               // entries of a wavefront
  int64_t chunks;
  const void *dout;
  int64_t stride;
  int dim;
  float scale;
  int add;                 // to what dtable holds
  void *dtable;
  int64_t dstride;
  float *head, *tail;      // chunks x dim: the sums of a run that began before, that goes on
};

constexpr int kSumCols = 512;   // columns of a wavefront
constexpr int kSumFlight = 4;   // rows asked for at once, twice

// A lane's 8 columns of a row: those from `at` on, of which the first `skip` are another
// lane's.  So a row's last columns too are read and written 8 at a time, and no branch
// keeps a wavefront's loads apart (65,536 x 768 bfloat16 45 us, 2.2 TB/s of dout alone; 68
// with a branch for the last columns).  Rows of less than 8: WIDE false.
struct SumLane {
  int at, skip;
};
__device__ __forceinline__ SumLane sum_lane(int dim) {
  const int c = int(blockIdx.y) * kSumCols + 8 * int(threadIdx.x & 63);
  const int at = min(c, dim - 8);
  return SumLane{at, min(c - at, 8)};
}
template <int T, bool WIDE>
__device__ __forceinline__ void sum_load(Raw8<T> &p, const void *row, const SumLane &l, int dim) {
  typedef typename FloatType<T>::type F;
  if constexpr (!WIDE) {
    load_raw8<T>(p, row, 0, dim);
  } else if constexpr (T == RSLM_F32) {
    const F32x8u a = *reinterpret_cast<const F32x8u *>(static_cast<const F *>(row) + l.at);
    __builtin_memcpy(&p, &a, sizeof(a));
  } else {
    const H16x8u a = *reinterpret_cast<const H16x8u *>(static_cast<const F *>(row) + l.at);
    __builtin_memcpy(&p, &a, sizeof(a));
  }
}
template <int T, bool WIDE>
__device__ __forceinline__ void sum_store(const float (&v)[8], void *row, const SumLane &l, int dim) {
  if constexpr (!WIDE) {
    if (l.skip == 0) store_float8<T>(v, row, 0, dim);
  } else if (l.skip == 0) {
    store_float8<T>(v, row, l.at, dim);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= l.skip) store_float<T>(row, l.at + i, v[i]);
  }
}

template <int TO, bool WIDE>
__device__ __forceinline__ void put_row(const EmbedSumArgs &a, uint32_t id, const SumLane &l, const float (&acc)[8]) {
  typename FloatType<TO>::type *o = static_cast<typename FloatType<TO>::type *>(a.dtable) + int64_t(id) * a.dstride;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = acc[i] * a.scale;
  if (a.add) {
    Raw8<TO> old;
    sum_load<TO, WIDE>(old, o, l, a.dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += float(old.v[i]);
  }
  sum_store<TO, WIDE>(v, o, l, a.dim);
}

// A wavefront: `chunk` sorted entries by 512 columns.  Runs inside them go to the table,
// those that begin before or go on after to `head` and `tail`.
template <int T, int TO, bool WIDE>
__global__ void __launch_bounds__(256) k_embed_sum(EmbedSumArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t chunk = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  const int64_t e0 = chunk * a.chunk, e1 = min(a.n, e0 + a.chunk);
  SumLane l = sum_lane(WIDE ? a.dim : 8);
  if (!WIDE) l.skip = lane ? 8 : 0;
  const uint32_t none = a.rows;
  uint32_t id = e0 > 0 ? a.sorted[e0 - 1].x : none;   // of the run that acc sums
  bool from_before = true;
  float acc[8] = {};
  for (int64_t b = e0; b < e1; b += 64) {
    const int count = int(e1 - b < 64 ? e1 - b : 64);
    Entry mine = make_uint2(none, 0u);
    if (lane < count) mine = a.sorted[b + lane];
    Raw8<T> raw[2][kSumFlight];
    auto fetch = [&](int set, int k) {
#pragma unroll
      for (int u = 0; u < kSumFlight; ++u) {
        // behind the last entry, that one's row again; of one outside the table its row, unused
        const uint32_t place = __builtin_amdgcn_readlane(mine.y, min(k + u, count - 1));
        sum_load<T, WIDE>(raw[set][u], static_cast<const typename FloatType<T>::type *>(a.dout) + int64_t(place) * a.stride,
                          l, a.dim);
      }
    };
    fetch(0, 0);
    for (int k0 = 0; k0 < count; k0 += 2 * kSumFlight) {
#pragma unroll
      for (int set = 0; set < 2; ++set) {
        const int k = k0 + set * kSumFlight;
        fetch(set ^ 1, k + kSumFlight);
#pragma unroll
        for (int u = 0; u < kSumFlight; ++u) {
          if (k + u >= count) break;
          const uint32_t next = __builtin_amdgcn_readlane(mine.x, k + u);
          if (next != id) {
            if (b + k + u > e0 && id != none) {
              if (from_before) sum_store<RSLM_F32, WIDE>(acc, a.head + chunk * a.dim, l, a.dim);
              else put_row<TO, WIDE>(a, id, l, acc);
            }
            id = next;
            from_before = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += float(raw[set][u].v[i]);
        }
      }
    }
  }
  if (id == none) return;
  const bool goes_on = e1 < a.n && a.sorted[e1].x == id;
  if (from_before) sum_store<RSLM_F32, WIDE>(acc, a.head + chunk * a.dim, l, a.dim);
  else if (goes_on) sum_store<RSLM_F32, WIDE>(acc, a.tail + chunk * a.dim, l, a.dim);
  else put_row<TO, WIDE>(a, id, l, acc);
}

// Runs over several chunks: the tail of the one that they begin in, and the heads after
// it, every fourth of them to a wavefront.
constexpr int kJoinWaves = 4;
template <int TO, bool WIDE>
__global__ void __launch_bounds__(64 * kJoinWaves) k_embed_join(EmbedSumArgs a) {
  __shared__ float sums[kJoinWaves - 1][kSumCols];
  __shared__ int ends;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t chunk = blockIdx.x, e0 = chunk * a.chunk, e1 = e0 + a.chunk;
  const uint32_t id = a.sorted[e1 - 1].x;
  const uint32_t behind = a.sorted[e1].x, ahead = e0 > 0 ? a.sorted[e0 - 1].x : a.rows;
  if (id == a.rows || behind != id || ahead == id) return;   // ends here, or began before
  // the last head: that of the first chunk whose end is not the run's
  int64_t last = chunk + 1;
  for (;; last += 64 * kJoinWaves) {
    if (tid == 0) ends = 64 * kJoinWaves;
    __syncthreads();
    const int64_t end = (last + tid + 1) * a.chunk;
    if (end >= a.n || a.sorted[end].x != id) atomicMin(&ends, tid);
    __syncthreads();
    const int first = ends;
    __syncthreads();
    if (first < 64 * kJoinWaves) {
      last += first;
      break;
    }
  }
  SumLane l = sum_lane(WIDE ? a.dim : 8);
  if (!WIDE) l.skip = lane ? 8 : 0;
  float acc[8] = {};
  if (wid == 0) {
    Raw8<RSLM_F32> v;
    sum_load<RSLM_F32, WIDE>(v, a.tail + chunk * a.dim, l, a.dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = v.v[i];
  }
  constexpr int U = 4;   // heads asked for at once
  for (int64_t j = chunk + 1 + wid; j <= last; j += kJoinWaves * U) {
    Raw8<RSLM_F32> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      sum_load<RSLM_F32, WIDE>(v[u], a.head + min(j + kJoinWaves * u, last) * a.dim, l, a.dim);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += j + kJoinWaves * u <= last ? v[u].v[i] : 0.f;
  }
  if (wid > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wid - 1][8 * lane + i] = acc[i];
  }
  __syncthreads();
  if (wid > 0) return;
#pragma unroll
  for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += sums[w][8 * lane + i];
  put_row<TO, WIDE>(a, id, l, acc);
}

// ---- host

struct EmbedPlan {
  int passes, bits, tiles, chunk;
  int64_t per, chunks;
  size_t entries, counts, sums, total;   // bytes
};

static size_t rounded(size_t b) { return (b + 255) / 256 * 256; }

static EmbedPlan embed_plan(int64_t n, int64_t rows, int dim) {
  EmbedPlan p{};
  int bits = 1;
  while (bits < 32 && (uint64_t(rows) >> bits)) ++bits;   // of 0 .. rows
  p.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  const int64_t rounds = (n + kSortRound - 1) / kSortRound;
  p.per = (rounds + kSortMaxTiles - 1) / kSortMaxTiles * kSortRound;
  p.tiles = p.per ? int((n + p.per - 1) / p.per) : 0;
  if (n <= kSortSmall) p.tiles = 1;
  // 8 wavefronts to a CU, chunks of 8 to 512 entries; up to 16 in one, which has nothing to
  // join (11 of 12,000 x 512: 13.2 us, 16.4 in two; 32 of 12,000 x 64: 19.3 in one, 16.3)
  const int64_t cols = (dim + kSumCols - 1) / kSumCols;
  p.chunk = n <= 16 ? 16 : 8;
  while (p.chunk < 512 && (n + p.chunk - 1) / p.chunk * cols > 2048) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  p.entries = rounded(size_t(n) * sizeof(Entry));
  p.counts = rounded(size_t(p.tiles) * (size_t(1) << p.bits) * 4);
  p.sums = rounded(size_t(p.chunks) * dim * 4);
  p.total = 2 * p.entries + p.counts + 2 * p.sums;
  return p;
}

// grid: one workgroup that sorts, and others of 256 threads that fill.
template <int THREADS>
static void launch_sort_small(const SortArgs &a, int passes, dim3 grid, hipStream_t s) {
  const unsigned fill = (grid.x - 1 + THREADS / 256 - 1) / (THREADS / 256);
  hipLaunchKernelGGL(k_sort_small<THREADS>, dim3(1 + fill), dim3(THREADS), 0, s, a, passes);
}

template <int T, int TO, bool WIDE>
static void launch_sums_one(const EmbedSumArgs &a, hipStream_t s) {
  const dim3 grid(unsigned((a.chunks + 3) / 4), unsigned((a.dim + kSumCols - 1) / kSumCols));
  hipLaunchKernelGGL((k_embed_sum<T, TO, WIDE>), grid, dim3(256), 0, s, a);
  // the last chunk has none after it
  if (a.chunks > 1)
    hipLaunchKernelGGL((k_embed_join<TO, WIDE>), dim3(unsigned(a.chunks - 1), grid.y),
                       dim3(64 * kJoinWaves), 0, s, a);
}
template <int T, int TO>
static void launch_sums(const EmbedSumArgs &a, hipStream_t s) {
  if (a.dim >= 8) launch_sums_one<T, TO, true>(a, s);
  else launch_sums_one<T, TO, false>(a, s);
}

template <int S>
static void launch_embed(const EmbedArgs &a, int dtype, hipStream_t s) {
  const int64_t wg = (a.n + 15) / 16;
  const dim3 grid(unsigned(wg < (1 << 20) ? wg : (1 << 20)), unsigned((a.steps + a.each - 1) / a.each));
  if (dtype == RSLM_F32) hipLaunchKernelGGL((k_embed<S, RSLM_F32>), grid, dim3(256), 0, s, a);
  else if (dtype == RSLM_F16) hipLaunchKernelGGL((k_embed<S, RSLM_F16>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_embed<S, RSLM_BF16>), grid, dim3(256), 0, s, a);
}

static int embed_each(int64_t n, int steps) {
  const int64_t rows = (n + 15) / 16, runs = (4096 + rows - 1) / rows, each = (steps + runs - 1) / runs;
  return int(each < kEmbedFlight ? kEmbedFlight : each);
}

static bool embed_sizes_ok(int64_t n, int64_t rows, int dim) {
  return n >= 0 && n <= kMx4MaxRows && rows >= 0 && rows <= kMx4MaxRows && dim >= 1 && dim <= kMx4MaxDim;
}

static int embed_call(EmbedArgs a, int stype, int out_dtype, void *stream) {
  a.steps = mx4_steps(a.dim);
  a.each = embed_each(a.n, a.steps);
  const hipStream_t s = as_stream(stream);
  if (stype == RSLM_F32) launch_embed<RSLM_F32>(a, out_dtype, s);
  else if (stype == RSLM_F16) launch_embed<RSLM_F16>(a, out_dtype, s);
  else if (stype == RSLM_BF16) launch_embed<RSLM_BF16>(a, out_dtype, s);
  else launch_embed<kMx4Table>(a, out_dtype, s);
  return check_launch();
}

// Workgroups that fill rows with zeros, 8 values a thread: with more of them the sort's
// reads beside wait longer (65,536 x 768 with the lookup: 138 us, 144 with 2,048, 146 with 256).
static unsigned fill_groups(int64_t rows, int dim) {
  const int64_t wg = (rows * ((dim + 7) / 8) + 255) / 256;
  return unsigned(wg < 512 ? wg : 512);
}

static bool ids_ok(const void *ids, int id_bytes) { return ids && aligned_to(ids, id_bytes); }

}  // namespace rslm

using namespace rslm;

extern "C" {

int rslm_embed(const void *table, int32_t dtype, int64_t rows, int32_t dim, int64_t stride, const void *ids,
               int32_t id_bytes, int64_t n, float scale, void *out, int32_t out_dtype, int64_t out_stride,
               void *stream) {
  if (!embed_sizes_ok(n, rows, dim) || !float_type_ok(dtype) || !float_type_ok(out_dtype) || stride < 0 ||
      (id_bytes != 4 && id_bytes != 8) || (n > 1 && out_stride < dim))
    return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;
  if ((rows > 0 && !table) || !out || !ids_ok(ids, id_bytes) || !aligned_to(table, float_bytes(dtype)) ||
      !aligned_to(out, float_bytes(out_dtype)))
    return RSLM_ERR_INVALID_ARG;
  return embed_call(EmbedArgs{table, nullptr, rows, stride, ids, id_bytes == 8, n, dim, 0, 0, scale, out, out_stride},
                    dtype, out_dtype, stream);
}

int rslm_mx4_embed(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t dim, const void *ids,
                   int32_t id_bytes, int64_t n, float scale, void *out, int32_t out_dtype, int64_t out_stride,
                   void *stream) {
  if (!embed_sizes_ok(n, rows, dim) || !float_type_ok(out_dtype) || (id_bytes != 4 && id_bytes != 8) ||
      (n > 1 && out_stride < dim))
    return RSLM_ERR_INVALID_ARG;
  if (n == 0) return RSLM_OK;
  if ((rows > 0 && (!codes || !scales)) || !out || !ids_ok(ids, id_bytes) || !aligned_to(codes, 16) ||
      !aligned_to(scales, 4) || !aligned_to(out, float_bytes(out_dtype)))
    return RSLM_ERR_INVALID_ARG;
  return embed_call(EmbedArgs{codes, scales, rows, 0, ids, id_bytes == 8, n, dim, 0, 0, scale, out, out_stride},
                    kMx4Table, out_dtype, stream);
}

size_t rslm_embed_backward_workspace(int64_t n, int64_t rows, int32_t dim) {
  if (!embed_sizes_ok(n, rows, dim) || n == 0) return 0;
  return embed_plan(n, rows, dim).total;
}

int rslm_embed_backward(const void *dout, int32_t dtype, int64_t n, int32_t dim, int64_t stride, const void *ids,
                        int32_t id_bytes, int64_t rows, float scale, int32_t accumulate, void *dtable,
                        int32_t table_dtype, int64_t table_stride, void *ws, size_t ws_bytes, void *stream) {
  if (!embed_sizes_ok(n, rows, dim) || !float_type_ok(dtype) || !float_type_ok(table_dtype) || stride < 0 ||
      (id_bytes != 4 && id_bytes != 8) || (rows > 1 && table_stride < dim))
    return RSLM_ERR_INVALID_ARG;
  if (table_dtype != RSLM_F32 && table_dtype != dtype) return RSLM_ERR_UNSUPPORTED;
  if (rows == 0 || (n == 0 && accumulate)) return RSLM_OK;
  if (!dtable || !aligned_to(dtable, float_bytes(table_dtype)) ||
      (n > 0 && (!dout || !ids_ok(ids, id_bytes) || !aligned_to(dout, float_bytes(dtype)))))
    return RSLM_ERR_INVALID_ARG;
  const EmbedPlan p = embed_plan(n, rows, dim);
  if (n > 0 && ws_bytes < p.total) return RSLM_ERR_WORKSPACE;
  if (n > 0 && (!ws || !aligned_to(ws, 16))) return RSLM_ERR_INVALID_ARG;
  const hipStream_t s = as_stream(stream);
  if (n == 0) {
    const dim3 grid(fill_groups(rows, dim));
    hipLaunchKernelGGL(k_embed_fill, grid, dim3(256), 0, s, Fill{dtable, 0, rows, table_stride, dim, table_dtype, 0});
    return check_launch();
  }
  char *w = static_cast<char *>(ws);
  Entry *in = reinterpret_cast<Entry *>(w), *out = reinterpret_cast<Entry *>(w + p.entries);
  SortArgs a{ids, id_bytes == 8, rows, in, out, n, p.per, 0, p.bits, p.tiles,
             reinterpret_cast<uint32_t *>(w + 2 * p.entries)};
  // a part of the table's rows is filled beside each pass's longer kernel
  const int64_t parts = p.tiles == 1 ? 1 : p.passes;
  int64_t part = 0;
  auto grid = [&] {
    const int64_t row0 = rows * part / parts, row1 = rows * (part + 1) / parts;
    ++part;
    a.fill = Fill{dtable, row0, row1, table_stride, dim, table_dtype, p.tiles};
    return dim3(unsigned(p.tiles) + (accumulate ? 0u : fill_groups(row1 - row0, dim)));
  };
  if (p.tiles == 1) {
    if (n <= 256 * kSortEach) launch_sort_small<256>(a, p.passes, grid(), s);
    else if (n <= 512 * kSortEach) launch_sort_small<512>(a, p.passes, grid(), s);
    else launch_sort_small<1024>(a, p.passes, grid(), s);
    a.in = a.out;
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      hipLaunchKernelGGL(k_sort_count, dim3(unsigned(p.tiles)), dim3(kSortThreads), 0, s, a);
      const dim3 g1 = grid();
      hipLaunchKernelGGL(k_sort_move, g1, dim3(kSortThreads), 0, s, a);
      a.ids = nullptr;
      a.shift += p.bits;
      const Entry *sorted = a.out;
      a.out = const_cast<Entry *>(a.in);
      a.in = sorted;
    }
  }
  float *sums = reinterpret_cast<float *>(w + 2 * p.entries + p.counts);
  const EmbedSumArgs b{a.in,  n,   uint32_t(rows), p.chunk, p.chunks,     dout,   stride,
                       dim,   scale, accumulate,   dtable,  table_stride, sums,
                       reinterpret_cast<float *>(reinterpret_cast<char *>(sums) + p.sums)};
  if (dtype == RSLM_F32) launch_sums<RSLM_F32, RSLM_F32>(b, s);
  else if (dtype == RSLM_F16 && table_dtype == RSLM_F32) launch_sums<RSLM_F16, RSLM_F32>(b, s);
  else if (dtype == RSLM_F16) launch_sums<RSLM_F16, RSLM_F16>(b, s);
  else if (table_dtype == RSLM_F32) launch_sums<RSLM_BF16, RSLM_F32>(b, s);
  else launch_sums<RSLM_BF16, RSLM_BF16>(b, s);
  return check_launch();
}

}  // extern "C"
