// Rows of a table for given tokens, out_i = scale table[id_i] (0 for a token outside the
// table), and the gradient of a float table, dtable_v = scale sum over i with id_i = v of
// dout_i.
//
// Forward: bound by memory, a row read and written for each token.
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

// A token of the sort: its id (the number of rows: none) and its place.
typedef uint2 Entry;   // x: id, y: place

constexpr int kSortThreads = 256;
constexpr int kSortEach = 16;                                // entries of a thread
constexpr int kSortRound = kSortThreads * kSortEach;         // entries of a workgroup's round
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortMaxBits = 9;
constexpr int kSortMaxBins = 1 << kSortMaxBits;
constexpr int kSortMaxTiles = 256;

struct SortArgs {
  const void *ids;         // of the first pass; null: entries
  int wide;
  int64_t rows;
  const Entry *in;
  Entry *out;
  int64_t n, per;          // per: entries of a workgroup, a multiple of kSortRound
  int shift, bits, tiles;
  uint32_t *counts;        // tiles x bins
};

__device__ __forceinline__ Entry sort_entry(const SortArgs &a, int64_t i) {
  if (!a.ids) return a.in[i];
  const int64_t id = id_at(a.ids, a.wide, i);
  return make_uint2(id >= 0 && id < a.rows ? uint32_t(id) : uint32_t(a.rows), uint32_t(i));
}

// How many entries of a workgroup's run have each digit.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs a) {
  __shared__ uint32_t bins[kSortMaxBins];
  const int nb = 1 << a.bits;
  for (int b = threadIdx.x; b < nb; b += kSortThreads) bins[b] = 0u;
  __syncthreads();
  const int64_t i0 = int64_t(blockIdx.x) * a.per, i1 = min(a.n, i0 + a.per);
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads)
    atomicAdd(&bins[(sort_entry(a, i).x >> a.shift) & (nb - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < nb; b += kSortThreads) a.counts[int64_t(blockIdx.x) * nb + b] = bins[b];
}

// Entries to their places: behind those of lower digits, those of the same digit in the
// workgroups before this one, and those of the same digit before it here.  A wavefront
// takes 16 x 64 consecutive entries of a round; lanes with the same digit are found by a
// vote on each of its bits.
__global__ void __launch_bounds__(kSortThreads) k_sort_move(SortArgs a) {
  __shared__ uint32_t start[kSortMaxBins];              // of this workgroup's next entry of a digit
  __shared__ uint32_t own[kSortWaves][kSortMaxBins];    // counts, then places, of a wavefront's entries
  __shared__ uint32_t sums[kSortThreads];
  const int nb = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  // each thread: neighbouring digits
  const int each = (nb + kSortThreads - 1) / kSortThreads;
  uint32_t total[2] = {}, before[2] = {};
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int b = tid * each + q;
    if (q < each && b < nb)
      for (int t = 0; t < a.tiles; ++t) {
        const uint32_t c = a.counts[int64_t(t) * nb + b];
        total[q] += c;
        before[q] += t < int(blockIdx.x) ? c : 0u;
      }
  }
  uint32_t sum = total[0] + total[1];
  sums[tid] = sum;
  __syncthreads();
  for (int off = 1; off < kSortThreads; off <<= 1) {
    const uint32_t o = tid >= off ? sums[tid - off] : 0u;
    __syncthreads();
    sum += o;
    sums[tid] = sum;
    __syncthreads();
  }
  uint32_t at = sum - total[0] - total[1];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int b = tid * each + q;
    if (q < each && b < nb) start[b] = at + before[q];
    at += total[q];
  }
  const int64_t i0 = int64_t(blockIdx.x) * a.per, i1 = min(a.n, i0 + a.per);
  for (int64_t r0 = i0; r0 < i1; r0 += kSortRound) {
    for (int b = tid; b < nb; b += kSortThreads)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) own[w][b] = 0u;
    __syncthreads();
    Entry e[kSortEach];
    const int64_t w0 = r0 + wid * (64 * kSortEach) + lane;
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const int64_t i = w0 + 64 * k;
      e[k] = i < i1 ? sort_entry(a, i) : make_uint2(0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      if (w0 + 64 * k < i1) atomicAdd(&own[wid][(e[k].x >> a.shift) & (nb - 1)], 1u);
    __syncthreads();
    for (int b = tid; b < nb; b += kSortThreads) {
      uint32_t p = start[b];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = own[w][b];
        own[w][b] = p;
        p += c;
      }
      start[b] = p;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const bool on = w0 + 64 * k < i1;
      const uint32_t d = (e[k].x >> a.shift) & (nb - 1);
      uint64_t same = __ballot(on);
      for (int bit = 0; bit < a.bits; ++bit) {
        const uint64_t set = __ballot(on && (d >> bit & 1));
        same &= (d >> bit & 1) ? set : ~set;
      }
      if (on) {
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const uint32_t p = own[wid][d] + rank;
        a.out[p] = e[k];
        // the wavefront's reads of this step come before the write, its next ones after
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (rank == 0) own[wid][d] = p + __popcll(same);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
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
constexpr int kSumFlight = 4;   // rows asked for at once

template <int TO>
__device__ __forceinline__ void put_row(const EmbedSumArgs &a, uint32_t id, int c, const float (&acc)[8]) {
  typename FloatType<TO>::type *o = static_cast<typename FloatType<TO>::type *>(a.dtable) + int64_t(id) * a.dstride;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = acc[i] * a.scale;
  if (a.add) {
    float old[8];
    load_float8<TO>(old, o, c, a.dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += old[i];
  }
  store_float8<TO>(v, o, c, a.dim);
}

template <int TO>
__global__ void __launch_bounds__(256) k_embed_fill(void *p, int64_t rows, int64_t stride, int dim) {
  const float zero[8] = {};
  const int pieces = (dim + 7) / 8;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < rows * pieces; i += int64_t(gridDim.x) * 256) {
    const int64_t row = i / pieces;
    store_float8<TO>(zero, static_cast<typename FloatType<TO>::type *>(p) + row * stride, int(i - row * pieces) * 8, dim);
  }
}

// A wavefront: `chunk` sorted entries by 512 columns.  Runs inside them go to the table,
// those that begin before or go on after to `head` and `tail`.
template <int T, int TO>
__global__ void __launch_bounds__(256) k_embed_sum(EmbedSumArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t chunk = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  const int64_t e0 = chunk * a.chunk, e1 = min(a.n, e0 + a.chunk);
  const int c = int(blockIdx.y) * kSumCols + 8 * lane;
  const uint32_t none = a.rows;
  uint32_t id = e0 > 0 ? a.sorted[e0 - 1].x : none;   // of the run that acc sums
  bool from_before = true;
  float acc[8] = {};
  for (int64_t b = e0; b < e1; b += 64) {
    const int count = int(e1 - b < 64 ? e1 - b : 64);
    Entry mine = make_uint2(none, 0u);
    if (lane < count) mine = a.sorted[b + lane];
    for (int k = 0; k < count; k += kSumFlight) {
      Raw8<T> raw[kSumFlight];
      uint32_t next[kSumFlight];
#pragma unroll
      for (int u = 0; u < kSumFlight; ++u) {
        const int at = min(k + u, count - 1);
        next[u] = __builtin_amdgcn_readlane(mine.x, at);
        const uint32_t place = __builtin_amdgcn_readlane(mine.y, at);
        // entries outside the table are last, and their rows are not read
        load_raw8<T>(raw[u], static_cast<const typename FloatType<T>::type *>(a.dout) + int64_t(place) * a.stride, c,
                     next[u] == none ? 0 : a.dim);
      }
#pragma unroll
      for (int u = 0; u < kSumFlight; ++u) {
        if (k + u >= count) break;
        if (next[u] != id) {
          if (b + k + u > e0 && id != none) {
            if (from_before) store_float8<RSLM_F32>(acc, a.head + chunk * a.dim, c, a.dim);
            else put_row<TO>(a, id, c, acc);
          }
          id = next[u];
          from_before = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = 0.f;
        }
        float v[8];
        raw_values<T>(v, raw[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[i];
      }
    }
  }
  if (id == none) return;
  const bool goes_on = e1 < a.n && a.sorted[e1].x == id;
  if (from_before) store_float8<RSLM_F32>(acc, a.head + chunk * a.dim, c, a.dim);
  else if (goes_on) store_float8<RSLM_F32>(acc, a.tail + chunk * a.dim, c, a.dim);
  else put_row<TO>(a, id, c, acc);
}

// Runs over several chunks: the tail of the one that they begin in, and the heads after it.
template <int TO>
__global__ void __launch_bounds__(256) k_embed_join(EmbedSumArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t chunk = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  const int64_t e0 = chunk * a.chunk, e1 = e0 + a.chunk;
  if (e1 >= a.n) return;
  const uint32_t id = a.sorted[e1 - 1].x;
  if (id == a.rows || a.sorted[e1].x != id) return;
  if (e0 > 0 && a.sorted[e0 - 1].x == id) return;   // began before
  const int c = int(blockIdx.y) * kSumCols + 8 * lane;
  float acc[8];
  load_float8<RSLM_F32>(acc, a.tail + chunk * a.dim, c, a.dim);
  for (int64_t j = chunk + 1;; ++j) {
    float v[8];
    load_float8<RSLM_F32>(v, a.head + j * a.dim, c, a.dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += v[i];
    const int64_t end = (j + 1) * a.chunk;
    if (end >= a.n || a.sorted[end].x != id) break;
  }
  put_row<TO>(a, id, c, acc);
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
  // 16 wavefronts to a CU, chunks of 16 to 512 entries
  const int64_t cols = (dim + kSumCols - 1) / kSumCols;
  p.chunk = 16;
  while (p.chunk < 512 && (n + p.chunk - 1) / p.chunk * cols > 8192) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  p.entries = rounded(size_t(n) * sizeof(Entry));
  p.counts = rounded(size_t(p.tiles) * (size_t(1) << p.bits) * 4);
  p.sums = rounded(size_t(p.chunks) * dim * 4);
  p.total = 2 * p.entries + p.counts + 2 * p.sums;
  return p;
}

template <int T, int TO>
static void launch_sums(const EmbedSumArgs &a, hipStream_t s) {
  const dim3 grid(unsigned((a.chunks + 3) / 4), unsigned((a.dim + kSumCols - 1) / kSumCols));
  hipLaunchKernelGGL((k_embed_sum<T, TO>), grid, dim3(256), 0, s, a);
  if (a.chunks > 1) hipLaunchKernelGGL(k_embed_join<TO>, grid, dim3(256), 0, s, a);
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
  if (!accumulate) {
    const int64_t pieces = rows * ((dim + 7) / 8), wg = (pieces + 255) / 256;
    const dim3 grid(unsigned(wg < 8192 ? wg : 8192));
    if (table_dtype == RSLM_F32)
      hipLaunchKernelGGL(k_embed_fill<RSLM_F32>, grid, dim3(256), 0, s, dtable, rows, table_stride, dim);
    else
      hipLaunchKernelGGL(k_embed_fill<RSLM_F16>, grid, dim3(256), 0, s, dtable, rows, table_stride, dim);
  }
  if (n == 0) return check_launch();
  char *w = static_cast<char *>(ws);
  Entry *in = reinterpret_cast<Entry *>(w), *out = reinterpret_cast<Entry *>(w + p.entries);
  SortArgs a{ids, id_bytes == 8, rows, in, out, n, p.per, 0, p.bits, p.tiles,
             reinterpret_cast<uint32_t *>(w + 2 * p.entries)};
  for (int pass = 0; pass < p.passes; ++pass) {
    hipLaunchKernelGGL(k_sort_count, dim3(unsigned(p.tiles)), dim3(kSortThreads), 0, s, a);
    hipLaunchKernelGGL(k_sort_move, dim3(unsigned(p.tiles)), dim3(kSortThreads), 0, s, a);
    a.ids = nullptr;
    a.shift += p.bits;
    const Entry *sorted = a.out;
    a.out = const_cast<Entry *>(a.in);
    a.in = sorted;
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
