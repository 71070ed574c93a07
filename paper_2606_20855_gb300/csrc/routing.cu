// A routing matrix R transposed, and rows of dense matrices moved along it.
//
// R has a row per token and a column per expert.  Sorted by column (rows in
// order within a column) its entries are the rows of R^T: entry (i, e) has
//   slot = offsets[e] + entries of column e in the rows before i.
// A row stores a column at most once, so within a tile of 32 W rows an entry
// is one bit of a W-word bitmap per column, and the count of the rows before it
// is a population count: no sort, no order of atomics that matters.
//
// Rows move along R and R^T:
//   dispatch            xs[slot] = x[row]
//   its gradient        gx[i] = sum over row i of gxs[slot]
//   combine             y[i] = sum over row i of v ys[slot]
//   its gradient        gys[slot] = v gy[row],  gv = <gy[row], ys[slot]>
// All four go by the rows of R: a row's own side is read or written once, in
// one place, and sums of a row are taken in the order of its entries in 32 bits
// (one rounding, when stored), so equal inputs give equal bits.
// Entries whose column is no column of R have slot -1 and take no part.
#include <climits>

#include "routing.cuh"
#include "ws_internal.cuh"

namespace wsk {
namespace {

// ---------------------------------------------------------------- R transposed

// A tile is 32 rows for each warp of a CTA: 32 warps where one CTA builds the
// plan alone (a single launch), eight or 16 where many CTAs do (a launch that
// counts and one that places).  Bound by latencies, not bytes: 33 rows of eight
// entries over 64 columns 5 us in the single launch; in the two 8191 rows of
// eight over 64 columns 7 us, 16,385 rows of four over 257 columns 9 us.
constexpr int kSmallWarps = 32, kSmallRows = 32 * kSmallWarps;
// A tile's warps.  More of them make fewer chunks, whose counts every CTA adds up (rows / (32 W) times cols of them); fewer are less work
// for a CTA.  us with 8 | 16 warps: 8191 rows of four over 256 columns 7.7 | 8.1, 16,385 over 128 7.8 | 8.1, over 256 10.2 | 8.9,
// 65,537 over 96 13.8 | 10.0, of eight over 512 32 | 20; with 32 warps 13 for 16,385 over 257, where 16 take 9.
int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }
int build_warps(int64_t rows, int64_t cols) { return cols == 0 || rows < 3'000'000 / cols ? 8 : 16; }
constexpr int kHeld = 8;  // entries that a lane holds at once: loads in flight, and rows of 8 entries walked once

// The entries of a warp's 32 rows, kHeld a lane at a time.
struct WarpRows {
  int end;          // of the lane's row
  int64_t lo, hi;   // of all 32 rows
  int64_t first;    // their first row
  int col[kHeld];
  int row[kHeld];   // of 0..31; -1: no entry
  __device__ __forceinline__ void start(const ws_routing& r, int64_t first_row) {
    const int lane = threadIdx.x & 31;
    first = first_row;
    int begin = 0;
    end = 0;
    lo = hi = 0;
    if (first < r.nrows) {
      entry_range(r.rowptr, min(first + lane, r.nrows - 1), r.nnz, &begin, &end);
      if (first + lane >= r.nrows) begin = end;
      lo = __shfl_sync(0xffffffffu, begin, 0);
      hi = __shfl_sync(0xffffffffu, end, 31);
    }
  }
  __device__ __forceinline__ void load(const ws_routing& r, int64_t base) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) col[i] = base + 32 * i + lane < hi ? r.colidx[base + 32 * i + lane] : -1;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int64_t e = base + 32 * i + lane;
      int n = 0;  // rows that end at or before e
#pragma unroll
      for (int step = 16; step; step >>= 1) {
        const int last = __shfl_sync(0xffffffffu, end, n + step - 1);
        if (last <= e) n += step;
      }
      row[i] = e < hi && first + n < r.nrows ? n : -1;
    }
  }
};

// Marks the columns of the warp's rows: bit i of mask[warp * cols + e] is its row i.
__device__ __forceinline__ void mark_rows(const ws_routing& r, WarpRows& w, int cols, uint32_t* mask) {
  uint32_t* word = mask + (threadIdx.x >> 5) * cols;
  for (int64_t base = w.lo; base < w.hi; base += 32 * kHeld) {
    w.load(r, base);
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (w.row[i] >= 0 && static_cast<unsigned>(w.col[i]) < static_cast<unsigned>(cols))
        atomicOr(word + w.col[i], 1u << w.row[i]);
  }
}

// Where entries are counted from: a + b, at most the number of entries.  Row pointers that decrease make warps whose ranges overlap,
// which count entries more than once; slots from nnz on are then nobody's, and offsets end at nnz.
__device__ __forceinline__ int slots_before(const ws_routing& r, int64_t a, int64_t b) { return static_cast<int>(min(a + b, r.nnz)); }

// Slots of the warp's rows; pre[warp * cols + e] plus first[e] is the slot of the warp's first entry of column e.  staged: what
// goes to the slots' arrays is kept there (row and entry, 16 bits each) instead.
__device__ __forceinline__ void place_rows(const ws_routing& r, WarpRows& w, int cols, const uint32_t* mask,
                                           const uint16_t* pre, const int* first, uint32_t* staged = nullptr) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool held = w.hi - w.lo <= 32 * kHeld;  // by mark_rows
  for (int64_t base = w.lo; base < w.hi; base += 32 * kHeld) {
    if (!held) w.load(r, base);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (w.row[i] < 0) continue;
      const int64_t e = base + 32 * i + lane;
      const int col = w.col[i];
      int slot = -1;
      if (static_cast<unsigned>(col) < static_cast<unsigned>(cols)) {
        const uint32_t at = static_cast<uint32_t>(first[col]) + pre[warp * cols + col] +
                            __popc(mask[warp * cols + col] & ((1u << w.row[i]) - 1u));
        if (at < static_cast<uint32_t>(r.nnz)) slot = static_cast<int>(at);
        if (slot < 0) {  // counted more than once
        } else if (staged) {
          staged[slot] = static_cast<uint32_t>(w.first + w.row[i]) << 16 | static_cast<uint32_t>(e);
        } else {
          r.rows[slot] = static_cast<int32_t>(w.first + w.row[i]);
          r.entries[slot] = static_cast<int32_t>(e);
        }
      }
      r.slots[e] = slot;
    }
  }
}

// Clears `words` words, 16 bytes at a time (the masks start at a multiple of that).
__device__ __forceinline__ void clear_words(uint32_t* p, int words) {
  for (int i = 4 * threadIdx.x; i < words; i += 4 * blockDim.x) {
    if (i + 4 <= words) *reinterpret_cast<uint4*>(p + i) = make_uint4(0, 0, 0, 0);
    else
      for (int j = i; j < words; ++j) p[j] = 0;
  }
}

// total[e] (shared; at most one a row) becomes the first slot of column e; returns the number of placed entries.  V holds rows times
// columns: what is marked may be more than the entries are.
template <typename V>
__device__ __forceinline__ int scan_columns(const ws_routing& r, int cols, int* total, V* scratch) {
  V sum = 0;
  for (int e0 = 0; e0 < cols; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    const V n = e < cols ? total[e] : 0;
    V all = 0;
    const V before = block_exclusive_scan(n, scratch, &all);
    if (e < cols) total[e] = slots_before(r, sum, before);
    sum += all;
  }
  __syncthreads();
  return slots_before(r, sum, 0);
}

// Entries of no row, where arrays are longer than the row pointer says: f(entry) for each.
template <typename F>
__device__ __forceinline__ void for_rowless(const ws_routing& r, F f) {
  int begin, end, unused;
  entry_range(r.rowptr, 0, r.nnz, &begin, &unused);
  entry_range(r.rowptr, r.nrows - 1, r.nnz, &unused, &end);
  for (int64_t e = threadIdx.x; e < begin; e += blockDim.x) f(e);
  for (int64_t e = end + static_cast<int64_t>(threadIdx.x); e < r.nnz; e += blockDim.x) f(e);
}

// Offsets of all columns, and -1 in the slots that entries of no column leave over and for the entries of no row.
__device__ __forceinline__ void write_offsets(const ws_routing& r, int cols, const int* first, int placed) {
  for (int e = threadIdx.x; e < cols; e += blockDim.x) r.offsets[e] = first[e];
  if (threadIdx.x == 0) {
    r.offsets[cols] = placed;
    *r.status = 0;
  }
  for (int64_t i = placed + static_cast<int64_t>(threadIdx.x); i < r.nnz; i += blockDim.x) r.rows[i] = r.entries[i] = -1;
  if (placed < r.nnz) for_rowless(r, [&](int64_t e) { r.slots[e] = -1; });
}

// Entries of column e in the warps' rows; pre[w * cols + e] receives those of the warps before w.
__device__ __forceinline__ int count_column(const uint32_t* mask, uint16_t* pre, int cols, int e, int warps) {
  int n = 0;
#pragma unroll 8
  for (int w = 0; w < warps; ++w) {
    pre[w * cols + e] = static_cast<uint16_t>(n);
    n += __popc(mask[w * cols + e]);
  }
  return n;
}

// Shared memory: mask [W][cols], two int arrays [cols], pre [W][cols].
constexpr size_t build_smem(int cols, int W) { return static_cast<size_t>(cols) * (W * 4 + 8 + W * 2); }

// The most that a plan in a single launch takes.  A kernel's limit of dynamic shared memory is set to a constant: it is the kernel's,
// whichever thread launches it, and a smaller plan of one thread may not lower it under another's.
constexpr size_t kMostSmall = 200 * 1024;
static_assert(build_smem(kRouteMaxCols, kSmallWarps) <= kMostSmall);

// As many warps as the rows need.  stage: rows and entries are put in the order of their slots in shared memory first, because one SM
// stores the 32 places of a warp one after the other.  us without | with: 1001 rows of eight entries over 64 columns 14.0 | 8.6
// (two launches of many CTAs 6.5, a launch more of the host's time), 512 rows 8.2 | 5.6, 1001 rows of three over 17 8.0 | 7.0.
__global__ void __launch_bounds__(32 * kSmallWarps) routing_small_kernel(ws_routing r, int cols, bool stage) {
  const int warps = blockDim.x >> 5;
  extern __shared__ __align__(16) int sm[];
  __shared__ int scratch[32];
  may_start_next();
  uint32_t* mask = reinterpret_cast<uint32_t*>(sm);
  int* first = sm + warps * cols;
  uint16_t* pre = reinterpret_cast<uint16_t*>(first + 2 * cols);
  WarpRows w;
  w.start(r, threadIdx.x & ~31u);
  clear_words(mask, warps * cols);
  __syncthreads();
  mark_rows(r, w, cols, mask);
  __syncthreads();
  for (int e = threadIdx.x; e < cols; e += blockDim.x) first[e] = count_column(mask, pre, cols, e, warps);
  __syncthreads();
  const int placed = scan_columns(r, cols, first, scratch);
  write_offsets(r, cols, first, placed);
  uint32_t* const staged = stage ? reinterpret_cast<uint32_t*>(pre + ((warps * cols + 1) & ~1)) : nullptr;
  place_rows(r, w, cols, mask, pre, first, staged);
  if (!stage) return;
  __syncthreads();
  for (int i = threadIdx.x; i < placed; i += blockDim.x) {
    const uint32_t v = staged[i];
    r.rows[i] = static_cast<int32_t>(v >> 16);
    r.entries[i] = static_cast<int32_t>(v & 0xffffu);
  }
}

template <int W>
__global__ void __launch_bounds__(32 * W) routing_count_kernel(ws_routing r, int cols, int64_t chunk, int32_t* counts) {
  extern __shared__ __align__(16) int sm[];
  uint32_t* mask = reinterpret_cast<uint32_t*>(sm);
  int* cnt = sm + W * cols;
  may_start_next();
  for (int e = threadIdx.x; e < cols; e += blockDim.x) cnt[e] = 0;
  const int64_t begin = chunk * blockIdx.x, end = min(begin + chunk, r.nrows);
  for (int64_t row0 = begin; row0 < end; row0 += 32 * W) {
    WarpRows w;
    w.start(r, row0 + (threadIdx.x & ~31u));
    clear_words(mask, W * cols);
    __syncthreads();
    mark_rows(r, w, cols, mask);
    __syncthreads();
    for (int e = threadIdx.x; e < cols; e += blockDim.x) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < W; ++i) n += __popc(mask[i * cols + e]);
      cnt[e] += n;
    }
    __syncthreads();
  }
  const int padded = (cols + 3) & ~3;
  for (int e = threadIdx.x; e < padded; e += blockDim.x) counts[static_cast<int64_t>(blockIdx.x) * padded + e] = e < cols ? cnt[e] : 0;
}

// Every CTA adds up the counts of all chunks by itself (a few hundred KB from L2, the threads split over the chunks):
// a launch less than a scan of its own.  It marks its first tile while the counting launch still runs.
template <int W>
__global__ void __launch_bounds__(32 * W) routing_place_kernel(ws_routing r, int cols, int64_t chunk,
                                                               const int32_t* counts) {
  extern __shared__ __align__(16) int sm[];
  __shared__ int64_t scratch[32];
  uint32_t* mask = reinterpret_cast<uint32_t*>(sm);
  int* next = sm + W * cols;            // first slot of the tile in every column
  int* before = next + cols;            // entries of the chunks before this one
  uint16_t* pre = reinterpret_cast<uint16_t*>(before + cols);
  const int64_t begin = chunk * blockIdx.x, end = min(begin + chunk, r.nrows);
  WarpRows w;
  w.start(r, begin + (threadIdx.x & ~31u));
  clear_words(mask, W * cols);
  for (int e = threadIdx.x; e < cols; e += blockDim.x) next[e] = before[e] = 0;
  __syncthreads();
  mark_rows(r, w, cols, mask);
  may_start_next();
  wait_for_last();
  const int quads = (cols + 3) / 4, groups = 32 * W / quads;  // at most 256 quads: a thread each, or more
  const int g = static_cast<int>(threadIdx.x) / quads, v = static_cast<int>(threadIdx.x) - g * quads;
  if (g < groups) {
    int4 total = make_int4(0, 0, 0, 0), mine = total;
    const int4* from = reinterpret_cast<const int4*>(counts) + v;
#pragma unroll 8
    for (int c = g; c < static_cast<int>(gridDim.x); c += groups) {
      const int4 n = from[static_cast<int64_t>(c) * quads];
      total.x += n.x, total.y += n.y, total.z += n.z, total.w += n.w;
      if (c < static_cast<int>(blockIdx.x)) mine.x += n.x, mine.y += n.y, mine.z += n.z, mine.w += n.w;
    }
    const int t[4] = {total.x, total.y, total.z, total.w}, m[4] = {mine.x, mine.y, mine.z, mine.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * v + i < cols) {
        atomicAdd(&next[4 * v + i], t[i]);
        atomicAdd(&before[4 * v + i], m[i]);
      }
  }
  __syncthreads();
  const int placed = scan_columns(r, cols, next, scratch);
  if (blockIdx.x == 0) write_offsets(r, cols, next, placed);
  __syncthreads();
  for (int e = threadIdx.x; e < cols; e += blockDim.x) {
    next[e] = slots_before(r, next[e], before[e]);
    before[e] = count_column(mask, pre, cols, e, W);
  }
  __syncthreads();
  place_rows(r, w, cols, mask, pre, next);
  for (int64_t row0 = begin + 32 * W; row0 < end; row0 += 32 * W) {
    __syncthreads();
    for (int e = threadIdx.x; e < cols; e += blockDim.x) next[e] = slots_before(r, next[e], before[e]);
    w.start(r, row0 + (threadIdx.x & ~31u));
    clear_words(mask, W * cols);
    __syncthreads();
    mark_rows(r, w, cols, mask);
    __syncthreads();
    for (int e = threadIdx.x; e < cols; e += blockDim.x) before[e] = count_column(mask, pre, cols, e, W);
    __syncthreads();
    place_rows(r, w, cols, mask, pre, next);
  }
}

// ------------------------------------------------------------------ rows moved

constexpr int kMoveThreads = 256;
constexpr int kMoveWarps = kMoveThreads / 32;

// The slot of entry e, or -1.
__device__ __forceinline__ int slot_of(const ws_routing& r, int e) {
  const int s = r.slots[e];
  return static_cast<unsigned>(s) < static_cast<unsigned>(r.nnz) ? s : -1;
}

// The rows behind the placed entries (there are some only if entries have no column) are zero:
// team `team` of `teams`, whose members go by `lane` of `lanes`, clears every teams-th of them.
template <typename P>
__device__ __forceinline__ void zero_rest(const ws_routing& r, char* rows, int64_t ld, int packs, int64_t team,
                                          int64_t teams, int lane, int lanes) {
  for (int64_t s = r.offsets[r.ncols] + team; s < r.nnz; s += teams)
    for (int i = lane; i < packs; i += lanes) *reinterpret_cast<P*>(rows + s * ld + i * static_cast<int64_t>(sizeof(P))) = P{};
}

// A warp per (row, segment of 32 U packs): the segment is read once and stored to every slot of the row.  Bound by memory: 8191
// rows of 4096 bfloat16, eight entries each, 604 MB: 90 us, 6.7 TB/s.
template <typename P, int U>
__global__ void __launch_bounds__(kMoveThreads)
    dispatch_kernel(ws_routing r, const char* x, int64_t ldx, char* xs, int64_t ldxs,
                    int packs, int segs) {
  may_start_next();
  wait_for_last();
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kMoveWarps + (threadIdx.x >> 5);
  zero_rest<P>(r, xs, ldxs, packs, unit, static_cast<int64_t>(gridDim.x) * kMoveWarps, threadIdx.x & 31, 32);
  const int64_t row = unit / segs;
  if (row >= r.nrows) return;
  const int at = static_cast<int>(unit - row * segs) * 32 * U + (threadIdx.x & 31);
  int begin, end;
  entry_range(r.rowptr, row, r.nnz, &begin, &end);
  P v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at + 32 * u < packs) v[u] = *reinterpret_cast<const P*>(x + row * ldx + (at + 32 * u) * static_cast<int64_t>(sizeof(P)));
  for (int e = begin; e < end; ++e) {
    const int s = slot_of(r, e);
    if (s < 0) continue;
    char* dst = xs + s * ldxs;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + 32 * u < packs) *reinterpret_cast<P*>(dst + (at + 32 * u) * static_cast<int64_t>(sizeof(P))) = v[u];
  }
}

// Threads in groups of 2^log_group, a group per (row, part of it): a thread sums one pack over the row's entries, kBatch loads in
// flight, and goes on to the group's next packs with the slots it has.  One part of a row where rows fill the GPU: the rows'
// loads then run along whole rows.  (A warp per 32 packs of a row: 110 us for 8191 rows of 4096 bfloat16, eight entries each; warps that
// went from row to row and read ahead: 138 us; this: 95 us, 6.4 TB/s of 604 MB.)
constexpr int kSumThreads = 128;

template <typename T, int N, bool weighted>
__global__ void __launch_bounds__(kSumThreads, 8)
    combine_kernel(ws_routing r, const T* ys, int64_t ldys, T* y, int64_t ldy, int packs,
                   int log_group, int parts) {
  may_start_next();
  wait_for_last();
  constexpr int kBatch = 4;
  const int group = 1 << log_group;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kSumThreads + threadIdx.x) >> log_group;
  const int64_t row = unit / parts;
  if (row >= r.nrows) return;
  int begin, end;
  entry_range(r.rowptr, row, r.nnz, &begin, &end);
  const int part = static_cast<int>(unit - row * parts);
  for (int at = part * group + (threadIdx.x & (group - 1)); at < packs; at += parts * group) {
    float acc[N] = {};
    for (int e0 = begin; e0 < end; e0 += kBatch) {
      Pack<T, N> p[kBatch];
      float w[kBatch];
      bool on[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = e0 + j < end ? slot_of(r, e0 + j) : -1;
        on[j] = s >= 0;
        if (on[j]) {
          p[j] = *reinterpret_cast<const Pack<T, N>*>(ys + s * ldys + at * N);
          w[j] = weighted ? r.vals[e0 + j] : 1.0f;
        }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (!on[j]) continue;
        float f[N];
        unpack<T, N>(p[j], f);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = weighted ? fmaf(w[j], f[i], acc[i]) : acc[i] + f[i];
      }
    }
    *reinterpret_cast<Pack<T, N>*>(y + row * ldy + at * N) = pack<T, N>(acc);
  }
}

// A CTA per row: gy's row is read once for each group of four entries, whose
// products with it are summed by the CTA in a fixed order.  A thread takes 16
// bytes of a row at a time, in packs of M values as far as the addresses
// allow, so the order does not depend on strides and alignment.
// Bound by memory: 16,385 rows of 2048 floats, 55,300 entries, 1.04 GB: 150 us, 6.9 TB/s.
constexpr int kDotThreads = 128;
constexpr int kDotGroup = 4;

template <typename T, int M, int N>
__device__ __forceinline__ void load_group(const T* p, int count, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += M) {
    float part[M] = {};
    if (M == N || i < count) unpack<T, M>(*reinterpret_cast<const Pack<T, M>*>(p + i), part);
#pragma unroll
    for (int j = 0; j < M; ++j) f[i + j] = part[j];
  }
}
template <typename T, int M, int N>
__device__ __forceinline__ void store_group(T* p, int count, const float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += M) {
    float part[M];
#pragma unroll
    for (int j = 0; j < M; ++j) part[j] = f[i + j];
    if (M == N || i < count) *reinterpret_cast<Pack<T, M>*>(p + i) = pack<T, M>(part);
  }
}

template <typename T, int M>
__global__ void __launch_bounds__(kDotThreads)
    combine_backward_kernel(ws_routing r, const T* gy, int64_t ldgy, const T* ys,
                            int64_t ldys, T* gys, int64_t ldgys, float* gvals, int width) {
  may_start_next();
  wait_for_last();
  constexpr int N = 16 / sizeof(T);
  __shared__ float part[kDotThreads / 32][kDotGroup];
  const int64_t row = blockIdx.x;
  zero_rest<Pack<T, M>>(r, reinterpret_cast<char*>(gys), ldgys * static_cast<int64_t>(sizeof(T)), width / M, row,
                        gridDim.x, threadIdx.x, kDotThreads);
  if (row == 0 && r.offsets[r.ncols] < r.nnz) for_rowless(r, [&](int64_t e) { gvals[e] = 0.0f; });
  int begin, end;
  entry_range(r.rowptr, row, r.nnz, &begin, &end);
  const T* g = gy + row * ldgy;
  for (int e0 = begin; e0 < end; e0 += kDotGroup) {
    int s[kDotGroup];
    float w[kDotGroup], dot[kDotGroup];
#pragma unroll
    for (int j = 0; j < kDotGroup; ++j) {
      s[j] = e0 + j < end ? slot_of(r, e0 + j) : -1;
      w[j] = e0 + j < end ? r.vals[e0 + j] : 0.0f;
      dot[j] = 0.0f;
    }
    for (int at = threadIdx.x * N; at < width; at += kDotThreads * N) {
      const int count = width - at;
      float a[N], f[kDotGroup][N];
#pragma unroll
      for (int j = 0; j < kDotGroup; ++j)
        if (s[j] >= 0) load_group<T, M, N>(ys + s[j] * ldys + at, count, f[j]);
      load_group<T, M, N>(g + at, count, a);
#pragma unroll
      for (int j = 0; j < kDotGroup; ++j) {
        if (s[j] < 0) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          dot[j] = fmaf(a[i], f[j][i], dot[j]);
          f[j][i] = w[j] * a[i];
        }
        store_group<T, M, N>(gys + s[j] * ldgys + at, count, f[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kDotGroup; ++j) dot[j] = warp_sum(dot[j]);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int j = 0; j < kDotGroup; ++j) part[threadIdx.x >> 5][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < kDotGroup && e0 + static_cast<int>(threadIdx.x) < end) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < kDotThreads / 32; ++i) sum += part[i][threadIdx.x];
      gvals[e0 + threadIdx.x] = sum;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ rows for the copy engine

// Rows of 16-bit values copied to rows that start at multiples of 16 bytes (the copy engine and 16-byte loads need that): a
// thread per 16 bytes of the copy, up to three matrices in a launch, no matrix of an expert without rows.  3,003 rows of 1003 halves
// (rows that start at any multiple of 2 bytes): 5 us, most of it the launch; with one launch a matrix both gradients of nine experts
// took 148 us, with one for all 79 us.
constexpr int kAlignThreads = 256;

__global__ void __launch_bounds__(kAlignThreads) align_rows_kernel(const AlignedCopies c) {
  may_start_next();
  wait_for_last();
  int64_t at = static_cast<int64_t>(blockIdx.x) * kAlignThreads + threadIdx.x;
  int i = 0;
  while (i < c.count && at >= c.m[i].groups * c.m[i].rows * c.m[i].packs) at -= c.m[i].groups * c.m[i].rows * c.m[i].packs, ++i;
  if (i == c.count) return;
  const AlignedCopy& m = c.m[i];
  const int64_t line = at / m.packs, group = line / m.rows, row = line - group * m.rows;
  const int k = 8 * static_cast<int>(at - line * m.packs);
  if (m.offsets && m.offsets[group] == m.offsets[group + 1]) return;
  const uint16_t* src = m.src + group * m.stride + row * m.ld + k;
  uint32_t w[4] = {};
  if (reinterpret_cast<uintptr_t>(src) % 4 == 0 && k + 8 <= m.width) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = reinterpret_cast<const uint32_t*>(src)[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k + j < m.width) w[j >> 1] |= static_cast<uint32_t>(src[j]) << (16 * (j & 1));
  }
  reinterpret_cast<uint4*>(m.dst)[at] = make_uint4(w[0], w[1], w[2], w[3]);
}

// Calls f with the widest pack (16, 8, 4 or 2 bytes) that every address and row length allows.
template <typename F>
void for_pack(uint64_t bits, F f) {
  if (bits % 16 == 0) f(std::integral_constant<int, 16>());
  else if (bits % 8 == 0) f(std::integral_constant<int, 8>());
  else if (bits % 4 == 0) f(std::integral_constant<int, 4>());
  else f(std::integral_constant<int, 2>());
}
template <int B>
struct Bytes;
template <>
struct Bytes<16> { using type = uint4; };
template <>
struct Bytes<8> { using type = uint2; };
template <>
struct Bytes<4> { using type = uint32_t; };
template <>
struct Bytes<2> { using type = uint16_t; };

template <typename F>
void for_type(ws_dtype_t dt, F f) {
  if (dt == WS_F32) f(float());
  else if (dt == WS_BF16) f(__nv_bfloat16());
  else f(__half());
}

int64_t value_size(ws_dtype_t dt) { return dt == WS_F32 ? 4 : 2; }
uint64_t address_bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

unsigned warp_grid(int64_t units) { return static_cast<unsigned>((units + kMoveWarps - 1) / kMoveWarps); }

}  // namespace

// As many chunks as SMs at most, of whole tiles.
int64_t routing_chunks(int64_t nrows, int64_t ncols, int num_sms) {
  if (nrows <= kSmallRows) return 1;
  const int64_t tiles = up(nrows, 32 * build_warps(nrows, ncols));
  return up(tiles, up(tiles, num_sms));
}

void launch_routing_build(const ws_routing& r, int32_t* counts, int num_sms, cudaStream_t s) {
  const int cols = static_cast<int>(r.ncols);
  const int64_t chunks = routing_chunks(r.nrows, cols, num_sms);
  const auto allow = [&](const void* kernel, size_t smem, size_t most) {
    if (smem > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
  };
  if (chunks == 1) {
    const int warps = r.nrows <= 128 ? 4 : static_cast<int>((r.nrows + 31) / 32);  // four at least, for the columns
    const size_t own = build_smem(cols, warps), all = ((own + 3) & ~size_t{3}) + static_cast<size_t>(r.nnz) * 4;
    const bool stage = r.nnz <= 65536 && all <= kMostSmall;
    const size_t smem = stage ? all : own;
    allow(reinterpret_cast<const void*>(routing_small_kernel), smem, kMostSmall);
    routing_small_kernel<<<1, 32 * warps, smem, s>>>(r, cols, stage);
    return;
  }
  const auto both = [&](auto warps) {
    constexpr int W = decltype(warps)::value;
    const size_t smem = build_smem(cols, W);
    const int64_t chunk = up(up(r.nrows, 32 * W), chunks) * 32 * W;
    allow(reinterpret_cast<const void*>(routing_count_kernel<W>), smem, build_smem(kRouteMaxCols, W));
    allow(reinterpret_cast<const void*>(routing_place_kernel<W>), smem, build_smem(kRouteMaxCols, W));
    routing_count_kernel<W><<<static_cast<unsigned>(chunks), 32 * W, smem, s>>>(r, cols, chunk, counts);
    launch_early(routing_place_kernel<W>, dim3(static_cast<unsigned>(chunks)), 32 * W, smem, s, 1, r, cols, chunk, counts);
  };
  if (build_warps(r.nrows, cols) == 8) both(std::integral_constant<int, 8>());
  else both(std::integral_constant<int, 16>());
}

void launch_align(const AlignedCopies& c, cudaStream_t s) {
  int64_t packs = 0;
  for (int i = 0; i < c.count; ++i) packs += c.m[i].groups * c.m[i].rows * c.m[i].packs;
  if (packs > 0) launch_early(align_rows_kernel, dim3(static_cast<unsigned>((packs + kAlignThreads - 1) / kAlignThreads)), kAlignThreads, 0, s, 1, c);
}

void launch_dispatch(const ws_routing& r, const void* x, int64_t ldx, void* xs, int64_t ldxs, int64_t width,
                     ws_dtype_t dt, cudaStream_t s) {
  const int64_t z = value_size(dt);
  for_pack(address_bits(x) | address_bits(xs) | (ldx * z) | (ldxs * z) | (width * z), [&](auto b) {
    constexpr int B = decltype(b)::value;
    using P = typename Bytes<B>::type;
    const int packs = static_cast<int>(width * z / B);
    const char* src = static_cast<const char*>(x);
    char* dst = static_cast<char*>(xs);
    // Four packs a lane where the warps still fill the GPU, else one: a short call lasts as long as its longest warp.
    if (r.nrows * static_cast<int64_t>(packs) >= 32 * 4 * 8192) {
      const int segs = (packs + 127) / 128;
      launch_early(dispatch_kernel<P, 4>, dim3(warp_grid(r.nrows * segs)), kMoveThreads, 0, s, 1, r, src, ldx * z, dst, ldxs * z, packs, segs);
    } else {
      const int segs = (packs + 31) / 32;
      launch_early(dispatch_kernel<P, 1>, dim3(warp_grid(r.nrows * segs)), kMoveThreads, 0, s, 1, r, src, ldx * z, dst, ldxs * z, packs, segs);
    }
  });
}

void launch_combine(const ws_routing& r, bool weighted, const void* ys, int64_t ldys, void* y, int64_t ldy,
                    int64_t width, ws_dtype_t dt, int num_sms, cudaStream_t s) {
  const int64_t z = value_size(dt);
  for_type(dt, [&](auto t) {
    using T = decltype(t);
    for_pack(address_bits(ys) | address_bits(y) | (ldys * z) | (ldy * z) | (width * z), [&](auto b) {
      constexpr int B = decltype(b)::value;
      if constexpr (B >= static_cast<int>(sizeof(T))) {
        constexpr int N = B / sizeof(T);
        const int packs = static_cast<int>(width / N);
        int log_group = 0;
        while ((1 << log_group) < packs && (1 << log_group) < kSumThreads) ++log_group;
        const int group = 1 << log_group;
        const int parts = r.nrows * group >= int64_t{8} * kSumThreads * num_sms ? 1 : (packs + group - 1) / group;
        const auto kernel = weighted ? combine_kernel<T, N, true> : combine_kernel<T, N, false>;
        launch_early(kernel, dim3(static_cast<unsigned>((r.nrows * parts * group + kSumThreads - 1) / kSumThreads)), kSumThreads, 0, s, 1,
                     r, static_cast<const T*>(ys), ldys, static_cast<T*>(y), ldy, packs, log_group, parts);
      }
    });
  });
}

void launch_combine_backward(const ws_routing& r, const void* gy, int64_t ldgy, const void* ys, int64_t ldys,
                             void* gys, int64_t ldgys, float* gvals, int64_t width, ws_dtype_t dt, cudaStream_t s) {
  const int64_t z = value_size(dt);
  for_type(dt, [&](auto t) {
    using T = decltype(t);
    for_pack(address_bits(gy) | address_bits(ys) | address_bits(gys) | (ldgy * z) | (ldys * z) | (ldgys * z) | (width * z),
             [&](auto b) {
               constexpr int B = decltype(b)::value;
               if constexpr (B >= static_cast<int>(sizeof(T))) {
                 constexpr int N = B / sizeof(T);
                 launch_early(combine_backward_kernel<T, N>, dim3(static_cast<unsigned>(r.nrows)), kDotThreads, 0, s, 1, r, static_cast<const T*>(gy), ldgy, static_cast<const T*>(ys), ldys, static_cast<T*>(gys), ldgys,
                     gvals, static_cast<int>(width));
               }
             });
  });
}

}  // namespace wsk
