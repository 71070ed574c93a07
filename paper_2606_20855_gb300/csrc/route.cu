// Rows of a routing matrix chosen from logits, and the gradient of that choice.
//
// Row i of R holds the k largest of row i's E logits l (ties to the lowest
// column) with the weights
//   normalize       v_j = exp(l_j - m) / sum over the chosen of exp(l - m)
//   else            v_j = exp(l_j - m) / sum over all columns of exp(l - m),   m = the row's largest logit.
// A logit of -inf has weight 0 and is chosen last; a row of nothing else has
// weights 0, not 0 / 0.  NaN counts as the largest value and makes the row's
// weights NaN.  With g the gradient of v and a = sum over the chosen of v g,
//   normalize       dl_j = v_j (g_j - a) at the chosen columns, 0 elsewhere
//   else            dl_j = p_j (g_j [j chosen] - a) at every column, p the softmax over all.
// Exponentials and sums are held in 32 bits whatever the logits' type; the
// gradient of a 16-bit logit is rounded once, when it is stored.
#include <cmath>

#include "routing.cuh"

namespace wsk {
namespace {

constexpr int kRouteWarps = 8;

// Order of floats as unsigned numbers: NaN last of all, -0 as +0; 0 is below -inf and marks "no logit".
// Adding zero makes -0 positive and any NaN the canonical one, 0x7fffffff.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(__fadd_rn(f, 0.0f));
  return u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);
}

// V consecutive logits of a row from column `at` on; -inf and key 0 past the row's end.
template <typename T, int V>
__device__ __forceinline__ void load_row(const T* row, int at, int cols, bool vec, float (&f)[V]) {
  constexpr int N = V * sizeof(T) >= 16 ? 16 / sizeof(T) : V;
  if (vec && at + V <= cols) {
#pragma unroll
    for (int i = 0; i < V; i += N) {
      float part[N];
      unpack<T, N>(*reinterpret_cast<const Pack<T, N>*>(row + at + i), part);
#pragma unroll
      for (int j = 0; j < N; ++j) f[i + j] = part[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = at + i < cols ? to_f32<T>(row[at + i]) : -INFINITY;
  }
}

__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float(key ^ (static_cast<uint32_t>(static_cast<int>(~key) >> 31) | 0x80000000u));
}

// A warp per row; a lane holds V consecutive logits, so that among equal
// logits the lowest lane holds the lowest column and a ballot settles ties.
//
// The k-th largest of the lanes' own maxima is at most the row's k-th largest
// logit, so every chosen logit is at or above it, and few others are: those
// candidates go to one a lane, by column, and k rounds of a warp maximum choose
// among them.  Rows with more than 32 candidates (many equal logits, or k near
// the number of lanes) choose among all logits, a round at a time: the lane
// that held the maximum looks for its next.  65,537 rows of 256 (k = 8,
// float, 67 MB read, 10 us at the copy rate): 29 us, bound by issue (400
// instructions a row, 82% of the issue slots); 51 us with that way alone (900
// instructions).  Candidates that each count those above them, in place of the
// second k rounds: 30 us.
template <typename T, int V>
__global__ void __launch_bounds__(32 * kRouteWarps)
    topk_route_kernel(const T* logits, int64_t rows, int cols, int64_t ld, bool vec, int k, bool normalize, int64_t* rowptr,
                      int32_t* colidx, float* vals) {
  may_start_next();
  wait_for_last();
  __shared__ uint2 cand[kRouteWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp;
  if (row >= rows) return;
  float f[V];
  load_row<T, V>(logits + row * ld, lane * V, cols, vec, f);
  uint32_t key[V];
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] = lane * V + i < cols ? order_key(f[i]) : 0u;
  uint32_t my_key = key[0];  // the lane's candidate
  int my_col = lane;
  bool one_each = V == 1;
  int all = 32;  // candidates
  if constexpr (V > 1) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) best = max(best, key[i]);
    uint32_t bound = 0;
#pragma unroll 4
    for (int r = 0; r < k; ++r) {  // equal maxima leave together: the bound is lower then, not wrong
      bound = __reduce_max_sync(0xffffffffu, best);
      if (best == bound) best = 0;
    }
    bound = max(bound, 1u);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) mine += key[i] >= bound;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    all = __shfl_sync(0xffffffffu, upto, 31);
    one_each = all <= 32;
    if (one_each) {
      int at = upto - mine;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (key[i] >= bound) cand[warp][at++] = make_uint2(key[i], lane * V + i);
      __syncwarp();
      const uint2 c = lane < all ? cand[warp][lane] : make_uint2(0, 0);
      my_key = c.x;
      my_col = c.y;
    }
  }
  bool chosen = false;
  int rank;
  if (one_each) {
    if (all == k) {
      chosen = lane < k;
    } else {
      uint32_t left = my_key;
#pragma unroll 4
      for (int r = 0; r < k; ++r) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, left);
        if (lane == __ffs(__ballot_sync(0xffffffffu, left == top)) - 1) left = 0, chosen = true;
      }
    }
    rank = __popc(__ballot_sync(0xffffffffu, chosen) & ((1u << lane) - 1u));
  } else {
    uint32_t best = 0;
    int where = 0;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] >= best) best = key[i], where = i;
    my_col = 0x7fffffff;
    for (int r = 0; r < k; ++r) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, best);
      const int owner = __ffs(__ballot_sync(0xffffffffu, best == top)) - 1;
      const int col = __shfl_sync(0xffffffffu, lane * V + where, owner);
      if (lane == r) my_key = top, my_col = col;
      if (lane == owner) {  // the logit leaves; the lane's next best
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i == where) key[i] = 0;
        best = 0;
#pragma unroll
        for (int i = V - 1; i >= 0; --i)
          if (key[i] >= best) best = key[i], where = i;
      }
    }
    chosen = lane < k;
    rank = 0;  // places by column
    for (int r = 0; r < k; ++r) rank += __shfl_sync(0xffffffffu, my_col, r) < my_col;
  }
  float m = key_value(__reduce_max_sync(0xffffffffu, chosen ? my_key : 0u));
  if (m == -INFINITY) m = 0.0f;
  const float e = chosen ? expf(key_value(my_key) - m) : 0.0f;
  float total = e;
  if (!normalize) {
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) total += expf(f[i] - m);  // 0 past the row's end
  }
  total = warp_sum(total);
  const int64_t at = row * k;
  if (chosen) {
    colidx[at + rank] = my_col;
    vals[at + rank] = total == 0.0f ? 0.0f : e / total;
  }
  if (lane == 0) {
    rowptr[row] = at;
    if (row == rows - 1) rowptr[rows] = at + k;
  }
}

// A warp per row: the softmax again (not kept from the choice: a row of logits is read faster than weights of all columns are
// stored), the chosen columns put over it in shared memory, every value of the row stored once, in packs.  Bound by the store:
// 65,537 rows of 256 (k = 8, float, 67 MB written, 10 us at the copy rate): 13.5 us; 17 us with a lane's values stored side by side
// (half sectors), and as long with four rows a warp.
template <typename T, int V>
__global__ void __launch_bounds__(32 * kRouteWarps)
    topk_route_backward_kernel(const T* logits, int64_t rows, int cols, int64_t ld, bool vec, int k, bool normalize,
                               const int32_t* colidx, const float* vals, const float* gvals, T* glogits, int64_t ldg, bool vecg) {
  may_start_next();
  wait_for_last();
  constexpr int N = V * sizeof(T) >= 16 ? 16 / sizeof(T) : V;
  __shared__ __align__(16) float lines[kRouteWarps][32 * V];
  const int lane = threadIdx.x & 31;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRouteWarps + (threadIdx.x >> 5);
  if (row >= rows) return;
  float v = 0.0f, g = 0.0f;
  int col = -1;
  if (lane < k) {
    col = colidx[row * k + lane];
    v = vals[row * k + lane];
    g = gvals[row * k + lane];
  }
  float out[V], a = 0.0f;
  if (normalize) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = 0.0f;
  } else {
    a = warp_sum(v * g);
    load_row<T, V>(logits + row * ld, lane * V, cols, vec, out);
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) best = max(best, order_key(out[i]));
    const uint32_t top = __reduce_max_sync(0xffffffffu, best);
    float m = key_value(top);
    if (m == -INFINITY) m = 0.0f;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) total += out[i] = expf(out[i] - m);
    total = warp_sum(total);
    const float scale = total == 0.0f ? 0.0f : -a / total;
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] *= scale;
  }
  // the chosen columns over the others, in shared memory: every value of the row is stored once
  float* line = lines[threadIdx.x >> 5];
#pragma unroll
  for (int i = 0; i < V; ++i) line[lane * V + i] = out[i];
  if (normalize) a = warp_sum(v * g);
  __syncwarp();
  if (static_cast<unsigned>(col) < static_cast<unsigned>(cols)) line[col] = v * (g - a);
  __syncwarp();
  T* dst = glogits + row * ldg;
  if (vecg) {  // neighbouring lanes store neighbouring packs
#pragma unroll
    for (int c = 0; c < V / N; ++c) {
      const int at = (32 * c + lane) * N;
      float part[N];
#pragma unroll
      for (int j = 0; j < N; ++j) part[j] = line[at + j];
      if (at + N <= cols) *reinterpret_cast<Pack<T, N>*>(dst + at) = pack<T, N>(part);
      else
        for (int j = at; j < cols; ++j) dst[j] = from_f32<T>(line[j]);
    }
  } else {
    for (int i = lane; i < cols; i += 32) dst[i] = from_f32<T>(line[i]);
  }
}

template <typename F>
void for_values(int cols, F f) {
  if (cols <= 32) f(std::integral_constant<int, 1>());
  else if (cols <= 64) f(std::integral_constant<int, 2>());
  else if (cols <= 128) f(std::integral_constant<int, 4>());
  else if (cols <= 256) f(std::integral_constant<int, 8>());
  else if (cols <= 512) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
}

template <typename F>
void for_type(ws_dtype_t dt, F f) {
  if (dt == WS_F32) f(float());
  else if (dt == WS_BF16) f(__nv_bfloat16());
  else f(__half());
}

// Whether V values from every V-th column of every row may be moved as packs.
bool packs(const void* p, int64_t ld, int V, int size) {
  const int64_t bytes = V * size < 16 ? V * size : 16;
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % bytes == 0;
}

}  // namespace

void launch_topk_route(const void* logits, int64_t rows, int cols, int64_t ld, ws_dtype_t dt, int k, bool normalize,
                       int64_t* rowptr, int32_t* colidx, float* vals, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>((rows + kRouteWarps - 1) / kRouteWarps);
  for_type(dt, [&](auto t) {
    using T = decltype(t);
    for_values(cols, [&](auto v) {
      constexpr int V = decltype(v)::value;
      launch_early(topk_route_kernel<T, V>, dim3(grid), 32 * kRouteWarps, 0, s, 1, static_cast<const T*>(logits), rows, cols, ld,
                   packs(logits, ld, V, sizeof(T)), k, normalize, rowptr, colidx, vals);
    });
  });
}

void launch_topk_route_backward(const void* logits, int64_t rows, int cols, int64_t ld, ws_dtype_t dt, int k,
                                bool normalize, const int32_t* colidx, const float* vals, const float* gvals,
                                void* glogits, int64_t ldg, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>((rows + kRouteWarps - 1) / kRouteWarps);
  for_type(dt, [&](auto t) {
    using T = decltype(t);
    for_values(cols, [&](auto v) {
      constexpr int V = decltype(v)::value;
      launch_early(topk_route_backward_kernel<T, V>, dim3(grid), 32 * kRouteWarps, 0, s, 1, static_cast<const T*>(logits), rows, cols, ld,
                   packs(logits, ld, V, sizeof(T)), k, normalize, colidx, vals, gvals, static_cast<T*>(glogits), ldg,
                   packs(glogits, ldg, V, sizeof(T)));
    });
  });
}

}  // namespace wsk
