// Low-rank adapters of many requests at once, beside a projection they share:
//   y[t] = base[t] + sum over row t of S of  v * B[a] (A[a] x[t])
// S: tokens x adapters in CSR (a column and value per adapter of a token, none
// for most), A: adapters x rank x K, B: adapters x N x rank, 16-bit; base is the
// shared projection's result.
//
// Two kernels: inner products h = v A[a] x[t] for every entry of S, then
// y = base + B[a] h.  Both are bound by memory (x, base and y, and the met
// adapters, once each; 2 rank multiply-adds per value), so h stays small: sums
// are 32-bit, and h is kept as a pair of 16-bit values, its rounding and the
// rounding of what that left over, 16 (bfloat16) or 22 (half) significant bits.
// One 16-bit value would add an error as large as the result's own rounding.
// A half pair holds |h| up to 65504.
//
// Few tokens ("step"): every token is on its own; a warp per entry and pair of
// ranks, then a thread per value of y: everything in flight at once, no
// reuse.  Many tokens ("prompt"): tiles of 32 tokens on the warp-level matrix
// instruction.  The tokens of a tile mostly share an adapter, and the tile goes
// through the adapters it meets in ascending order: every lane stands at its
// token's first entry, the smallest column among the lanes is next, and the
// lanes that have it move on (columns ascend within a row).  The matrix
// instruction's operands go from global memory to registers in 16-byte loads:
// the order of the contraction index is free as long as both operands agree, so
// a lane's eight neighbouring values serve as the pairs of two instructions.
#include <climits>
#include <type_traits>

#include "routing.cuh"

namespace wsk {
namespace {

constexpr int kAdThreads = 256;
constexpr int kAdWarps = kAdThreads / 32;
constexpr int kTileTok = 32;

// h as {roundings, remainders} of two neighbouring ranks.
template <bool half>
__device__ __forceinline__ uint2 split_pair(float a, float b) {
  const uint16_t ha = bits16<half>(a), hb = bits16<half>(b);
  // an infinite or NaN rounding has no remainder
  const float ra = a - value16<half>(ha), rb = b - value16<half>(hb);
  const uint16_t la = bits16<half>(ra == ra && fabsf(ra) <= 3.4e38f ? ra : 0.0f);
  const uint16_t lb = bits16<half>(rb == rb && fabsf(rb) <= 3.4e38f ? rb : 0.0f);
  return make_uint2(ha | static_cast<uint32_t>(hb) << 16, la | static_cast<uint32_t>(lb) << 16);
}

// d += (roundings + remainders of h, rows a and b) times v.
template <bool half>
__device__ __forceinline__ void mma_pair(float (&d)[4], const uint4& a, const uint4& b, const uint2& v) {
  mma16<half>(d, a.x, b.x, a.z, b.z, v.x, v.y);
  mma16<half>(d, a.y, b.y, a.w, b.w, v.x, v.y);
}

// Ranks k .. k + 3 of a row of B, zero past its end.
__device__ __forceinline__ uint2 load4(const uint16_t* row, int k, int r, bool vec) {
  if (vec) return k < r ? *reinterpret_cast<const uint2*>(row + k) : make_uint2(0, 0);
  uint32_t w[2] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (k + i < r) w[i >> 1] |= static_cast<uint32_t>(row[k + i]) << (16 * (i & 1));
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ bool met(const ws_adapters_call& c, int col) {
  return static_cast<int64_t>(col) >= 0 && col < c.ncols;
}

// A lane's place in its token's row of S.
struct Walk {
  int at, end, col;
  __device__ __forceinline__ void settle(const ws_adapters_call& c) {
    col = INT_MAX;
    while (at < end) {
      const int x = c.colidx[at];
      if (met(c, x)) {
        col = x;
        return;
      }
      ++at;
    }
  }
  __device__ __forceinline__ void start(const ws_adapters_call& c, int64_t row) {
    at = end = 0;
    if (row < c.nrows) entry_range(c.rowptr, row, c.nnz, &at, &end);
    settle(c);
  }
  __device__ __forceinline__ void next(const ws_adapters_call& c) {
    ++at;
    settle(c);
  }
};

// ---------------------------------------------------------------- many tokens

// h of a tile of 32 tokens, 8 NR ranks from 8 NR blockIdx.y on; the warps take every eighth step of 32 values.
// Rows that are not there (tokens past the last, ranks past r) repeat one that is; what comes of them is not used.
template <bool half, int NR>
__global__ void __launch_bounds__(kAdThreads, NR <= 4 ? 2 : 1) shrink_tile_kernel(const ws_adapters_call c, uint2* __restrict__ h, int rpad) {
  extern __shared__ float red[];  // [warps][32][8 NR]
  __shared__ int entry[kTileTok];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTileTok;
  const int r0 = blockIdx.y * 8 * NR;
  const int K = static_cast<int>(c.K), r = static_cast<int>(c.r);
  Walk w;
  w.start(c, t0 + lane);
  const uint16_t* xrow[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    xrow[i] = static_cast<const uint16_t*>(c.x) + min(t0 + 8 * i + g, c.nrows - 1) * c.ldx;
  for (;;) {
    const int a = __reduce_min_sync(0xffffffffu, w.col);
    if (a == INT_MAX) break;
    const bool mine = w.col == a;
    if (warp == 0) entry[lane] = mine ? w.at : -1;
    const uint16_t* A = static_cast<const uint16_t*>(c.A) + a * c.strideA;
    const uint16_t* arow[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) arow[j] = A + min(r0 + 8 * j + g, r - 1) * c.lda;
    float acc[2][NR][4] = {};
    const auto step = [&](const uint4(&xv)[4], const uint4(&av)[NR]) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < NR; ++j) {
          mma16<half>(acc[m][j], xv[2 * m].x, xv[2 * m + 1].x, xv[2 * m].y, xv[2 * m + 1].y, av[j].x, av[j].y);
          mma16<half>(acc[m][j], xv[2 * m].z, xv[2 * m + 1].z, xv[2 * m].w, xv[2 * m + 1].w, av[j].z, av[j].w);
        }
    };
    int k = 32 * warp + 8 * q;
    constexpr int U = NR <= 4 ? 2 : 1;  // steps whose loads are in flight together
    for (; k - 8 * q + 32 * kAdWarps * (U - 1) + 32 <= K; k += 32 * kAdWarps * U) {
      uint4 xv[U][4], av[U][NR];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) xv[u][i] = *reinterpret_cast<const uint4*>(xrow[i] + k + 32 * kAdWarps * u);
#pragma unroll
        for (int j = 0; j < NR; ++j) av[u][j] = *reinterpret_cast<const uint4*>(arow[j] + k + 32 * kAdWarps * u);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) step(xv[u], av[u]);
    }
#pragma unroll 1
    for (; k - 8 * q < K; k += 32 * kAdWarps) {
      uint4 xv[4], av[NR];
#pragma unroll
      for (int i = 0; i < 4; ++i) xv[i] = load8(xrow[i], k, K);
#pragma unroll
      for (int j = 0; j < NR; ++j) av[j] = load8(arow[j], k, K);
      step(xv, av);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          *reinterpret_cast<float2*>(red + ((warp * kTileTok) + 16 * m + 8 * i + g) * (8 * NR) + 8 * j + 2 * q) =
              make_float2(acc[m][j][2 * i], acc[m][j][2 * i + 1]);
    __syncthreads();
    for (int i = threadIdx.x; i < kTileTok * 4 * NR; i += kAdThreads) {
      const int tok = i / (4 * NR), pair = i - tok * (4 * NR);
      if (entry[tok] < 0 || r0 + 2 * pair >= rpad) continue;
      float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
      for (int k = 0; k < kAdWarps; ++k) {
        const float2 f = *reinterpret_cast<const float2*>(red + (k * kTileTok + tok) * (8 * NR) + 2 * pair);
        s0 += f.x;
        s1 += f.y;
      }
      const float v = c.vals[entry[tok]];
      h[static_cast<int64_t>(entry[tok]) * (rpad / 2) + r0 / 2 + pair] =
          split_pair<half>(r0 + 2 * pair < r ? v * s0 : 0.0f, r0 + 2 * pair + 1 < r ? v * s1 : 0.0f);
    }
    __syncthreads();
    if (mine) w.next(c);
  }
}

// y of 32 tokens: a warp takes 64 values of each; in tile j of eight, column g of the instruction is value
// 32 (j / 4) + 8 (g / 2) + 2 (j % 4) + g % 2, so that a lane ends up with two times eight neighbouring values of a row.
template <bool half, bool vec>
__global__ void __launch_bounds__(kAdThreads, 2)
    expand_tile_kernel(const ws_adapters_call c, const uint2* __restrict__ h, int rpad, bool vecB) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTileTok;
  const int N = static_cast<int>(c.N), r = static_cast<int>(c.r);
  const int n0 = (blockIdx.y * kAdWarps + warp) * 64;
  if (n0 >= N) return;
  const uint16_t* base = static_cast<const uint16_t*>(c.base);
  uint4 bv16[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // rows g, g + 8, g + 16, g + 24
    const int64_t t = t0 + 8 * i + g;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int n = n0 + 32 * s + 8 * q;
      if (vec) {  // rows start at multiples of 16 bytes and N is a multiple of 8
        bv16[i][s] = base && t < c.nrows && n < N ? *reinterpret_cast<const uint4*>(base + t * c.ldbase + n) : make_uint4(0, 0, 0, 0);
      } else {
        uint32_t v[4] = {};
        if (base && t < c.nrows)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (n + e < N) v[e >> 1] |= static_cast<uint32_t>(base[t * c.ldbase + n + e]) << (16 * (e & 1));
        bv16[i][s] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  }
  float acc[2][8][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t v[4] = {bv16[i][s].x, bv16[i][s].y, bv16[i][s].z, bv16[i][s].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i >> 1][4 * s + j][2 * (i & 1)] = value16<half>(static_cast<uint16_t>(v[j]));
        acc[i >> 1][4 * s + j][2 * (i & 1) + 1] = value16<half>(static_cast<uint16_t>(v[j] >> 16));
      }
    }
  Walk w;
  w.start(c, t0 + lane);
  for (;;) {
    const int a = __reduce_min_sync(0xffffffffu, w.col);
    if (a == INT_MAX) break;
    const bool mine = w.col == a;
    int entry[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) entry[i] = __shfl_sync(0xffffffffu, mine ? w.at : -1, 8 * i + g);
    const uint16_t* B = static_cast<const uint16_t*>(c.B) + a * c.strideB;
    // {roundings, remainders} of ranks k + 4 q, + 1 and of + 2, + 3 of the lane's rows
    const auto load_h = [&](int k, uint4(&hv)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        hv[i] = entry[i] >= 0 ? *reinterpret_cast<const uint4*>(h + static_cast<int64_t>(entry[i]) * (rpad / 2) + k / 2 + 2 * q)
                              : make_uint4(0, 0, 0, 0);
    };
    const auto load_b = [&](int k, int j) {  // a row past the last repeats it: its sums are not stored
      const int n = min(n0 + 32 * (j >> 2) + 8 * (g >> 1) + 2 * (j & 3) + (g & 1), N - 1);
      return load4(B + n * c.ldb, k + 4 * q, r, vecB);
    };
    if (__all_sync(0xffffffffu, mine || t0 + lane >= c.nrows)) {
#pragma unroll 1
      for (int k = 0; k < rpad; k += 16) {
        uint4 hv[4];
        uint2 bv[8];
        load_h(k, hv);
#pragma unroll
        for (int j = 0; j < 8; ++j) bv[j] = load_b(k, j);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int m = 0; m < 2; ++m) mma_pair<half>(acc[m][j], hv[2 * m], hv[2 * m + 1], bv[j]);
      }
    } else {
      // Some tokens do not have this adapter.  A zero h would leave them alone but for infinities and NaN in B, so
      // the sum is taken apart and added to the tokens that have it.
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float d[2][4] = {};
#pragma unroll 1
        for (int k = 0; k < rpad; k += 16) {
          uint4 hv[4];
          load_h(k, hv);
          const uint2 bv = load_b(k, j);
#pragma unroll
          for (int m = 0; m < 2; ++m) mma_pair<half>(d[m], hv[2 * m], hv[2 * m + 1], bv);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (entry[i] >= 0) {
            acc[i >> 1][j][2 * (i & 1)] += d[i >> 1][2 * (i & 1)];
            acc[i >> 1][j][2 * (i & 1) + 1] += d[i >> 1][2 * (i & 1) + 1];
          }
      }
    }
    if (mine) w.next(c);
  }
  uint16_t* y = static_cast<uint16_t*>(c.y);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + 8 * i + g;
    if (t >= c.nrows) continue;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int n = n0 + 32 * s + 8 * q;
      uint32_t v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = bits16<half>(acc[i >> 1][4 * s + j][2 * (i & 1)]) |
               static_cast<uint32_t>(bits16<half>(acc[i >> 1][4 * s + j][2 * (i & 1) + 1])) << 16;
      uint16_t* dst = y + t * c.ldy + n;
      if (vec) {
        if (n < N) *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < N) dst[e] = static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// ---------------------------------------------------------------- few tokens

// A CTA per token and two pairs of ranks: four warps a pair, each with a quarter of K.  (One warp a pair: 12.4 us for 48 tokens
// of 4096 values and rank 16, the time of a lane's 16 steps of loads.)
constexpr int kStepSplit = 4;

template <bool half>
__global__ void __launch_bounds__(kAdThreads) shrink_step_kernel(const ws_adapters_call c, uint2* __restrict__ h, int rpad) {
  __shared__ float2 part[kAdWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int K = static_cast<int>(c.K), r = static_cast<int>(c.r), pairs = rpad / 2;
  int begin, end;
  entry_range(c.rowptr, blockIdx.x, c.nnz, &begin, &end);
  const uint16_t* x = static_cast<const uint16_t*>(c.x) + blockIdx.x * c.ldx;
  const int p = blockIdx.y * (kAdWarps / kStepSplit) + warp / kStepSplit;  // pairs is a multiple of 8
  for (int e = begin; e < end; ++e) {
    const int a = c.colidx[e];
    if (!met(c, a)) continue;
    float s0 = 0.0f, s1 = 0.0f;
    if (2 * p < r) {
      const uint16_t* A0 = static_cast<const uint16_t*>(c.A) + a * c.strideA + 2 * p * c.lda;
      const uint16_t* A1 = 2 * p + 1 < r ? A0 + c.lda : A0;
      const auto add = [&](const uint4& xv, const uint4& av, const uint4& bv) {
        const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, aw[4] = {av.x, av.y, av.z, av.w}, bw[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = value16<half>(static_cast<uint16_t>(xw[i])), x1 = value16<half>(static_cast<uint16_t>(xw[i] >> 16));
          s0 = fmaf(x0, value16<half>(static_cast<uint16_t>(aw[i])), s0);
          s0 = fmaf(x1, value16<half>(static_cast<uint16_t>(aw[i] >> 16)), s0);
          s1 = fmaf(x0, value16<half>(static_cast<uint16_t>(bw[i])), s1);
          s1 = fmaf(x1, value16<half>(static_cast<uint16_t>(bw[i] >> 16)), s1);
        }
      };
      constexpr int kStep = 256 * kStepSplit, U = 4;  // U steps whose loads are in flight together
      const int k0 = 256 * (warp % kStepSplit);
      int k = k0 + 8 * lane;
      for (; k - 8 * lane + kStep * (U - 1) + 256 <= K; k += kStep * U) {
        uint4 xv[U], av[U], bv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          xv[u] = *reinterpret_cast<const uint4*>(x + k + kStep * u);
          av[u] = *reinterpret_cast<const uint4*>(A0 + k + kStep * u);
          bv[u] = *reinterpret_cast<const uint4*>(A1 + k + kStep * u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) add(xv[u], av[u], bv[u]);
      }
      for (; k < K; k += kStep) add(load8(x, k, K), load8(A0, k, K), load8(A1, k, K));
      if (2 * p + 1 >= r) s1 = 0.0f;
    }
    s0 = warp_sum(s0);
    s1 = warp_sum(s1);
    if (lane == 0) part[warp] = make_float2(s0, s1);
    __syncthreads();
    if (lane == 0 && warp % kStepSplit == 0) {
#pragma unroll
      for (int i = 1; i < kStepSplit; ++i) s0 += part[warp + i].x, s1 += part[warp + i].y;
      const float v = c.vals[e];
      h[static_cast<int64_t>(e) * pairs + p] = 2 * p < r ? split_pair<half>(v * s0, v * s1) : make_uint2(0, 0);
    }
    __syncthreads();
  }
}

// A thread per value of y.
template <bool half>
__global__ void __launch_bounds__(kAdThreads) expand_step_kernel(const ws_adapters_call c, const uint2* __restrict__ h, int rpad, bool vecB) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * kAdThreads + threadIdx.x, t = blockIdx.y;
  if (n >= c.N) return;
  const int r = static_cast<int>(c.r);
  int begin, end;
  entry_range(c.rowptr, t, c.nnz, &begin, &end);
  float acc = c.base ? value16<half>(static_cast<const uint16_t*>(c.base)[t * c.ldbase + n]) : 0.0f;
  for (int e = begin; e < end; ++e) {
    const int a = c.colidx[e];
    if (!met(c, a)) continue;
    const uint16_t* row = static_cast<const uint16_t*>(c.B) + a * c.strideB + n * c.ldb;
    const uint4* hv = reinterpret_cast<const uint4*>(h + static_cast<int64_t>(e) * (rpad / 2));
#pragma unroll 4
    for (int k = 0; k < r; k += 4) {
      const uint2 b = load4(row, k, r, vecB);
      const uint4 p = hv[k / 4];
      const uint32_t hi[2] = {p.x, p.z}, lo[2] = {p.y, p.w}, bw[2] = {b.x, b.y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc = fmaf(value16<half>(static_cast<uint16_t>(hi[i])) + value16<half>(static_cast<uint16_t>(lo[i])),
                   value16<half>(static_cast<uint16_t>(bw[i])), acc);
        acc = fmaf(value16<half>(static_cast<uint16_t>(hi[i] >> 16)) + value16<half>(static_cast<uint16_t>(lo[i] >> 16)),
                   value16<half>(static_cast<uint16_t>(bw[i] >> 16)), acc);
      }
    }
  }
  static_cast<uint16_t*>(c.y)[t * c.ldy + n] = bits16<half>(acc);
}

constexpr int64_t kStepRows = 128;  // most tokens that go one by one

template <bool half>
void launch(const ws_adapters_call& c, uint2* h, cudaStream_t s) {
  const int rpad = adapters_rank(c.r);
  const bool vecB = c.r % 4 == 0 && reinterpret_cast<uintptr_t>(c.B) % 8 == 0 && c.ldb % 4 == 0 && c.strideB % 4 == 0;
  const auto rows16 = [](const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; };
  const unsigned T = static_cast<unsigned>(c.nrows);
  if (c.nrows <= kStepRows) {
    if (c.nnz > 0) {
      const unsigned split = static_cast<unsigned>(rpad / 2 / (kAdWarps / kStepSplit));
      shrink_step_kernel<half><<<dim3(T, split), kAdThreads, 0, s>>>(c, h, rpad);
    }
    expand_step_kernel<half><<<dim3(static_cast<unsigned>((c.N + kAdThreads - 1) / kAdThreads), T), kAdThreads, 0, s>>>(c, h, rpad, vecB);
    return;
  }
  const unsigned tiles = (T + kTileTok - 1) / kTileTok;
  if (c.nnz > 0) {
    const auto run = [&](auto nr) {
      constexpr int NR = decltype(nr)::value;
      constexpr int smem = kAdWarps * kTileTok * 8 * NR * static_cast<int>(sizeof(float));
      if (smem > 48 * 1024)
        cudaFuncSetAttribute(reinterpret_cast<const void*>(shrink_tile_kernel<half, NR>), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      shrink_tile_kernel<half, NR><<<dim3(tiles, static_cast<unsigned>((rpad + 8 * NR - 1) / (8 * NR))), kAdThreads, smem, s>>>(c, h, rpad);
    };
    if (rpad <= 16) run(std::integral_constant<int, 2>());
    else if (rpad <= 32) run(std::integral_constant<int, 4>());
    else run(std::integral_constant<int, 8>());
  }
  const bool vec = c.N % 8 == 0 && (!c.base || rows16(c.base, c.ldbase)) && rows16(c.y, c.ldy);
  const auto expand = vec ? expand_tile_kernel<half, true> : expand_tile_kernel<half, false>;
  expand<<<dim3(tiles, static_cast<unsigned>((c.N + 64 * kAdWarps - 1) / (64 * kAdWarps))), kAdThreads, 0, s>>>(c, h, rpad, vecB);
}

}  // namespace

void launch_adapters(const ws_adapters_call& c, void* scratch, cudaStream_t s) {
  if (c.dtype == WS_F16) launch<true>(c, static_cast<uint2*>(scratch), s);
  else launch<false>(c, static_cast<uint2*>(scratch), s);
}

}  // namespace wsk
