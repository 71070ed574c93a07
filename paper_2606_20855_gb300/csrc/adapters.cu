// Low-rank adapters of many requests at once, beside a projection they share:
//   y[t] = base[t] + sum over row t of S of  v * B[a] (A[a] x[t])
// S: tokens x adapters in CSR (a column and value per adapter of a token, none
// for most), A: adapters x rank x K, B: adapters x N x rank, 16-bit; base is the
// shared projection's result.
//
// Two kernels: inner products h = A[a] x[t] for every entry of S, then
// y = base + B[a] (v h).  Both are bound by memory (x, base and y, and the met
// adapters, once each; 2 rank multiply-adds per value), so h stays small: sums
// are 32-bit, and where v h meets B on the tensor cores (many tokens) it is a pair of 16-bit values, its rounding and the
// rounding of what that left over.
// One 16-bit value would add an error as large as the result's own rounding.
// A pair of bfloat16 holds 16 significant bits over the range of floats.  Halves end at 65504 and 2^-24, so a token's v h are
// multiplied by a power of two, which its sums are divided by: the one that brings the largest of the token's first 32 ranks to
// 2^10 .. 2^11.  The pair then is off by at most 2^-23 of a value, plus 2^-35 of the largest one.  Further ranks and
// adapters of the token are multiplied by the same power; if that leaves the largest of 32 of them outside 1 .. 2^15, where
// the second bound would be above 2^-25 of it, or it overflows, the token's values are computed one by one in 32 bits.
//
// Few tokens ("step"): every token is on its own, its inner products split over warps, then
// a thread per value of y: everything in flight at once, no
// reuse.  Many tokens ("prompt"): tiles of 128 tokens on the tcgen05 tensor cores, x, A, B, base and y moved by the copy engine.
// The tokens of a tile mostly share an adapter, and the tile goes
// through the adapters it meets in ascending order: every thread stands at its
// token's first entry, the smallest column among the threads is next, and the
// threads that have it move on (columns ascend within a row).
#include <climits>

#include "routing.cuh"
#include "tensor.cuh"

namespace wsk {
namespace {

constexpr int kAdThreads = 256;
constexpr int kAdWarps = kAdThreads / 32;

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

// Of the largest |v h| of 32 ranks of a token, when halves are to hold them: the power of two that the token has, or gets now
// (0: none yet), and whether that does not fit these ranks.  Below 2^-60 they are less than any half, whatever B holds.
struct HalfScale {
  float power;
  bool unfit;
};
__device__ __forceinline__ HalfScale half_scale(float power, float largest) {
  if (!(largest > 8.7e-19f && largest <= 3.4e38f)) return {power, false};
  if (power == 0.0f) {  // 2^(10 - e) for a largest of 2^e and more
    const int e = static_cast<int>(__float_as_uint(largest) >> 23) - 127;
    power = __uint_as_float(static_cast<uint32_t>(10 - e + 127) << 23);
  }
  const float z = largest * power;
  return {power, !(z >= 1.0f && z <= 32768.0f)};
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

constexpr int kTok = 128;           // tokens of a tile: lanes of tensor memory
constexpr int kRankBlock = 64;      // ranks, of one adapter or of several, that a pass over x takes
constexpr int kShrinkStages = 8;
constexpr int kShrinkStage = kTok * 128 + kRankBlock * 128;  // 64 values of x's and of A's rows
constexpr int kShrinkThreads = 192;
constexpr size_t kShrinkSmem = kShrinkStages * kShrinkStage + 1024;
constexpr int kList = 64;           // adapters that a tile collects at once
constexpr int kMaxSplit = 4;        // parts of K

// The smallest column at which the CTA's tokens stand (INT_MAX: none).  All threads call it; those without a token with INT_MAX.
template <int kWarps>
__device__ __forceinline__ int next_adapter(int col, int* mins) {
  const int m = __reduce_min_sync(0xffffffffu, col);
  if ((threadIdx.x & 31) == 0) mins[threadIdx.x >> 5] = m;
  __syncthreads();
  int a = mins[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) a = min(a, mins[i]);
  __syncthreads();
  return a;
}

// h of 128 tokens over one part of K: one lane fetches x's and A's values through a ring of stages, one multiplies (D: tokens x
// ranks, two accumulators), a thread per token stores.  Adapters of up to 32 or 16 ranks go two or four to a pass: a tile at
// the border of two requests then reads x once, like the others.  (8191 tokens of 4096 halves, rank 32, 67 MB of x, 10 us at the copy
// rate: 16 us; 24 us with tiles of 32 tokens on the warp-level instruction, 29 us with a pass for each adapter, 19 us without
// asking for a stage ahead.)
__global__ void __launch_bounds__(kShrinkThreads, 1)
    shrink_tile_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a,
                       const ws_adapters_call c, float* __restrict__ h, int rpad, int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full_bar[kShrinkStages], empty_bar[kShrinkStages], acc_full[2], acc_empty[2], last_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  __shared__ int list[kList], mins[kShrinkThreads / 32];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTok;
  const int r0 = blockIdx.z * kRankBlock, n = min(kRankBlock, rpad - r0);  // of one adapter
  const int group = kRankBlock / min(kRankBlock, rpad);                      // adapters of a pass
  const int all = static_cast<int>((c.K + 63) / 64);
  const int k0 = static_cast<int>(static_cast<int64_t>(all) * blockIdx.y / gridDim.y);
  const int k1 = static_cast<int>(static_cast<int64_t>(all) * (blockIdx.y + 1) / gridDim.y);
  h += static_cast<int64_t>(blockIdx.y) * c.nnz * rpad;
  may_start_next();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kShrinkStages; ++i) {
      bar_init(smem_u32(&full_bar[i]), 1);
      bar_init(smem_u32(&empty_bar[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(smem_u32(&acc_full[i]), 1);
      bar_init(smem_u32(&acc_empty[i]), 4);
    }
    bar_init(smem_u32(&last_bar), 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<2 * kRankBlock>(smem_u32(&tmem_slot));
  // warps 2 .. 5: a token a thread, in the lanes of tensor memory that the warp may read
  const int quarter = warp & 3, m = quarter * 32 + lane;
  Walk ahead, behind;  // the list is made ahead of what the stores have come to
  ahead.at = ahead.end = 0;
  ahead.col = INT_MAX;
  if (warp >= 2) ahead.start(c, t0 + m);
  behind = ahead;
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;

  int stage = 0, acc = 0;
  uint32_t phase = 0, acc_phase = 0;
  int filled = 0;
  bool ok = true, ready = false;  // ready: the role's next stage is known to be empty, or full
  for (;;) {
    int items = 0;
    while (items < kList) {
      const int a = next_adapter<kShrinkThreads / 32>(ahead.col, mins);
      if (a == INT_MAX) break;
      if (threadIdx.x == 0) list[items] = a;
      if (ahead.col == a) ahead.next(c);
      ++items;
    }
    __syncthreads();
    if (items == 0) break;
    if (warp == 0) {
      if (elect_one()) {
        for (int i = 0; ok && i < items; i += group) {
          const int these = min(group, items - i);
          for (int k = k0; k < k1; ++k) {
            if (!ready && !bar_wait(smem_u32(&empty_bar[stage]), phase ^ 1, &dead)) {
              ok = false;
              break;
            }
            const int next = stage + 1 == kShrinkStages ? 0 : stage + 1;
            const uint32_t next_phase = next == 0 ? phase ^ 1 : phase;
            ready = bar_ask(smem_u32(&empty_bar[next]), next_phase ^ 1);
            const uint32_t bar = smem_u32(&full_bar[stage]), at = base + stage * kShrinkStage;
            const int rows = min(kRankBlock, rpad);  // of the copy; past r they are zero
            bar_expect(bar, kTok * 128 + these * rows * 128);
            tma_2d(at, &map_x, 64 * k, static_cast<int>(t0), bar);
            for (int j = 0; j < these; ++j) tma_3d(at + kTok * 128 + j * rows * 128, &map_a, 64 * k, r0, list[i + j], bar);
            ++filled;
            stage = next;
            phase = next_phase;
          }
        }
      }
    } else if (warp == 1) {
      if (elect_one()) {
        for (int i = 0; ok && i < items; i += group) {
          const uint32_t idesc = instr_desc(c.dtype == WS_F16, false, false, kTok, n * min(group, items - i));
          ok = bar_wait(smem_u32(&acc_empty[acc]), acc_phase ^ 1, &dead);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          for (int k = k0; ok && k < k1; ++k) {
            ok = ready || bar_wait(smem_u32(&full_bar[stage]), phase, &dead);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int next = stage + 1 == kShrinkStages ? 0 : stage + 1;
            const uint32_t next_phase = next == 0 ? phase ^ 1 : phase;
            ready = bar_ask(smem_u32(&full_bar[next]), next_phase);
            const uint32_t at = base + stage * kShrinkStage;
            const uint64_t da = smem_desc(at, false), db = smem_desc(at + kTok * 128, false);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              mma_f16(tmem + acc * kRankBlock, da + j * (32 >> 4), db + j * (32 >> 4), idesc, k > k0 || j > 0);
            mma_commit(smem_u32(&empty_bar[stage]));
            if (k == k1 - 1) mma_commit(smem_u32(&acc_full[acc]));
            stage = next;
            phase = next_phase;
          }
          if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
      }
    } else {
      for (int i = 0; ok && i < items; ++i) {
        const int at = i % group;
        if (at == 0) {
          ok = bar_wait_warp(smem_u32(&acc_full[acc]), acc_phase, &dead);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
        const bool mine = behind.col == list[i];
        for (int j = 0; j < n; j += 16) {
          float f[16];
          tmem_load16(tmem + acc * kRankBlock + at * n + j + (static_cast<uint32_t>(quarter * 32) << 16), f);
          if (mine) {
            if (r0 + j + 16 > c.r) {  // past the rank: zero, also where x is infinite (times a zero that the copy filled in)
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (r0 + j + e >= c.r) f[e] = 0.0f;
            }
            float4* dst = reinterpret_cast<float4*>(h + static_cast<int64_t>(behind.at) * rpad + r0 + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[e] = make_float4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
          }
        }
        if (mine) behind.next(c);
        if (at == group - 1 || i == items - 1) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(smem_u32(&acc_empty[acc]));
          if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
      }
    }
    __syncwarp();
    __syncthreads();
    if (items < kList || dead) break;
  }
  if (dead) {  // no copy and no product may be in flight when the CTA leaves
    // by the lanes that copied and multiplied
    if (warp == 0 && elect_one())
      for (int f = max(0, filled - kShrinkStages); f < filled; ++f)
        bar_wait_short(smem_u32(&full_bar[f % kShrinkStages]), static_cast<uint32_t>(f / kShrinkStages) & 1);
    if (warp == 1 && elect_one()) {
      mma_commit(smem_u32(&last_bar));
      bar_wait_short(smem_u32(&last_bar), 0);
      atomicOr(status, 1);
    }
    __syncwarp();
    __syncthreads();
  }
  if (warp == 1) tmem_free<2 * kRankBlock>(tmem);
}

constexpr int kExpandThreads = 256;  // two threads a token
constexpr int kExpandN = 256;        // values of y a CTA takes of every token
constexpr int kExpandRanks = 32;     // ranks multiplied at once: 64 bytes of roundings and 64 of remainders a row
constexpr int kExpandA = kTok * 128, kExpandB = kExpandN * 64, kExpandY = kTok * 128;  // bytes; y in four pieces of 64 values
constexpr size_t kExpandSmem = kExpandA + kExpandB + 4 * kExpandY + 1024;

// h of an entry, rank j: the parts of K summed, times the entry's value.
__device__ __forceinline__ float4 scaled_h(const ws_adapters_call& c, const float* h, int rpad, int split, int entry, int j, float v) {
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i = 0; i < split; ++i) {
    const float4 f = *reinterpret_cast<const float4*>(h + (static_cast<int64_t>(i) * c.nnz + entry) * rpad + j);
    s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
  }
  return make_float4(v * s.x, v * s.y, v * s.z, v * s.w);
}

// What the adapters add to value n of token t, by itself.
template <bool half>
__device__ __noinline__ float added(const ws_adapters_call& c, const float* h, int rpad, int split, int64_t t, int64_t n) {
  Walk w;
  float sum = 0.0f;
  for (w.start(c, t); w.col != INT_MAX; w.next(c)) {
    const uint16_t* row = static_cast<const uint16_t*>(c.B) + w.col * c.strideB + n * c.ldb;
    for (int j = 0; j < c.r; j += 4) {
      const float4 f = scaled_h(c, h, rpad, split, w.at, j, c.vals[w.at]);
      const float v[4] = {f.x, f.y, f.z, f.w};
      for (int i = 0; i < 4 && j + i < c.r; ++i) sum = fmaf(v[i], value16<half>(row[j + i]), sum);
    }
  }
  return sum;
}

// 256 values of 128 tokens: base arrives while the products run; the sums go through the same piece of shared memory to y.  Two
// CTAs share an SM, so that one's latencies (row pointer, column, h and B, product, store) pass under the other's
// work.  8192 tokens of 12 requests, 2048 values: 14 us without adapters (base to y, 67 MB; 10 us at the copy rate), 24 us
// (bfloat16) and 25.6 us (half, whose power of two is sought) with rank 16, 25.7 and 27.4 us with rank 32.  In half, before that power:
// 24 us with rank 32; on the warp-level instruction 31 us, with a CTA that keeps v h for two columns 34 us, with a thread for each token's
// v h 25-28 us (its loads touch 32 rows at a time).  128 columns a CTA: inner products and sums take 51.7 us with three CTAs an SM and
// 60.2 with four, where this took 44.4, because each CTA goes through h again.
template <bool half>
__global__ void __launch_bounds__(kExpandThreads, 2)
    expand_tile_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_base,
                       const __grid_constant__ CUtensorMap map_y, const ws_adapters_call c, const float* h,
                       int rpad, int split, bool copies, int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t base_bar, b_bar, m_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  __shared__ int mins[kExpandThreads / 32], entry[kTok];
  __shared__ float value[kTok], power[half ? kTok : 1];  // power: of two, for v h of the token (0: none yet)
  __shared__ bool alone[half ? kTok : 1];                // the token's values are computed one by one
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = threadIdx.x & (kTok - 1), side = threadIdx.x / kTok;
  const uint32_t sa = (smem_u32(raw) + 1023u) & ~1023u, sy = sa + kExpandA, sb = sy + 4 * kExpandY;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTok, t = t0 + m;
  const int N = static_cast<int>(c.N);
  const int n0 = blockIdx.y * kExpandN;
  const int pieces = min(4, (N - n0 + 63) / 64);  // of 64 values that are there
  const bool there = t < c.nrows;
  // S and base are there before the inner products start; without those, what comes before is another call, which may write them
  if (c.nnz == 0) wait_for_last();
  if (threadIdx.x == 0) {
    bar_init(smem_u32(&base_bar), 1);
    bar_init(smem_u32(&b_bar), 1);
    bar_init(smem_u32(&m_bar), 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (copies && c.base) {
      bar_expect(smem_u32(&base_bar), pieces * kExpandY);
      for (int i = 0; i < pieces; ++i) tma_2d(sy + i * kExpandY, &map_base, n0 + 64 * i, static_cast<int>(t0), smem_u32(&base_bar));
    }
  }
  if (warp == 0) tmem_alloc<kExpandN>(smem_u32(&tmem_slot));
  if constexpr (half)
    if (side == 0) power[m] = 0.0f, alone[m] = false;
  Walk w;
  w.start(c, t);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  const uint32_t idesc = instr_desc(half, false, false, kTok, kExpandN);

  int done = 0;        // products of 32 ranks
  bool mixed = false;  // some token does not have some adapter of the tile
  for (;;) {
    const int a = next_adapter<kExpandThreads / 32>(w.col, mins);
    if (a == INT_MAX || dead) break;  // dead was set before the barrier in there, or is not for a while
    const bool mine = w.col == a;
    if (side == 0) {
      entry[m] = mine ? w.at : -1;
      value[m] = mine ? c.vals[w.at] : 0.0f;
    }
    __syncthreads();
    for (int r0 = 0; r0 < rpad; r0 += kExpandRanks) {
      const int ranks = min(kExpandRanks, rpad - r0);  // 16 or 32
      if (done > 0) bar_wait(smem_u32(&m_bar), (done - 1) & 1, &dead);  // what reads A and B is over
      if (threadIdx.x == 0 && !dead) {
        bar_expect(smem_u32(&b_bar), kExpandB);
        tma_3d(sb, &map_b, r0, n0, a, smem_u32(&b_bar));
      }
      if (done == 0) wait_for_last();  // the inner products
      // v h of 128 tokens, four ranks a thread and turn, neighbouring threads along a token's ranks; all loads in flight at once
      const int log_quads = ranks == kExpandRanks ? 3 : 2;
      constexpr int kTurns = kTok * (kExpandRanks / 4) / kExpandThreads;
      float4 part[kTurns][kMaxSplit];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int at = threadIdx.x + kExpandThreads * i, e = at >> log_quads < kTok ? entry[at >> log_quads] : -1;
#pragma unroll
        for (int k = 0; k < kMaxSplit; ++k)
          part[i][k] = e >= 0 && k < split ? *reinterpret_cast<const float4*>(h + (static_cast<int64_t>(k) * c.nnz + e) * rpad + r0 +
                                                                               4 * (at & ((1 << log_quads) - 1)))
                                           : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      }
      float4 vh[kTurns];
      float had[kTurns], largest[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int row = (threadIdx.x + kExpandThreads * i) >> log_quads;
        float4 f = part[i][0];
#pragma unroll
        for (int k = 1; k < kMaxSplit; ++k) f.x += part[i][k].x, f.y += part[i][k].y, f.z += part[i][k].z, f.w += part[i][k].w;
        const float s = row < kTok ? value[row] : 0.0f;
        vh[i] = make_float4(s * f.x, s * f.y, s * f.z, s * f.w);
        if constexpr (half) {
          had[i] = row < kTok ? power[row] : 0.0f;
          largest[i] = fmaxf(fmaxf(fabsf(vh[i].x), fabsf(vh[i].y)), fmaxf(fabsf(vh[i].z), fabsf(vh[i].w)));
        }
      }
      if constexpr (half) {  // of all ranks of a token, which neighbouring lanes hold
        for (int o = 1; o < 1 << log_quads; o <<= 1)
#pragma unroll
          for (int i = 0; i < kTurns; ++i) largest[i] = fmaxf(largest[i], __shfl_xor_sync(0xffffffffu, largest[i], o));
        __syncwarp();  // all of them have read its power
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int at = threadIdx.x + kExpandThreads * i, row = at >> log_quads, quad = at & ((1 << log_quads) - 1);
        if (row >= kTok) break;
        float4 f = vh[i];
        if constexpr (half) {
          const HalfScale now = half_scale(had[i], largest[i]);
          if (quad == 0) {
            power[row] = now.power;
            if (now.unfit) alone[row] = true;
          }
          if (now.power != 0.0f) f = make_float4(now.power * f.x, now.power * f.y, now.power * f.z, now.power * f.w);
        }
        const uint2 a01 = split_pair<half>(f.x, f.y), a23 = split_pair<half>(f.z, f.w);
        const uint32_t to = sa + row * 128 + 8 * (quad & 1), hi = to + (((quad >> 1) ^ (row & 7)) << 4),
                       lo = to + (((4 + (quad >> 1)) ^ (row & 7)) << 4);
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(hi), "r"(a01.x), "r"(a23.x) : "memory");
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(lo), "r"(a01.y), "r"(a23.y) : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      if (!__syncthreads_and(mine || !there)) mixed = true;
      if (dead) {  // this turn's copy may be in flight; it is not among those that are waited for on the way out
        if (threadIdx.x == 0) bar_wait_short(smem_u32(&b_bar), done & 1);
        break;
      }
      if (threadIdx.x == 0 && bar_wait(smem_u32(&b_bar), done & 1, &dead)) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t da = smem_desc(sa, false), db = smem_desc64(sb);
        for (int j = 0; j < ranks / 16; ++j) {
          mma_f16(tmem, da + j * (32 >> 4), db + j * (32 >> 4), idesc, done > 0 || j > 0);
          mma_f16(tmem, da + ((64 + 32 * j) >> 4), db + j * (32 >> 4), idesc, true);
        }
        mma_commit(smem_u32(&m_bar));
      }
      ++done;
    }
    if (mine) w.next(c);
  }
  if (done == 0) wait_for_last();  // the kernel ends after the one before
  // Without the copy engine (rows that do not start at multiples of 16 bytes) the warps move base and y along their rows.
  const auto place = [&](int row, int col) { return sy + (col >> 6) * kExpandY + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4) + 2 * (col & 7); };
  const int columns = min(kExpandN, N - n0);
  const int64_t rows = min(static_cast<int64_t>(kTok), c.nrows - t0);
  if (!copies && c.base) {
    const uint16_t* src = static_cast<const uint16_t*>(c.base) + t0 * c.ldbase + n0;
    for (int row = warp; row < rows; row += kExpandThreads / 32) {
      uint16_t v[kExpandN / 32];
#pragma unroll
      for (int i = 0; i < kExpandN / 32; ++i) v[i] = 32 * i + lane < columns ? src[row * c.ldbase + 32 * i + lane] : 0;
#pragma unroll
      for (int i = 0; i < kExpandN / 32; ++i)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(place(row, 32 * i + lane)), "h"(v[i]) : "memory");
    }
  }
  if (done > 0) bar_wait(smem_u32(&m_bar), (done - 1) & 1, &dead);
  if (copies && c.base) bar_wait(smem_u32(&base_bar), 0, &dead);
  __syncthreads();
  if (!dead) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const bool by_itself = half && alone[half ? m : 0];
    const float times = half && !by_itself && power[half ? m : 0] != 0.0f ? power[half ? m : 0] : 1.0f, back = 1.0f / times;  // exact
#pragma unroll 1
    for (int q = 2 * side; q < 2 * side + 2 && q < pieces; ++q) {  // 64 columns, stored as soon as they are there
#pragma unroll 1
      for (int j = 64 * q; j < 64 * q + 64; j += 16) {
        const int left = N - n0 - j;
        if (left <= 0) break;
        float f[16] = {};
        __syncwarp();
        if (done > 0) tmem_load16(tmem + j + (static_cast<uint32_t>((warp & 3) * 32) << 16), f);
        if ((mixed || by_itself) && there) {
          // A token without an adapter got zero times its values: nothing, unless those are infinite or NaN.
          for (int i = 0; i < 16; ++i)
            if (i < left && (by_itself || !(fabsf(f[i]) <= 3.4e38f))) f[i] = times * added<half>(c, h, rpad, split, t, n0 + j + i);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const uint32_t at = place(m, j + 8 * s);
          uint32_t b[4] = {};
          if (c.base)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]) : "r"(at) : "memory");
#pragma unroll
          for (int i = 0; i < 4; ++i)
            b[i] = pair16<half>(fmaf(f[8 * s + 2 * i], back, value16<half>(static_cast<uint16_t>(b[i]))),
                                fmaf(f[8 * s + 2 * i + 1], back, value16<half>(static_cast<uint16_t>(b[i] >> 16))));
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]) : "memory");
        }
      }
      if (copies) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync %0, %1;" ::"r"(1 + side), "r"(kTok) : "memory");  // the side's threads
        if (m == 0) {
          tma_store_2d(&map_y, sy + q * kExpandY, n0 + 64 * q, static_cast<int>(t0));
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
    }
    if (copies && m == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  }
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0 && dead) {  // no copy and no product may be in flight when the CTA leaves
    atomicOr(status, 1);
    if (done > 0) bar_wait_short(smem_u32(&b_bar), (done - 1) & 1), bar_wait_short(smem_u32(&m_bar), (done - 1) & 1);
    if (copies && c.base) bar_wait_short(smem_u32(&base_bar), 0);
  }
  if (!copies && !dead) {
    uint16_t* dst = static_cast<uint16_t*>(c.y) + t0 * c.ldy + n0;
    for (int row = warp; row < rows; row += kExpandThreads / 32) {
      uint16_t v[kExpandN / 32];
#pragma unroll
      for (int i = 0; i < kExpandN / 32; ++i)
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[i]) : "r"(place(row, 32 * i + lane)) : "memory");
#pragma unroll
      for (int i = 0; i < kExpandN / 32; ++i)
        if (32 * i + lane < columns) dst[row * c.ldy + 32 * i + lane] = v[i];
    }
  }
  __syncwarp();
  __syncthreads();
  if (warp == 0) tmem_free<kExpandN>(tmem);
}

// ---------------------------------------------------------------- few tokens

// A CTA per token and two pairs of ranks: four warps a pair, each with a quarter of K.  (One warp a pair: 12.4 us for 48 tokens
// of 4096 values and rank 16, the time of a lane's 16 steps of loads; so 6.4 us.)
constexpr int kStepSplit = 4;

// vec: the rows of x and A start at multiples of 16 bytes.
template <bool half, bool vec>
__global__ void __launch_bounds__(kAdThreads) shrink_step_kernel(const ws_adapters_call c, float2* __restrict__ h, int rpad) {
  __shared__ float2 part[kAdWarps];
  may_start_next();
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
      for (; vec && k - 8 * lane + kStep * (U - 1) + 256 <= K; k += kStep * U) {
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
      for (; k < K; k += kStep) add(load8(x, k, K, vec), load8(A0, k, K, vec), load8(A1, k, K, vec));
    }
    s0 = warp_sum(s0);
    s1 = warp_sum(s1);
    if (lane == 0) part[warp] = make_float2(s0, s1);
    __syncthreads();
    if (lane == 0 && warp % kStepSplit == 0) {
#pragma unroll
      for (int i = 1; i < kStepSplit; ++i) s0 += part[warp + i].x, s1 += part[warp + i].y;
      const float v = c.vals[e];
      h[static_cast<int64_t>(e) * pairs + p] = make_float2(2 * p < r ? v * s0 : 0.0f, 2 * p + 1 < r ? v * s1 : 0.0f);
    }
    __syncthreads();
  }
}

// A thread per value of y: its row of B against v h, which every thread of the CTA reads.  Bound by latencies: 48 tokens of rank 16,
// 4096 values, 6.3 MB of B: 5 us, of which what does not need h passes while the inner products run (four
// tokens of 512 values, both kernels: 6.8 us without, 5.1 us with that).
template <bool half>
__global__ void __launch_bounds__(kAdThreads) expand_step_kernel(const ws_adapters_call c, const float2* h, int rpad, bool vecB) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * kAdThreads + threadIdx.x, t = blockIdx.y;
  if (n >= c.N) return;
  if (c.nnz == 0) wait_for_last();  // as in the tiles: another call may write base
  const int r = static_cast<int>(c.r);
  int begin, end;
  entry_range(c.rowptr, t, c.nnz, &begin, &end);
  float acc = c.base ? value16<half>(static_cast<const uint16_t*>(c.base)[t * c.ldbase + n]) : 0.0f;
  if (begin < end) {
    const int a = c.colidx[begin];
    if (met(c, a)) asm volatile("prefetch.global.L1 [%0];" ::"l"(static_cast<const uint16_t*>(c.B) + a * c.strideB + n * c.ldb));
  }
  wait_for_last();  // the inner products
  for (int e = begin; e < end; ++e) {
    const int a = c.colidx[e];
    if (!met(c, a)) continue;
    const uint16_t* row = static_cast<const uint16_t*>(c.B) + a * c.strideB + n * c.ldb;
    const float4* hv = reinterpret_cast<const float4*>(h + static_cast<int64_t>(e) * (rpad / 2));
#pragma unroll 4
    for (int k = 0; k < r; k += 4) {
      const uint2 b = load4(row, k, r, vecB);
      const float4 p = hv[k / 4];
      acc = fmaf(p.x, value16<half>(static_cast<uint16_t>(b.x)), acc);
      acc = fmaf(p.y, value16<half>(static_cast<uint16_t>(b.x >> 16)), acc);
      acc = fmaf(p.z, value16<half>(static_cast<uint16_t>(b.y)), acc);
      acc = fmaf(p.w, value16<half>(static_cast<uint16_t>(b.y >> 16)), acc);
    }
  }
  static_cast<uint16_t*>(c.y)[t * c.ldy + n] = bits16<half>(acc);
}

template <bool half>
ws_status_t launch_step(const ws_adapters_call& c, float2* h, cudaStream_t s) {
  const int rpad = adapters_rank(c.r);
  const bool vecB = c.r % 4 == 0 && reinterpret_cast<uintptr_t>(c.B) % 8 == 0 && c.ldb % 4 == 0 && c.strideB % 4 == 0;
  const unsigned T = static_cast<unsigned>(c.nrows);
  const auto rows16 = [](const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; };
  const bool vec = rows16(c.x, T > 1 ? c.ldx : 0) && rows16(c.A, c.r > 1 ? c.lda : 0) && (c.ncols <= 1 || c.strideA % 8 == 0);
  const auto shrink = vec ? shrink_step_kernel<half, true> : shrink_step_kernel<half, false>;
  if (c.nnz > 0)
    shrink<<<dim3(T, static_cast<unsigned>(rpad / 2 / (kAdWarps / kStepSplit))), kAdThreads, 0, s>>>(c, h, rpad);
  const dim3 grid(static_cast<unsigned>((c.N + kAdThreads - 1) / kAdThreads), T);
  const cudaError_t e = launch_early(expand_step_kernel<half>, grid, kAdThreads, 0, s, 1, c, h, rpad, vecB);
  if (e != cudaSuccess) return routing_fail(WS_ERR_CUDA, "adapters: %s", cudaGetErrorString(e));
  return WS_OK;
}

ws_status_t launch_prompt(const ws_adapters_call& c, float* h, int* status, int num_sms, cudaStream_t s) {
  const int rpad = adapters_rank(c.r);
  const bool half = c.dtype == WS_F16;
  const unsigned tiles = static_cast<unsigned>((c.nrows + kTok - 1) / kTok);
  int split = 1;
  if (!encoder()) return routing_fail(WS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int), s);
  if (e != cudaSuccess) return routing_fail(WS_ERR_CUDA, "adapters: %s", cudaGetErrorString(e));
  CUtensorMap x{}, a{}, b{};
  // a grid's y has 65535 CTAs at most: rows of 2^24 values take two launches of the sums
  constexpr int64_t kMost = int64_t{65535} * kExpandN;
  const auto describe_b = [&](const void* from, int64_t rows) {
    return c.nnz == 0 || encode(&b, from, half, c.r, rows, c.ldb, c.ncols, c.strideB, kExpandN, kExpandRanks);
  };
  if (c.nnz > 0) {
    // parts of K until every SM has a CTA
    const int64_t steps = (c.K + 63) / 64;
    while (split < kMaxSplit && 2 * split <= steps && tiles * split < static_cast<unsigned>(num_sms) / 2) split *= 2;
    if (!encode(&x, c.x, half, c.K, c.nrows, c.ldx, 0, 0, kTok) ||
        !encode(&a, c.A, half, c.K, c.r, c.lda, c.ncols, c.strideA, rpad < kRankBlock ? rpad : kRankBlock) ||
        !describe_b(c.B, c.N < kMost ? c.N : kMost))
      return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(shrink_tile_kernel), cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(kShrinkSmem));
    if (e != cudaSuccess) return routing_fail(WS_ERR_CUDA, "adapters: %s", cudaGetErrorString(e));
    const dim3 grid(tiles, static_cast<unsigned>(split), static_cast<unsigned>((rpad + kRankBlock - 1) / kRankBlock));
    shrink_tile_kernel<<<grid, kShrinkThreads, kShrinkSmem, s>>>(x, a, c, h, rpad, status);
  }
  const auto kernel = half ? expand_tile_kernel<true> : expand_tile_kernel<false>;
  e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize,
                           static_cast<int>(kExpandSmem));
  if (e != cudaSuccess) return routing_fail(WS_ERR_CUDA, "adapters: %s", cudaGetErrorString(e));
  for (int64_t n = 0; n < c.N; n += kMost) {
    ws_adapters_call p = c;
    p.N = c.N - n < kMost ? c.N - n : kMost;
    if (n > 0 && c.nnz > 0) p.B = static_cast<const uint16_t*>(c.B) + n * c.ldb;
    if (c.base) p.base = static_cast<const uint16_t*>(c.base) + n;
    p.y = static_cast<uint16_t*>(c.y) + n;
    if (n > 0 && !describe_b(p.B, p.N)) return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
    CUtensorMap base{}, y{};
    // base and y by the copy engine where their rows start at multiples of 16 bytes, else by loads and stores
    const auto rows16 = [](const void* q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % 8 == 0; };
    bool copies = (!c.base || rows16(p.base, c.ldbase)) && rows16(p.y, c.ldy);
    if (copies && !(encode(&y, p.y, half, p.N, c.nrows, c.ldy, 0, 0, kTok) &&
                    (!c.base || encode(&base, p.base, half, p.N, c.nrows, c.ldbase, 0, 0, kTok))))
      copies = false;
    const dim3 grid(tiles, static_cast<unsigned>((p.N + kExpandN - 1) / kExpandN));
    e = launch_early(kernel, grid, kExpandThreads, kExpandSmem, s, 1, b, base, y, p, static_cast<const float*>(h), rpad, split, copies, status);
    if (e != cudaSuccess) return routing_fail(WS_ERR_CUDA, "adapters: %s", cudaGetErrorString(e));
  }
  return WS_OK;
}

}  // namespace

ws_status_t launch_adapters(const ws_adapters_call& c, void* scratch, int num_sms, cudaStream_t s) {
  char* h = static_cast<char*>(scratch) + 16;  // behind the status word
  if (!adapters_step(c.nrows, c.r)) return launch_prompt(c, reinterpret_cast<float*>(h), static_cast<int*>(scratch), num_sms, s);
  return c.dtype == WS_F16 ? launch_step<true>(c, reinterpret_cast<float2*>(h), s) : launch_step<false>(c, reinterpret_cast<float2*>(h), s);
}

}  // namespace wsk
