// Products by column of a routing matrix: every column (expert) e has a matrix
// W[e] (N x K) and, in slot order, the rows offsets[e] .. offsets[e + 1].
//   forward    ys[s]  = W[e] xs[s]                      contraction over K
//   rows       gxs[s] = W[e]^T gys[s]                   contraction over N
//   weights    gW[e]  = sum over s of gys[s] xs[s]^T    contraction over the rows of e
// bfloat16 or half operands, products and sums in 32 bits on the tensor cores
// (tcgen05, accumulators in tensor memory), one rounding when a result is stored.
//
// One persistent CTA per SM: one warp's lane fetches operand tiles with TMA
// (128-byte swizzle, a ring of stages), one lane issues the matrix
// instructions, four warps store finished tiles while the next one is
// multiplied (two accumulators).  How many rows an expert has is known on the
// device only, so every CTA counts the tiles of all experts itself and takes
// every gridDim-th one.  Operands are read as they lie in memory: an operand
// whose contraction index runs along its rows (W in `rows`, both in `weights`)
// is given to the tensor cores as "MN-major", never transposed by a copy.
//
// Rows of the result behind the placed entries (there are some only if entries
// have no column) are zero, as in the rows that are moved.
// A tile of rows may reach past its expert's last row: such rows are computed
// and not stored.  In `weights` they would be summed, so the last stage is
// multiplied as far as it has rows, in steps of 16, and the rows past the end in the last
// step are cleared in shared memory (in both operands: 0 * inf is NaN).
#include <type_traits>

#include "routing.cuh"
#include "tensor.cuh"
#include "ws_internal.cuh"

namespace wsk {
namespace {

constexpr int kTileM = 128;   // rows of the M side: lanes of tensor memory
constexpr int kTileK = 64;    // 128 bytes: the swizzle's span
constexpr int kBytesA = kTileM * kTileK * 2;
constexpr int kTurnBytes = 32 * 128;
constexpr double kFewRows = 4;     // mean rows an expert up to which W's features fill the lanes, or warps read W by themselves
constexpr double kPairRows = 512;  // rows an expert from which on its row tiles go in pairs

// Where the rows of the experts are in the product D (M x N tile).
constexpr int kRowsM = 0;    // on the M side (lanes)
constexpr int kRowsN = 1;    // on the N side (columns): few rows per expert, W fills the lanes
constexpr int kRowsSum = 2;  // summed over

struct GroupedParams {
  const int64_t* offsets;
  int groups;
  int64_t nnz;
  int features;  // kRowsM, kRowsN: columns of the result; kRowsSum: rows of gW[e] (M side)
  int width;     // kRowsSum: columns of gW[e] (N side)
  int depth;     // contraction length; kRowsSum: unused
  void* out;
  int64_t ldo;   // values between rows of the result
  int64_t group_stride;  // kRowsSum: values between gW[e]
  bool half;
  int vec;       // rows of the result start at multiples of so many bytes: 16 (the copy engine may store them), 8, 4 or 2
  int* status;
};

__device__ __forceinline__ uint16_t round16(float f, bool half) {
  return half ? __half_as_ushort(__float2half_rn(f)) : __bfloat16_as_ushort(__float2bfloat16_rn(f));
}

// One tile of the product.
struct Tile {
  int group;
  int m0, n0;    // first lane and column, in features (or gW's rows and columns)
  int row0;      // first row of the experts' rows
  int rows;      // rows from row0 on that are the group's
  int steps;     // stages of the contraction
};

// A warp that copies, one that multiplies, four that store; where rows are summed over, one that clears.
template <int kRows>
constexpr int kThreadsOf = kRows == kRowsSum ? 224 : 192;

// Pieces of shared memory through which a storing warp's results go.
template <int kRows>
constexpr int kPieces = kRows == kRowsN ? 0 : kRows == kRowsM ? 1 : 2;

// Rows of a group in a tile, unless they are summed over.
template <int BN, int kRows>
constexpr int kRowTileOf = kRows == kRowsM ? kTileM : BN;

template <int BN, int kRows, bool kPair = false>
struct Shape {
  static constexpr int kBytesB = (kPair ? BN / 2 : BN) * kTileK * 2;
  static constexpr int kStageBytes = kBytesA + kBytesB;
  static constexpr int kStages = (196 * 1024) / kStageBytes > 10 ? 10 : (196 * 1024) / kStageBytes;
  static constexpr int kAccCols = 2 * BN < 32 ? 32 : 2 * BN;  // a power of two
  static constexpr size_t kSmem = static_cast<size_t>(kStages) * kStageBytes + 4 * kPieces<kRows> * kTurnBytes + 1024;
};

// Tile t of the sequence that all roles of all CTAs share.  first[e]: row tiles of the groups before e.  kPair: t is two
// tiles one below the other, of which `rank` is the CTA's.
template <int BN, int kRows, bool kPair>
__device__ __forceinline__ bool tile_at(const GroupedParams& p, const int* first, int64_t t, int rank, Tile* out) {
  constexpr int kSpan = kPair ? 2 * kTileM : kTileM;
  if constexpr (kRows == kRowsSum) {
    const int mt = (p.features + kSpan - 1) / kSpan, nt = (p.width + BN - 1) / BN;
    const int64_t each = static_cast<int64_t>(mt) * nt;
    if (t >= each * p.groups) return false;
    const int e = static_cast<int>(t / each);
    const int i = static_cast<int>(t - each * e);
    out->group = e;
    out->m0 = i % mt * kSpan + rank * kTileM;
    out->n0 = i / mt * BN;
    const int64_t b = p.offsets[e], n = p.offsets[e + 1] - b;
    out->row0 = static_cast<int>(b);
    out->rows = static_cast<int>(n);
    out->steps = static_cast<int>((n + kTileK - 1) / kTileK);
  } else {
    constexpr int kFeat = kRows == kRowsM ? BN : kTileM;
    constexpr int kRowTile = kPair ? kSpan : kRowTileOf<BN, kRows>;
    const int ft = (p.features + kFeat - 1) / kFeat;
    const int64_t q = t / ft;
    if (q >= first[p.groups]) return false;
    int lo = 0, hi = p.groups - 1;  // the last group with first[e] <= q; groups without rows have none of their own
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= q) lo = mid;
      else hi = mid - 1;
    }
    const int e = lo;
    const int rt = first[e + 1] - first[e];
    const int i = static_cast<int>(t - static_cast<int64_t>(first[e]) * ft);
    // eight row tiles side by side, so that CTAs at work together share rows and features in L2
    const int band = i / (8 * ft), in = i - band * 8 * ft;
    const int high = min(8, rt - 8 * band);
    const int r = 8 * band + in % high, f = in / high;
    out->group = e;
    const int64_t b = p.offsets[e];
    out->row0 = static_cast<int>(b) + r * kRowTile + rank * kTileM;
    out->rows = static_cast<int>(p.offsets[e + 1] - b) - r * kRowTile - rank * kTileM;  // none or fewer: nothing is stored
    out->m0 = kRows == kRowsM ? 0 : f * kFeat;
    out->n0 = kRows == kRowsM ? f * kFeat : 0;
    out->steps = (p.depth + kTileK - 1) / kTileK;
  }
  return true;
}

// Results leave a warp by 32 rows of 64 values, through 4 KB of shared memory: a row of 128 bytes a lane, its 16-byte pieces placed
// by the row's last three bits (the copy engine's 128-byte swizzle), so that lanes that write rows and lanes that read along them
// meet no bank twice.  From there the copy engine stores all 32 rows at once, where they start at multiples of 16 bytes and all are
// stored, while the warp turns to the next 64 columns in the other of two such pieces; else the warp stores along rows.  64 experts'
// gradients of 1024 x 2048 from 40 rows each, 268 MB written (40 us at the copy rate): 55 us, stored along rows 91 us (138 us with the
// values converted one by one, 96 us with eight warps, each half of the columns).  Where the experts' rows are the result's, one piece has
// to do, as the row tiles of all experts are counted in shared memory too.
__device__ __forceinline__ void put_rows(uint32_t turn, bool half, const float (&f)[64]) {
  const int lane = threadIdx.x & 31;
  uint32_t all[32];
  if (half) {
#pragma unroll
    for (int i = 0; i < 32; ++i) all[i] = pair16<true>(f[2 * i], f[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) all[i] = pair16<false>(f[2 * i], f[2 * i + 1]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t* w = all + 4 * j;
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(turn + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]),
                 "r"(w[2]), "r"(w[3])
                 : "memory");
  }
}

// Stores what put_rows left (from column 0 of dst on, `left` columns of them inside the result); on(row): the row is stored.
template <typename On>
__device__ __forceinline__ void store_turned(const GroupedParams& p, uint32_t turn, uint16_t* dst, int left, On on) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  // B bytes a lane: 16, 8, 4 or 2, as the rows of the result start
  const auto along = [&](auto bytes) {
    constexpr int B = decltype(bytes)::value, kValues = B / 2, kLanes = B == 2 ? 32 : 128 / B, kRowsAtOnce = 32 / kLanes;
    constexpr int kSides = 64 / (kLanes * kValues);  // 2 where a lane moves 2 bytes, else 1
#pragma unroll
    for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
      const int row = i * kRowsAtOnce + lane / kLanes;
#pragma unroll
      for (int side = 0; side < kSides; ++side) {
        const int col = kValues * (lane % kLanes) + 32 * side;
        Pack<uint16_t, kValues> v;
        const uint32_t at = turn + row * 128 + (((col >> 3) ^ (row & 7)) << 4) + 2 * (col & 7);
        if constexpr (B == 16) {
          uint32_t* w = reinterpret_cast<uint32_t*>(&v);
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
        } else if constexpr (B == 8) {
          uint32_t* w = reinterpret_cast<uint32_t*>(&v);
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
        } else if constexpr (B == 4) {
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(*reinterpret_cast<uint32_t*>(&v)) : "r"(at) : "memory");
        } else {
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v.v[0]) : "r"(at) : "memory");
        }
        if (!on(row)) continue;
        uint16_t* to = dst + row * p.ldo + col;
        if (col + kValues <= left) {
          *reinterpret_cast<Pack<uint16_t, kValues>*>(to) = v;
        } else {
#pragma unroll
          for (int e = 0; e < kValues; ++e)
            if (col + e < left) to[e] = v.v[e];
        }
      }
    }
  };
  if (p.vec == 16) along(std::integral_constant<int, 16>());
  else if (p.vec == 8) along(std::integral_constant<int, 8>());
  else if (p.vec == 4) along(std::integral_constant<int, 4>());
  else along(std::integral_constant<int, 2>());
  __syncwarp();
}

// Where rows are summed, a tile's last stage is fetched first and multiplied kAhead stages later than that place in the ring, so that its
// rows behind the group's last are cleared by then.  32 experts' gradients of 2048 x 2048 from about 1024 rows each: 177 us, 199 us in
// order (three stages later 178 us; 164-167 us where no stage is partly filled).
constexpr int kAhead = 2;
template <int kRows>
__device__ __forceinline__ bool tail_first(const Tile& t) {
  return kRows == kRowsSum && t.rows % kTileK != 0 && t.steps > kAhead;
}
// How far from its turn's place in the ring the stage of turn i lies.
__device__ __forceinline__ int ring_shift(bool tail_is_first, int i) { return !tail_is_first || i > kAhead ? 0 : i == kAhead ? -kAhead : 1; }

// a: the M side's operand (kRowsM: the experts' rows, kRowsN: W, kRowsSum: gys), b: the N side's.
// kWMN: W's contraction index runs along its rows (MN-major).
// kPair: two CTAs, whose tiles lie one below the other, multiply as one (256 x 256): each holds its 128 rows of the M side and half of
// the N side, so that a stage takes 32 KB of shared memory and of the way from L2 instead of 48, and six stages fit where four did.
// Rank 0 issues the products and counts both CTAs' bytes at its barriers (rank 1 counting its own and telling rank 0 cost a microsecond a
// stage).  8198 rows of eight experts, 2048 -> 8192: 169 us, 1630 TFLOP/s (about 200 us in a loop, at the power limit); 32768 rows of 32
// experts, 2048 x 2048: 167 us, 167 us for the rows' gradient and 179 us for the matrices' (about 620 us in a loop).  Before the steps
// that followed, the loops took 206 and 653 us with pairs, 214 and 665 us without.
template <int BN, int kRows, bool kWMN, bool kPair>
__global__ void __launch_bounds__(kThreadsOf<kRows>, 1)
    grouped_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_out, const GroupedParams p) {
  using S = Shape<BN, kRows, kPair>;
  constexpr bool kAMN = kRows == kRowsSum || (kRows == kRowsN && kWMN);
  constexpr bool kBMN = kRows == kRowsSum || (kRows == kRowsM && kWMN);
  constexpr int kHalfN = kPair ? BN / 2 : BN;  // of the N side in this CTA
  extern __shared__ uint8_t raw[];
  __shared__ int first[kRouteMaxCols + 1];
  __shared__ int scratch[32];
  __shared__ __align__(8) uint64_t full_bar[S::kStages], empty_bar[S::kStages], acc_full[2], acc_empty[2], last_bar;
  // stages with rows behind a group's last: have come, and are cleared
  __shared__ __align__(8) uint64_t tail_bar[kRows == kRowsSum ? S::kStages : 1], clear_bar[kRows == kRowsSum ? S::kStages : 1];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  const int rank = kPair ? blockIdx.x & 1 : 0;
  const int64_t team = kPair ? blockIdx.x >> 1 : blockIdx.x, teams = kPair ? gridDim.x >> 1 : gridDim.x;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      bar_init(smem_u32(&full_bar[i]), 1);
      bar_init(smem_u32(&empty_bar[i]), 1);
      if constexpr (kRows == kRowsSum) {
        bar_init(smem_u32(&tail_bar[i]), 1);
        bar_init(smem_u32(&clear_bar[i]), kPair ? 2 : 1);
      }
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(smem_u32(&acc_full[i]), 1);
      bar_init(smem_u32(&acc_empty[i]), kPair ? 8 : 4);
    }
    bar_init(smem_u32(&last_bar), 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<S::kAccCols, kPair>(smem_u32(&tmem_slot));
  wait_for_last();
  if constexpr (kRows != kRowsSum) {  // row tiles before every group
    int sum = 0;
    for (int e0 = 0; e0 < p.groups; e0 += kThreadsOf<kRows>) {
      const int e = e0 + threadIdx.x;
      constexpr int kRowTile = kPair ? 2 * kTileM : kRowTileOf<BN, kRows>;
      const int n = e < p.groups ? static_cast<int>((p.offsets[e + 1] - p.offsets[e] + kRowTile - 1) / kRowTile) : 0;
      int all = 0;
      const int before = block_exclusive_scan(n, scratch, &all);
      if (e < p.groups) first[e] = sum + before;
      sum += all;
    }
    if (threadIdx.x == 0) first[p.groups] = sum;
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (kPair) pair_sync();  // the other CTA's barriers are there
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  may_start_next();

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true, ready = false;  // ready: the stage is known to be empty
      Tile t;
      for (int64_t i = team; ok && tile_at<BN, kRows, kPair>(p, first, i, rank, &t); i += teams) {
        const bool swapped = tail_first<kRows>(t);
        for (int turn = 0; turn < t.steps; ++turn) {
          const int k = !swapped ? turn : turn == 0 ? t.steps - 1 : turn - 1;
          if (!ready && !bar_wait(smem_u32(&empty_bar[stage]), phase ^ 1, &dead)) {
            ok = false;
            break;
          }
          const int next = stage + 1 == S::kStages ? 0 : stage + 1;
          const uint32_t next_phase = next == 0 ? phase ^ 1 : phase;
          ready = bar_ask(smem_u32(&empty_bar[next]), next_phase ^ 1);
          const uint32_t sa = base + stage * S::kStageBytes, sb = sa + kBytesA;
          const int at = k * kTileK;
          const bool tail = kRows == kRowsSum && t.rows - at < kTileK;
          uint32_t bar = smem_u32(&full_bar[stage]);
          if (tail) {  // counted apart, for the warp that clears
            if (rank == 0) bar_arrive(bar);
            bar = smem_u32(&tail_bar[kRows == kRowsSum ? stage : 0]);
            bar_expect(bar, S::kStageBytes);
          } else if (!kPair) {
            bar_expect(bar, S::kStageBytes);
          } else if (rank == 0) {
            bar_expect(bar, 2 * S::kStageBytes);
          } else {
            bar = at_first(bar);
          }
          const auto copy2 = [&](uint32_t dst, const CUtensorMap* map, int x, int y) {
            if (kPair && rank == 1 && !tail) tma_2d_first(dst, map, x, y, bar);
            else tma_2d(dst, map, x, y, bar);
          };
          const auto copy3 = [&](uint32_t dst, const CUtensorMap* map, int x, int y, int z) {
            if (kPair && rank == 1 && !tail) tma_3d_first(dst, map, x, y, z, bar);
            else tma_3d(dst, map, x, y, z, bar);
          };
          if constexpr (kRows == kRowsM) {
            copy2(sa, &map_a, at, t.row0);
            if constexpr (kBMN) {
#pragma unroll
              for (int j = 0; j < kHalfN / 64; ++j) copy3(sb + j * 8192, &map_b, t.n0 + rank * kHalfN + 64 * j, at, t.group);
            } else {
              copy3(sb, &map_b, at, t.n0 + rank * kHalfN, t.group);
            }
          } else if constexpr (kRows == kRowsN) {
            if constexpr (kAMN) {
#pragma unroll
              for (int j = 0; j < kTileM / 64; ++j) copy3(sa + j * 8192, &map_a, t.m0 + 64 * j, at, t.group);
            } else {
              copy3(sa, &map_a, at, t.m0, t.group);
            }
            copy2(sb, &map_b, at, t.row0);
          } else {
#pragma unroll
            for (int j = 0; j < kTileM / 64; ++j) copy2(sa + j * 8192, &map_a, t.m0 + 64 * j, t.row0 + at);
#pragma unroll
            for (int j = 0; j < kHalfN / 64; ++j) copy2(sb + j * 8192, &map_b, t.n0 + rank * kHalfN + 64 * j, t.row0 + at);
          }
          stage = next;
          phase = next_phase;
        }
      }
      if constexpr (kPair)  // the other CTA's arrivals at this one's barriers are in
        for (int i = 0; ok && i < S::kStages; ++i) {
          ok = bar_wait(smem_u32(&empty_bar[stage]), phase ^ 1, &dead);
          if (++stage == S::kStages) stage = 0, phase ^= 1;
        }
      if (!ok) {  // no copy may be in flight when the CTA leaves: time enough for any
        const unsigned long long start = now_ns();
        while (now_ns() - start < kWaitLimitNs / 100) {
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = instr_desc(p.half, kAMN, kBMN, kPair ? 2 * kTileM : kTileM, BN);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      uint32_t cleared = 0;  // bit i: how often, modulo two, rows of stage i were cleared
      bool ok = true, ready = false;  // ready: the stage is known to be full
      Tile t;
      for (int64_t i = team; ok && tile_at<BN, kRows, kPair>(p, first, i, rank, &t); i += teams) {
        if (t.steps == 0) continue;
        ok = bar_wait<kPair>(smem_u32(&acc_empty[acc]), acc_phase ^ 1, &dead);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool swapped = tail_first<kRows>(t);
        if (swapped) ready = false;  // the stage that was asked for is the last one's
        for (int turn = 0; ok && turn < t.steps; ++turn) {
          const int next = stage + 1 == S::kStages ? 0 : stage + 1;
          const uint32_t next_phase = next == 0 ? phase ^ 1 : phase;
          const auto shifted = [&](int from, uint32_t from_phase, int by, uint32_t* its_phase) {
            const int at = from + by;
            *its_phase = at >= S::kStages || at < 0 ? from_phase ^ 1 : from_phase;
            return at >= S::kStages ? at - S::kStages : at < 0 ? at + S::kStages : at;
          };
          uint32_t use_phase, ask_phase;
          const int use = shifted(stage, phase, ring_shift(swapped, turn), &use_phase);
          const int ask = shifted(next, next_phase, turn + 1 < t.steps ? ring_shift(swapped, turn + 1) : 0, &ask_phase);
          const bool tail = swapped ? turn == kAhead : kRows == kRowsSum && t.rows - turn * kTileK < kTileK;
          const int rows = tail ? t.rows % kTileK : kTileK;  // in the stage
          const uint32_t sa = base + use * S::kStageBytes, sb = sa + kBytesA;
          if (kRows == kRowsSum && tail) {
            ok = bar_wait<kPair>(smem_u32(&clear_bar[use]), cleared >> use & 1, &dead);
            cleared ^= 1u << use;
          } else if (!ready) {
            ok = bar_wait(smem_u32(&full_bar[use]), use_phase, &dead);
          }
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          ready = bar_ask(smem_u32(&full_bar[ask]), ask_phase);
          const uint64_t da = smem_desc(sa, kAMN), db = smem_desc(sb, kBMN);
#pragma unroll
          for (int j = 0; j < kTileK / 16; ++j) {
            if (kRows == kRowsSum && 16 * j >= rows) break;
            const uint64_t a = da + j * (kAMN ? 2048 >> 4 : 32 >> 4), b = db + j * (kBMN ? 2048 >> 4 : 32 >> 4);
            if constexpr (kPair) mma_f16_pair(tmem + acc * BN, a, b, idesc, turn > 0 || j > 0);
            else mma_f16(tmem + acc * BN, a, b, idesc, turn > 0 || j > 0);
          }
          if constexpr (kPair) mma_commit_pair(smem_u32(&empty_bar[use]));
          else mma_commit(smem_u32(&empty_bar[use]));
          if (turn == t.steps - 1) {
            if constexpr (kPair) mma_commit_pair(smem_u32(&acc_full[acc]));
            else mma_commit(smem_u32(&acc_full[acc]));
          }
          stage = next;
          phase = next_phase;
        }
        if (++acc == 2) acc = 0, acc_phase ^= 1;
      }
      if (!ok) {  // nor may a product be under way
        if constexpr (kPair) mma_commit_pair(smem_u32(&last_bar));
        else mma_commit(smem_u32(&last_bar));
        bar_wait_short(smem_u32(&last_bar), 0);
      }
    }
  } else if (kRows == kRowsSum && warp == 6) {
    // clears the rows behind a group's last, up to the next multiple of 16, in the stage that holds them
    int64_t steps = 0;
    uint32_t cleared = 0;
    bool ok = true;
    Tile t;
    for (int64_t i = team; ok && tile_at<BN, kRows, kPair>(p, first, i, rank, &t); i += teams) {
      const int64_t at_stage = tail_first<kRows>(t) ? steps : steps + t.steps - 1;
      steps += t.steps;
      const int rows = t.rows - (t.steps - 1) * kTileK;
      if (t.steps == 0 || rows == kTileK) continue;
      const int stage = static_cast<int>(at_stage % S::kStages);
      ok = bar_wait_warp(smem_u32(&tail_bar[stage]), cleared >> stage & 1, &dead);
      if (!ok) break;
      const uint32_t at = base + stage * S::kStageBytes;
      for (int b = 0; b < S::kStageBytes / 8192; ++b)
        for (int c = rows * 8 + lane; c < ((rows + 15) & ~15) * 8; c += 32)
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + b * 8192 + c * 16), "r"(0) : "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (elect_one()) {
        if constexpr (kPair) bar_arrive_first(smem_u32(&clear_bar[stage]));
        else bar_arrive(smem_u32(&clear_bar[stage]));
      }
      cleared ^= 1u << stage;
    }
  } else {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    Tile t;
    uint16_t* const result = static_cast<uint16_t*>(p.out);
    int turns = 0;  // the piece that is next
    if constexpr (kRows != kRowsSum)  // rows behind the placed entries
      for (int64_t s = p.offsets[p.groups] + 4 * static_cast<int64_t>(blockIdx.x) + quarter; s < p.nnz; s += 4 * static_cast<int64_t>(gridDim.x))
        for (int c = lane; c < p.features; c += 32) result[s * p.ldo + c] = 0;
    for (int64_t i = team; ok && tile_at<BN, kRows, kPair>(p, first, i, rank, &t); i += teams) {
      if (t.steps > 0) {
        ok = bar_wait_warp(smem_u32(&acc_full[acc]), acc_phase, &dead);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t addr = tmem + acc * BN + (static_cast<uint32_t>(quarter * 32) << 16);
      if constexpr (kRows == kRowsN) {
        const int m = quarter * 32 + lane;
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
          const int left = t.rows - c;
          if (left <= 0) break;
          float f[16] = {};
          if (t.steps > 0) tmem_load16(addr + c, f);
          if (t.m0 + m < p.features) {
            uint16_t* dst = result + (static_cast<int64_t>(t.row0) + c) * p.ldo + t.m0 + m;
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < left) dst[j * p.ldo] = round16(f[j], p.half);
          }
        }
      } else {
        const uint32_t turn0 = base + S::kStages * S::kStageBytes + kPieces<kRows> * quarter * kTurnBytes;
        const int columns = kRows == kRowsM ? p.features : p.width;
        const int lines = (kRows == kRowsM ? t.rows : p.features - t.m0) - quarter * 32;  // rows of the warp that are stored
        const bool engine = p.vec == 16 && (kRows == kRowsSum || lines >= 32);
        uint16_t* const to = kRows == kRowsM ? result + (static_cast<int64_t>(t.row0) + quarter * 32) * p.ldo + t.n0
                                             : result + t.group * p.group_stride + (static_cast<int64_t>(t.m0) + quarter * 32) * p.ldo + t.n0;
#pragma unroll 1
        for (int c = 0; c < BN; c += 64) {
          const int left = columns - t.n0 - c;
          if (left <= 0 || lines <= 0) break;
          float f[64] = {};
          if (t.steps > 0) tmem_load64(addr + c, f);
          // the piece is free: at most the other one's store still reads
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kPieces<kRows> - 1) : "memory");
          __syncwarp();
          const uint32_t turn = turn0 + turns * kTurnBytes;
          if (++turns == kPieces<kRows>) turns = 0;
          put_rows(turn, p.half, f);
          if (engine) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if constexpr (kRows == kRowsSum) tma_store_3d(&map_out, turn, t.n0 + c, t.m0 + quarter * 32, t.group);
              else tma_store_2d(&map_out, turn, t.n0 + c, t.row0 + quarter * 32);
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          } else {
            store_turned(p, turn, to + c, left, [&](int row) { return row < lines; });
          }
        }
      }
      if (t.steps > 0) {
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) bar_arrive_first(smem_u32(&acc_empty[acc]));
          else bar_arrive(smem_u32(&acc_empty[acc]));
        }
        if (++acc == 2) acc = 0, acc_phase ^= 1;
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncwarp();
  __syncthreads();
  if constexpr (kPair) pair_sync();  // nothing of the other CTA's is on its way here
  if (threadIdx.x == 0 && dead) atomicOr(p.status, 1);
  if (warp == 1) tmem_free<S::kAccCols, kPair>(tmem);
}

// ---------------------------------------------------------------- few rows an expert, forward
//
// Bound by W, each met expert's once.  A CTA takes 32 features and up to eight rows of an expert; its eight warps split K and
// read W straight into the operands of the warp-level matrix instruction (16 features x 8 rows), 16 bytes a load, two steps
// in flight, three CTAs on an SM; the warps' sums meet in shared memory.  Six rows of four experts each of 64, N = 1024, K =
// 2048, bfloat16 (84 MB of W, 12.4 us at the copy rate): 18 us; in tiles of 128 features on the tcgen05 path 31 us
// (a fourth of the pieces of work); with four steps and two CTAs 18-19 us, two and four 22 us, three and three 25 us; with the
// loads as asynchronous copies to shared memory 29 us.

constexpr int kThinThreads = 256;
constexpr int kThinWarps = kThinThreads / 32;
constexpr int kThinRows = 8, kThinFeatures = 32;

template <bool half>
__global__ void __launch_bounds__(kThinThreads, 3)
    thin_kernel(const int64_t* offsets, int groups, int64_t nnz, const uint16_t* x, int64_t ldx,
                const uint16_t* W, int64_t ldw, int64_t group_stride, uint16_t* y, int64_t ldy,
                int N, int K) {
  __shared__ float red[kThinWarps][kThinFeatures][kThinRows + 1];
  __shared__ int scratch[32];
  __shared__ int found[3];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  if (threadIdx.x == 0) found[0] = -1;
  wait_for_last();
  const int64_t placed = offsets[groups];
  const int f0 = blockIdx.x * kThinFeatures;
  const auto zero_rest = [&] {  // rows behind the placed entries
    for (int64_t s = placed + static_cast<int64_t>(blockIdx.y) * kThinWarps + warp; s < nnz; s += static_cast<int64_t>(gridDim.y) * kThinWarps)
      if (f0 + lane < N) y[s * ldy + f0 + lane] = 0;
  };
  int sum = 0;
  const int want = blockIdx.y;
  for (int e0 = 0; e0 < groups && sum <= want; e0 += kThinThreads) {
    const int e = e0 + threadIdx.x;
    const int64_t b = e < groups ? offsets[e] : 0;
    const int rows = e < groups ? static_cast<int>(offsets[e + 1] - b) : 0;
    const int n = (rows + kThinRows - 1) / kThinRows;
    int all = 0;
    const int before = sum + block_exclusive_scan(n, scratch, &all);
    if (want >= before && want < before + n) {
      found[0] = e;
      found[1] = static_cast<int>(b) + (want - before) * kThinRows;
      found[2] = min(kThinRows, rows - (want - before) * kThinRows);
    }
    sum += all;
  }
  __syncthreads();
  const int e = found[0], row0 = found[1], rows = found[2];
  if (e < 0) {
    zero_rest();
    return;
  }
  const uint16_t* wrow[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) wrow[i] = W + e * group_stride + min(f0 + 8 * i + g, N - 1) * ldw;
  const uint16_t* xrow = x + (static_cast<int64_t>(row0) + min(g, rows - 1)) * ldx;
  float acc[2][4] = {};
  const auto step = [&](const uint4(&wv)[4], const uint4& xv) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      mma16<half>(acc[m], wv[2 * m].x, wv[2 * m + 1].x, wv[2 * m].y, wv[2 * m + 1].y, xv.x, xv.y);
      mma16<half>(acc[m], wv[2 * m].z, wv[2 * m + 1].z, wv[2 * m].w, wv[2 * m + 1].w, xv.z, xv.w);
    }
  };
  constexpr int kStep = 32 * kThinWarps, U = 2;  // U steps whose loads are in flight together
  int k = 32 * warp + 8 * q;
  for (; k - 8 * q + kStep * (U - 1) + 32 <= K; k += kStep * U) {
    uint4 wv[U][4], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) wv[u][i] = *reinterpret_cast<const uint4*>(wrow[i] + k + kStep * u);
      xv[u] = *reinterpret_cast<const uint4*>(xrow + k + kStep * u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) step(wv[u], xv[u]);
  }
#pragma unroll 1
  for (; k - 8 * q < K; k += kStep) {
    uint4 wv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) wv[i] = load8(wrow[i], k, K);
    step(wv, load8(xrow, k, K));
  }
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[warp][16 * m + 8 * (i >> 1) + g][2 * q + (i & 1)] = acc[m][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kThinFeatures * rows; i += kThinThreads) {
    const int f = i % kThinFeatures, row = i / kThinFeatures;
    if (f0 + f >= N) continue;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThinWarps; ++w) s += red[w][f][row];
    y[(static_cast<int64_t>(row0) + row) * ldy + f0 + f] = bits16<half>(s);
  }
  zero_rest();
}

cudaError_t launch_thin(const GroupedRows& g, cudaStream_t s) {
  const int64_t met = g.r->nnz < g.r->ncols ? g.r->nnz : g.r->ncols;
  const dim3 grid(static_cast<unsigned>((g.N + kThinFeatures - 1) / kThinFeatures),
                  static_cast<unsigned>(g.r->nnz / kThinRows + met));
  const auto kernel = g.half ? thin_kernel<true> : thin_kernel<false>;
  return launch_early(kernel, grid, kThinThreads, 0, s, 1, g.r->offsets, static_cast<int>(g.r->ncols), g.r->nnz,
                      static_cast<const uint16_t*>(g.x), g.ldx, static_cast<const uint16_t*>(g.w), g.ldw, g.group_stride, static_cast<uint16_t*>(g.out), g.ldo,
                      static_cast<int>(g.N), static_cast<int>(g.K));
}

// ---------------------------------------------------------------- host

template <int BN, int kRows, bool kWMN, bool kPair = false>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const GroupedParams& p, int64_t tiles, int num_sms,
                   cudaStream_t s) {
  using S = Shape<BN, kRows, kPair>;
  const auto kernel = grouped_kernel<BN, kRows, kWMN, kPair>;
  const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::kSmem));
  if (e != cudaSuccess) return e;
  const int64_t teams = kPair ? num_sms / 2 : num_sms;
  const unsigned grid = static_cast<unsigned>((tiles < teams ? tiles : teams) * (kPair ? 2 : 1));
  return launch_early(kernel, dim3(grid), kThreadsOf<kRows>, S::kSmem, s, kPair ? 2 : 1, a, b, out, p);
}

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

int row_alignment(uint64_t bits) { return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2; }

template <bool kWMN>
cudaError_t launch_rows(const GroupedRows& g, int num_sms, cudaStream_t s, bool* encoded) {
  const int64_t features = kWMN ? g.K : g.N, depth = kWMN ? g.N : g.K;
  GroupedParams p{};
  p.offsets = g.r->offsets;
  p.groups = static_cast<int>(g.r->ncols);
  p.nnz = g.r->nnz;
  p.features = static_cast<int>(features);
  p.depth = static_cast<int>(depth);
  p.out = g.out;
  p.ldo = g.ldo;
  p.half = g.half;
  p.vec = row_alignment(reinterpret_cast<uintptr_t>(g.out) | static_cast<uint64_t>(g.ldo * 2));
  p.status = g.r->status;
  CUtensorMap x, w, out{};
  if (p.vec == 16 && !encode(&out, g.out, g.half, features, g.r->nnz, g.ldo, 0, 0, 32)) p.vec = 8;
  const int64_t met = g.r->nnz < g.r->ncols ? g.r->nnz : g.r->ncols;  // groups that can have rows
  const double mean = static_cast<double>(g.r->nnz) / static_cast<double>(g.r->ncols);
  const auto run = [&](auto bn, auto side, auto pair) {
    constexpr int BN = decltype(bn)::value, kRows = decltype(side)::value;
    constexpr bool kPair = decltype(pair)::value;
    constexpr int kRowTile = kRowTileOf<BN, kRows>;
    constexpr int kFeat = kRows == kRowsM ? BN : kTileM;
    *encoded = encode(&x, g.x, g.half, depth, g.r->nnz, g.ldx, 0, 0, kRowTile) &&
               encode(&w, g.w, g.half, g.K, g.N, g.ldw, g.r->ncols, g.group_stride, kWMN ? 64 : kPair ? kFeat / 2 : kFeat);
    if (!*encoded) return cudaSuccess;
    const int64_t tiles = (g.r->nnz / (kPair ? 2 * kRowTile : kRowTile) + met) * up(features, kFeat);
    return launch<BN, kRows, kWMN, kPair>(kRows == kRowsM ? x : w, kRows == kRowsM ? w : x, out, p, tiles, num_sms, s);
  };
  using std::integral_constant;
  // Few rows an expert: W's features fill the 128 lanes and the rows are the short side.  us of the product and of the rows' gradient in
  // pieces of eight (product) or tiles of 16 rows | in tiles of 64, rows at random: 64 experts, K = 2048, N = 1024, mean 0.4 10.6, 10.5 |
  // 16.0, 14.7, mean 1 31.1, 30.7 | 34.6, 30.5, mean 4 43.0, 44.2 | 45.8, 42.8, mean 8 48.7, 44.3 | 46.6, 43.5, mean 12 59, 46 | 47, 44;
  // eight experts, N = 8192, mean 3 33.9, 35.0 | 41.8, 32.9, mean 8 48.1, 42.6 | 46.0, 41.2; 128 experts, K = 1024, N = 2048, mean 0.2
  // 12.2, 16.9 | 18.7, 20.2, mean 2 75.4, 71.4 | 71.3, 69.6, mean 12 142, 86 | 84, 82.
  // Forward: pieces of eight rows and 32 features also where they all are at work at once (24 rows of three experts, K = 1520, N =
  // 304: 14 us in tiles of 128 features, 8 us so).
  // The mean is over all columns: how many rows each has is known on the device only, so demand on few of many experts takes the
  // kernel of few rows.
  if constexpr (kWMN) {
    if (mean <= kFewRows) return run(integral_constant<int, 16>(), integral_constant<int, kRowsN>(), std::false_type());
  } else {
    if (mean <= kFewRows || (g.r->nnz / kThinRows + met) * up(features, kThinFeatures) <= 2 * num_sms) return launch_thin(g, s);
  }
  // Tiles of 64 rows | of 128, the rows on the lanes: 64 experts as above, mean 24 48, 45 | 49, 48, mean 48 49.5, 46.5 | 49.9, 49.2, mean
  // 64 50.2, 47.3 | 49.9, 48.5, mean 96 59, 61 | 52, 51; 16 experts, K = 4096, N = 2048, mean 24 45.4, 45.8 | 48.7, 44.9, mean 48 46.6,
  // 46.8 | 49.2, 45.9, mean 96 62, 56 | 50, 46.
  if (mean <= 48) return run(integral_constant<int, 64>(), integral_constant<int, kRowsN>(), std::false_type());
  // Pairs of row tiles where experts have enough of them that the odd one left over costs less than pairs gain.  2048 -> 4096, TFLOP/s
  // in pairs | one by one: 256 rows an expert 1060 | 1073, 512 1327 | 1277, 1024 1490 | 1364, 4096 1692 | 1536; with gradients 256
  // 634 | 679, 512 1029 | 1039, 1024 1318 | 1238, 4096 1615 | 1517.
  if (mean >= kPairRows && (g.r->nnz / (2 * kTileM) + up(met, 2)) * up(features, 256) >= num_sms / 2)
    return run(integral_constant<int, 256>(), integral_constant<int, kRowsM>(), std::true_type());
  // A tile of 128 features takes two thirds of the time of one of 256 (bound by its operands' way from L2), so the wider one is
  // taken unless the narrower fills the SMs' last turn so much better.
  const int64_t row_tiles = g.r->nnz / kTileM + up(met, 2);
  if (3 * up(row_tiles * up(features, 256), num_sms) <= 2 * up(row_tiles * up(features, 128), num_sms))
    return run(integral_constant<int, 256>(), integral_constant<int, kRowsM>(), std::false_type());
  return run(integral_constant<int, 128>(), integral_constant<int, kRowsM>(), std::false_type());
}

}  // namespace

ws_status_t launch_grouped(const GroupedRows& g, bool transposed, int num_sms, cudaStream_t s) {
  if (!encoder()) return routing_fail(WS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  bool encoded = true;
  const cudaError_t e = transposed ? launch_rows<true>(g, num_sms, s, &encoded) : launch_rows<false>(g, num_sms, s, &encoded);
  if (!encoded) return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "grouped product: %s", cudaGetErrorString(e));
}

ws_status_t launch_grouped_weights(const GroupedRows& g, const void* gys, int64_t ldgys, int num_sms, cudaStream_t s) {
  if (!encoder()) return routing_fail(WS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  GroupedParams p{};
  p.offsets = g.r->offsets;
  p.groups = static_cast<int>(g.r->ncols);
  p.nnz = g.r->nnz;
  p.features = static_cast<int>(g.N);
  p.width = static_cast<int>(g.K);
  p.out = g.out;
  p.ldo = g.ldo;
  p.group_stride = g.group_stride;
  p.half = g.half;
  p.vec = row_alignment(reinterpret_cast<uintptr_t>(g.out) | static_cast<uint64_t>(g.ldo * 2) | static_cast<uint64_t>(g.group_stride * 2));
  p.status = g.r->status;
  CUtensorMap a, b, out{};
  if (p.vec == 16 && !encode(&out, g.out, g.half, g.K, g.N, g.ldo, g.r->ncols, g.group_stride, 32)) p.vec = 8;
  if (!encode(&a, gys, g.half, g.N, g.r->nnz, ldgys, 0, 0, 64) || !encode(&b, g.x, g.half, g.K, g.r->nnz, g.ldx, 0, 0, 64))
    return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
  const int64_t wide = g.r->ncols * up(g.N, kTileM) * up(g.K, 256);
  const int64_t pairs = g.r->ncols * up(g.N, 2 * kTileM) * up(g.K, 256);
  const bool paired = static_cast<double>(g.r->nnz) >= kPairRows * static_cast<double>(g.r->ncols) && pairs >= num_sms / 2 &&
                      up(g.N, kTileM) % 2 == 0;
  const cudaError_t e = paired
                            ? launch<256, kRowsSum, false, true>(a, b, out, p, pairs, num_sms, s)
                        : wide >= num_sms
                            ? launch<256, kRowsSum, false>(a, b, out, p, wide, num_sms, s)
                            : launch<128, kRowsSum, false>(a, b, out, p, g.r->ncols * up(g.N, kTileM) * up(g.K, 128), num_sms, s);
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "grouped product: %s", cudaGetErrorString(e));
}

}  // namespace wsk
