// Kernels of the products by column of a routing matrix (grouped.cu: the products alone; fused.cu: with an epilogue, and
// sums of two products): every column (expert) e has a matrix
// W[e] (N x K) and, in slot order, the rows offsets[e] .. offsets[e + 1].
//   forward    ys[s]  = W[e] xs[s]                      contraction over K
//   rows       gxs[s] = W[e]^T gys[s]                   contraction over N
//   weights    gW[e]  = sum over s of gys[s] xs[s]^T    contraction over the rows of e
// bfloat16 or half operands, products and sums in 32 bits on the tensor cores
// (tcgen05, accumulators in tensor memory), one rounding when a result is stored.
//
// One persistent CTA per SM: one warp's lane fetches operand tiles with TMA
// (128-byte swizzle, a ring of stages), one lane issues the matrix
// instructions, four warps, or with an epilogue eight or twelve, finish and
// store tiles while the next one is multiplied (two accumulators).  How many rows an expert has is known on the
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
#pragma once

#include <type_traits>

#include "activation.cuh"
#include "routing.cuh"
#include "tensor.cuh"
#include "ws_internal.cuh"

namespace wsk {
namespace {

constexpr int kTileM = 128;   // rows of the M side: lanes of tensor memory
constexpr int kTileK = 64;    // 128 bytes: the swizzle's span
constexpr int kBytesA = kTileM * kTileK * 2;
constexpr int kTurnBytes = 32 * 128;
constexpr double kPairRows = 512;  // rows an expert from which on its row tiles go in pairs

// Where the rows of the experts are in the product D (M x N tile).
constexpr int kRowsM = 0;    // on the M side (lanes)
constexpr int kRowsN = 1;    // on the N side (columns): few rows per expert, W fills the lanes
constexpr int kRowsSum = 2;  // summed over

// What becomes of a product before it is stored.
constexpr int kPlain = 0;
constexpr int kLinear = 1;  // act(product + bias) + residual
constexpr int kGated = 2;   // act(product + bias) * (product with the second matrices + bias2)

struct Epilogue {
  int act;
  const uint16_t *bias, *bias2;  // groups x features, rows ldb values apart; NULL: none
  int64_t ldb, ldb2;
  const uint16_t* res;  // rows of the result's length, ldr values apart; NULL: none
  int64_t ldr;
  int res_vec;          // they start at multiples of so many bytes: 32, 16, 8, 4 or 2
  uint16_t *kept, *kept2;  // the sums before the activation, and the second matrices'; NULL: not wanted
  int64_t ldk, ldk2;
};

// kTwo: the contraction goes on over the second matrices.
template <int kEpi, bool kTwo>
struct Extra {
  CUtensorMap second, kept, kept2;
  Epilogue e;
  int apart;  // kRowsSum, kTwo: columns between the operands of the two results, of which the second is described by `second` and starts
  uint16_t* out;  // here, strides like the first's
  int vec_kept;   // as GroupedParams::vec, of the sums that are kept
};
template <>
struct Extra<kPlain, false> {};

struct GroupedParams {
  const int64_t* offsets;
  int groups;
  int64_t nnz;
  int features;  // kRowsM, kRowsN: columns of the result; kRowsSum: rows of gW[e] (M side)
  int width;     // kRowsSum: columns of gW[e] (N side)
  int steps;     // stages of the contraction; kRowsSum: unused
  void* out;
  int64_t ldo;   // values between rows of the result
  int64_t group_stride;  // kRowsSum: values between gW[e]
  bool half;
  int vec;       // rows of the result start at multiples of so many bytes: 32 (an epilogue's lanes store them), 16 (the copy engine may), 8, 4 or 2
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
  int part;      // kRowsSum, kTwo: of the two results
};

// Tiles of a CTA that one warp finds when the kernel begins, a lane each, for all roles to read: to find one takes about 2800 cycles (64-bit
// divisions, a search, loads of offsets), a fourth of what its epilogue may take.  Those behind them are found by every role when it
// comes to them.  32,768 rows of 32 experts, 1024 -> 2048: 92.8 -> 90.8 us.
constexpr int kListed = 32;

// A warp that copies, one that multiplies, four that store; where rows are summed over, one that clears.  Where a result is finished before it is
// stored that takes longer than the products, and is bound by no unit but by each warp's chain of loads, sums and stores, which more warps
// hide (32,768 rows of 32 experts, 1024 -> 2048, bias, gelu, sums kept, 125 us: tensor cores 55% of the cycles, issue slots 36%, DRAM 41%; the
// products alone 93): twelve warps 127 us, eight 139, when both were measured.  Sixteen need the room of a sixth stage, without which the
// products alone take 10% longer.  Gated blocks, twelve | eight: 44,272 rows of nine experts, 64 -> 1152, silu 51 | 61, gelu with kept sums
// 82 | 97; 8198 of eight, 512 -> 4096 55 | 57, 77 | 88, 2048 -> 4096, sums kept 185 | 183; 32,768 of 32, 1024 -> 2048, silu, sums kept
// 197 | 192 (the one that loses more than noise), gelu 199 | 206.
template <int BN, int kRows, bool kPair, int kEpi>
constexpr int kStorers = kRows != kRowsM || kEpi == kPlain ? 4 : kPair || BN <= 128 ? 12 : 8;
template <int BN, int kRows, bool kPair, int kEpi>
constexpr int kThreadsOf = kRows == kRowsSum ? 224 : 64 + 32 * kStorers<BN, kRows, kPair, kEpi>;

// Pieces of shared memory through which a storing warp's results go.
template <int kRows>
constexpr int kPieces = kRows == kRowsN ? 0 : kRows == kRowsM ? 1 : 2;

// Rows of a group in a tile, unless they are summed over.
template <int BN, int kRows>
constexpr int kRowTileOf = kRows == kRowsM ? kTileM : BN;

template <int BN, int kRows, bool kPair = false, int kEpi = kPlain>
struct Shape {
  static constexpr int kBytesB = (kPair ? BN / 2 : BN) * kTileK * 2;
  static constexpr int kStageBytes = kBytesA + kBytesB;
  static constexpr int kTurnSpace = kPieces<kRows> == 0 ? 0 : kRows == kRowsM && kEpi != kPlain ? kStorers<BN, kRows, kPair, kEpi> * (kTurnBytes / 2)
                                                                                                : 4 * kPieces<kRows> * kTurnBytes;
  static constexpr int kStages = (196 * 1024) / kStageBytes > 10 ? 10 : (196 * 1024) / kStageBytes;
  static constexpr int kAccCols = 2 * BN < 32 ? 32 : 2 * BN;  // a power of two
  static constexpr size_t kSmem = static_cast<size_t>(kStages) * kStageBytes + kTurnSpace + 1024;
};

// Tile t of the sequence that all roles of all CTAs share.  first[e]: row tiles of the groups before e.  kPair: t is two
// tiles one below the other, of which `rank` is the CTA's.
template <int BN, int kRows, int kEpi>
constexpr int kFeaturesOf = (kRows == kRowsM ? BN : kTileM) / (kEpi == kGated ? 2 : 1);

template <int BN, int kRows, bool kPair, int kEpi, bool kTwo>
__device__ __forceinline__ bool tile_at(const GroupedParams& p, const int* first, int64_t t, int rank, Tile* out) {
  constexpr int kSpan = kPair ? 2 * kTileM : kTileM;
  if constexpr (kRows == kRowsSum) {
    const int mt = (p.features + kSpan - 1) / kSpan, nt = (p.width + BN - 1) / BN;
    const int64_t each = static_cast<int64_t>(mt) * nt;
    constexpr int kParts = kTwo ? 2 : 1;
    if (t >= each * p.groups * kParts) return false;
    const int both = static_cast<int>(t / each);
    const int i = static_cast<int>(t - each * both), e = both / kParts;
    out->group = e;
    out->part = both % kParts;
    out->m0 = i % mt * kSpan + rank * kTileM;
    out->n0 = i / mt * BN;
    const int64_t b = p.offsets[e], n = p.offsets[e + 1] - b;
    out->row0 = static_cast<int>(b);
    out->rows = static_cast<int>(n);
    out->steps = static_cast<int>((n + kTileK - 1) / kTileK);
  } else {
    constexpr int kFeat = kFeaturesOf<BN, kRows, kEpi>;
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
    out->steps = p.steps;
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

// 32 columns: rounded to pairs, and put into rows of 64 bytes, whose pieces are placed by the second and third last bits of the row
// (64-byte swizzle).
__device__ __forceinline__ void pack32(const float (&f)[32], bool half, uint32_t (&w)[16]) {
  if (half) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = pair16<true>(f[2 * i], f[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = pair16<false>(f[2 * i], f[2 * i + 1]);
  }
}
__device__ __forceinline__ void put_rows32(uint32_t turn, const uint32_t (&w)[16]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(turn + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4)), "r"(w[4 * j]), "r"(w[4 * j + 1]),
                 "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                 : "memory");
}

// Stores what put_rows left (from column 0 of dst on, `left` columns of them inside the result); on(row): the row is stored.
template <typename On>
__device__ __forceinline__ void store_turned(int vec, uint32_t turn, uint16_t* dst, int64_t ld, int left, On on) {
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
        uint16_t* to = dst + row * ld + col;
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
  if (vec == 16) along(std::integral_constant<int, 16>());
  else if (vec == 8) along(std::integral_constant<int, 8>());
  else if (vec == 4) along(std::integral_constant<int, 4>());
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

// A 16-bit value of a type that is known when the kernel runs.
__device__ __forceinline__ float any16(uint16_t u, bool half) { return half ? value16<true>(u) : value16<false>(u); }

// Adds 32 columns' biases, in shared memory.
__device__ __forceinline__ void add32(float (&f)[32], const float* add) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const float4 b = *reinterpret_cast<const float4*>(add + i);
    split(add2(two(f[i], f[i + 1]), two(b.x, b.y)), &f[i], &f[i + 1]);
    split(add2(two(f[i + 2], f[i + 3]), two(b.z, b.w)), &f[i + 2], &f[i + 3]);
  }
}

// Adds 32 16-bit values.
__device__ __forceinline__ void add_row(float (&f)[32], const uint4 (&w)[4], bool half) {
  const auto add = [&](auto type) {
    constexpr bool kHalf = decltype(type)::value;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t v[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[8 * j + 2 * i] += value16<kHalf>(static_cast<uint16_t>(v[i] & 0xffff));
        f[8 * j + 2 * i + 1] += value16<kHalf>(static_cast<uint16_t>(v[i] >> 16));
      }
    }
  };
  if (half) add(std::true_type());
  else add(std::false_type());
}

// A lane's row of 32 columns, 32 bytes at a time (the address is a multiple of that): of what an epilogue stores no piece of shared memory is
// waited for, and no fence waits.  us, so | by the copy engine, with eight storing warps: 15,190 rows of 14 experts, 48 -> 3792, gated, sums
// kept 117 | 143 (84 with twelve, so), linear, gelu, sums kept 88 | 104; 32,768 rows of 32 experts, 1024 -> 2048, linear, gelu, sums kept
// 133 | 137.  By the engine where there is a residual, whose loads such stores hold up (32,768 rows as above 128 | 121, 40,000 of eight,
// 64 -> 4096, 199 | 189), and where products of pairs of gated tiles have more than kDirectSteps stages (8191 rows, 4096 -> 4096, sums kept:
// 303 | 298; of 16 stages 219 | 217).
constexpr int kDirectSteps = 8;
__device__ __forceinline__ void store_row32(uint16_t* to, const uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 2 * i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]),
                 "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                 : "memory");
}

__device__ __forceinline__ void load_row32(const uint16_t* from, uint4 (&w)[4]) {
#pragma unroll
  for (int j = 0; j < 4; j += 2)
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[j].x), "=r"(w[j].y), "=r"(w[j].z), "=r"(w[j].w), "=r"(w[j + 1].x), "=r"(w[j + 1].y), "=r"(w[j + 1].z), "=r"(w[j + 1].w)
                 : "l"(from + 8 * j));
}

// Stores the first `lines` rows of what put_rows32 left, from dst on, `left` columns of them, B bytes a lane: a batch is read before it is stored.
template <int B>
__device__ __forceinline__ void store_rows32(uint32_t turn, uint16_t* dst, int64_t ld, int lines, int left) {
  constexpr int kValues = B / 2, kLanes = 32 / kValues, kAtOnce = kValues;  // lanes a row, rows at once
  constexpr int kBatch = 32 / kAtOnce < 16 ? 32 / kAtOnce : 16;
  const int lane = threadIdx.x & 31, col = kValues * (lane % kLanes);
#pragma unroll
  for (int i0 = 0; i0 < 32 / kAtOnce; i0 += kBatch) {
    Pack<uint16_t, kValues> v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int row = (i0 + i) * kAtOnce + lane / kLanes;
      const uint32_t at = turn + row * 64 + (((col >> 3) ^ (row >> 1 & 3)) << 4) + 2 * (col & 7);
      uint32_t* w = reinterpret_cast<uint32_t*>(&v[i]);
      if constexpr (B == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
      else if constexpr (B == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
      else if constexpr (B == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
      else asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[i].v[0]) : "r"(at) : "memory");
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int row = (i0 + i) * kAtOnce + lane / kLanes;
      if (row >= lines) continue;
      uint16_t* to = dst + row * ld + col;
      if (col + kValues <= left) {
        *reinterpret_cast<Pack<uint16_t, kValues>*>(to) = v[i];
      } else {
#pragma unroll
        for (int e = 0; e < kValues; ++e)
          if (col + e < left) to[e] = v[i].v[e];
      }
    }
  }
  __syncwarp();
}

// Rows that do not start at multiples of 16 bytes, read along rows, `bytes` (8, 4 or 2) a lane, into a piece as put_rows32 lays it out: `lines` of
// them, `left` values each.  15,398 rows of five experts, 48 -> 4722, sigmoid, residual (rows at multiples of 4 bytes): 193 us,
// 2 bytes at a time 288.
template <int B>
__device__ __forceinline__ void take_rows32(uint32_t turn, const uint16_t* from, int64_t ld, int lines, int left) {
  constexpr int kValues = B / 2, kLanes = 32 / kValues, kAtOnce = kValues;  // lanes a row, rows at once
  using Value = std::conditional_t<B == 8, uint2, std::conditional_t<B == 4, uint32_t, uint16_t>>;
  const int lane = threadIdx.x & 31, col = kValues * (lane % kLanes);
  constexpr int kBatch = 32 / kAtOnce < 16 ? 32 / kAtOnce : 16;
#pragma unroll
  for (int i0 = 0; i0 < 32 / kAtOnce; i0 += kBatch) {
    Value v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int row = (i0 + i) * kAtOnce + lane / kLanes;
      v[i] = Value();
      if (row >= lines) continue;
      const uint16_t* src = from + row * ld + col;
      if (col + kValues <= left) {
        v[i] = *reinterpret_cast<const Value*>(src);
      } else {
        uint16_t some[kValues] = {};
#pragma unroll
        for (int e = 0; e < kValues; ++e)
          if (col + e < left) some[e] = src[e];
        if constexpr (B == 8) v[i] = make_uint2(some[0] | static_cast<uint32_t>(some[1]) << 16, some[2] | static_cast<uint32_t>(some[3]) << 16);
        else if constexpr (B == 4) v[i] = some[0] | static_cast<uint32_t>(some[1]) << 16;
        else v[i] = some[0];
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int row = (i0 + i) * kAtOnce + lane / kLanes;
      const uint32_t at = turn + row * 64 + (((col >> 3) ^ (row >> 1 & 3)) << 4) + 2 * (col & 7);
      if constexpr (B == 8) asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(v[i].x), "r"(v[i].y) : "memory");
      else if constexpr (B == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v[i]) : "memory");
      else asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(v[i]) : "memory");
    }
  }
  __syncwarp();
}
// A lane's row of a piece.
__device__ __forceinline__ void own_row32(uint32_t turn, uint4 (&w)[4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[j].x), "=r"(w[j].y), "=r"(w[j].z), "=r"(w[j].w)
                 : "r"(turn + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4))
                 : "memory");
}

// a: the M side's operand (kRowsM: the experts' rows, kRowsN: W, kRowsSum: gys), b: the N side's.
// kWMN: W's contraction index runs along its rows (MN-major).
// kPair: two CTAs, whose tiles lie one below the other, multiply as one (256 x 256): each holds its 128 rows of the M side and half of
// the N side, so that a stage takes 32 KB of shared memory and of the way from L2 instead of 48, and six stages fit where four did.
// Rank 0 issues the products and counts both CTAs' bytes at its barriers (rank 1 counting its own and telling rank 0 cost a microsecond a
// stage).  8198 rows of eight experts, 2048 -> 8192: 169 us, 1630 TFLOP/s (about 200 us in a loop, at the power limit); 32768 rows of 32
// experts, 2048 x 2048: 167 us, 167 us for the rows' gradient and 179 us for the matrices' (about 620 us in a loop).  Before the steps
// that followed, the loops took 206 and 653 us with pairs, 214 and 665 us without.
// kGated: a tile's features are half as many, each with a place in both matrices' products.  On the N side the second matrices' are behind the
// first's (in a pair the CTA of rank 1 fetches the second), so that a lane finds both in its row of tensor memory; on the M side they take
// turns of 16 lanes, so that a warp has both and lanes 16 apart exchange them.
// kTwo: stages in the first half of the contraction take W, the others the second matrices; the rows' second half follows their first, padded
// to whole stages.  In `weights` there are two results instead, of operands side by side in a row.
template <int BN, int kRows, bool kWMN, bool kPair, int kEpi, bool kTwo>
__global__ void __launch_bounds__(kThreadsOf<BN, kRows, kPair, kEpi>, 1)
    grouped_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_out, const GroupedParams p,
                   const __grid_constant__ Extra<kEpi, kTwo> x) {
  using S = Shape<BN, kRows, kPair, kEpi>;
  constexpr bool kAMN = kRows == kRowsSum || (kRows == kRowsN && kWMN);
  constexpr bool kBMN = kRows == kRowsSum || (kRows == kRowsM && kWMN);
  constexpr int kHalfN = kPair ? BN / 2 : BN;  // of the N side in this CTA
  extern __shared__ uint8_t raw[];
  __shared__ int first[kRouteMaxCols + 1];
  __shared__ int scratch[32];
  __shared__ __align__(8) uint64_t full_bar[S::kStages], empty_bar[S::kStages], acc_full[2], acc_empty[2], last_bar;
  // stages with rows behind a group's last: have come, and are cleared
  __shared__ __align__(8) uint64_t tail_bar[kRows == kRowsSum ? S::kStages : 1], clear_bar[kRows == kRowsSum ? S::kStages : 1];
  __shared__ __align__(16) float biases[kRows == kRowsM && kEpi != kPlain ? kStorers<BN, kRows, kPair, kEpi> : 1][kEpi == kGated ? 64 : 32];
  __shared__ Tile listed[kListed];
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
      bar_init(smem_u32(&acc_empty[i]), (kPair ? 2 : 1) * kStorers<BN, kRows, kPair, kEpi>);
    }
    bar_init(smem_u32(&last_bar), 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<S::kAccCols, kPair>(smem_u32(&tmem_slot));
  wait_for_last();
  if constexpr (kRows != kRowsSum) {  // row tiles before every group
    int sum = 0;
    for (int e0 = 0; e0 < p.groups; e0 += kThreadsOf<BN, kRows, kPair, kEpi>) {
      const int e = e0 + threadIdx.x;
      constexpr int kRowTile = kPair ? 2 * kTileM : kRowTileOf<BN, kRows>;
      const int n = e < p.groups ? static_cast<int>((p.offsets[e + 1] - p.offsets[e] + kRowTile - 1) / kRowTile) : 0;
      int all = 0;
      const int before = block_exclusive_scan(n, scratch, &all);
      if (e < p.groups) first[e] = sum + before;
      sum += all;
    }
    if (threadIdx.x == 0) first[p.groups] = sum;
    __syncthreads();
  }
  if (threadIdx.x < kListed) {
    Tile t;
    if (!tile_at<BN, kRows, kPair, kEpi, kTwo>(p, first, team + threadIdx.x * teams, rank, &t)) t.steps = -1;
    listed[threadIdx.x] = t;
  }
  const auto tile_of = [&](int i, Tile* t) {
    if (i >= kListed) return tile_at<BN, kRows, kPair, kEpi, kTwo>(p, first, team + i * teams, rank, t);
    *t = listed[i];
    return t->steps >= 0;
  };
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
      for (int i = 0; ok && tile_of(i, &t); ++i) {
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
              const CUtensorMap* map = &map_b;
              int row = at;
              if constexpr (kTwo)
                if (turn >= p.steps / 2) map = &x.second, row -= p.steps / 2 * kTileK;
#pragma unroll
              for (int j = 0; j < kHalfN / 64; ++j) copy3(sb + j * 8192, map, t.n0 + rank * kHalfN + 64 * j, row, t.group);
            } else if constexpr (kEpi == kGated) {
              if constexpr (kPair) {
                if (rank == 0) copy3(sb, &map_b, at, t.n0, t.group);
                else copy3(sb, &x.second, at, t.n0, t.group);
              } else {
                copy3(sb, &map_b, at, t.n0, t.group);
                copy3(sb + S::kBytesB / 2, &x.second, at, t.n0, t.group);
              }
            } else {
              copy3(sb, &map_b, at, t.n0 + rank * kHalfN, t.group);
            }
          } else if constexpr (kRows == kRowsN) {
            if constexpr (kAMN) {
              const CUtensorMap* map = &map_a;
              int row = at;
              if constexpr (kTwo)
                if (turn >= p.steps / 2) map = &x.second, row -= p.steps / 2 * kTileK;
#pragma unroll
              for (int j = 0; j < kTileM / 64; ++j) copy3(sa + j * 8192, map, t.m0 + 64 * j, row, t.group);
            } else if constexpr (kEpi == kGated) {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if (j & 1) copy3(sa + j * 2048, &x.second, at, t.m0 + 8 * (j - 1), t.group);
                else copy3(sa + j * 2048, &map_a, at, t.m0 + 8 * j, t.group);
              }
            } else {
              copy3(sa, &map_a, at, t.m0, t.group);
            }
            copy2(sb, &map_b, at, t.row0);
          } else {
#pragma unroll
            for (int j = 0; j < kTileM / 64; ++j) {
              int col = t.m0 + 64 * j;
              if constexpr (kTwo) col += t.part * x.apart;
              copy2(sa + j * 8192, &map_a, col, t.row0 + at);
            }
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
      for (int i = 0; ok && tile_of(i, &t); ++i) {
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
    for (int i = 0; ok && tile_of(i, &t); ++i) {
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
        for (int c = lane; c < p.features; c += 32) {
          result[s * p.ldo + c] = 0;
          if constexpr (kEpi != kPlain) {
            if (x.e.kept) x.e.kept[s * x.e.ldk + c] = 0;
            if (x.e.kept2) x.e.kept2[s * x.e.ldk2 + c] = 0;
          }
        }
    // Warps of a quarter take its columns by turns, 32 at a time, and go on from tile to tile where they stopped: with eight turns for three
    // warps, so that none has three of each tile's (32,768 rows of 32 experts, 1024 -> 2048, gelu, sums kept: 131 -> 127 us, with a
    // residual 121 -> 115; 40,000 of eight, 64 -> 4096, residual: 190 -> 168).
    constexpr int kSides = kStorers<BN, kRows, kPair, kEpi> / 4, kTurns = kFeaturesOf<BN, kRows, kEpi> / 32;
    int side = (warp - 2) >> 2;
    for (int i = 0; ok && tile_of(i, &t); ++i) {
      // what the epilogue of the next 32 columns reads, asked for while those before it, or the products, are under way
      struct Ahead {
        uint16_t bias, bias2;  // as they are stored: what converts them would wait for them
        uint4 res[kEpi == kLinear ? 4 : 1];
      } ahead{};
      const uint32_t pieces0 = base + S::kStages * S::kStageBytes + (warp - 2) * (kTurnBytes / 2);
      const auto look_ahead = [&](int c) {
        if constexpr (kRows == kRowsM && kEpi != kPlain) {
          const int left = p.features - t.n0 - c, col = t.n0 + c, line = quarter * 32 + lane;
          if (c >= kFeaturesOf<BN, kRows, kEpi> || left <= 0) return;
          if (x.e.bias && lane < left) ahead.bias = x.e.bias[t.group * x.e.ldb + col + lane];
          if constexpr (kEpi == kGated)
            if (x.e.bias2 && lane < left) ahead.bias2 = x.e.bias2[t.group * x.e.ldb2 + col + lane];
          if constexpr (kEpi == kLinear)
            if (x.e.res && x.e.res_vec >= 16) {
              const uint16_t* row = x.e.res + (static_cast<int64_t>(t.row0) + line) * x.e.ldr + col;
              if (x.e.res_vec == 32 && left >= 32) {
                if (line < t.rows) load_row32(row, ahead.res);
                return;
              }
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (line < t.rows) ahead.res[j] = load8(row, 8 * j, left);
            } else if (x.e.res && t.rows > quarter * 32) {  // through the piece
              if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
              __syncwarp();
              const uint16_t* from = x.e.res + (static_cast<int64_t>(t.row0) + quarter * 32) * x.e.ldr + col;
              if (x.e.res_vec == 8) take_rows32<8>(pieces0, from, x.e.ldr, t.rows - quarter * 32, left);
              else if (x.e.res_vec == 4) take_rows32<4>(pieces0, from, x.e.ldr, t.rows - quarter * 32, left);
              else take_rows32<2>(pieces0, from, x.e.ldr, t.rows - quarter * 32, left);
              own_row32(pieces0, ahead.res);
              __syncwarp();
            }
        }
      };
      look_ahead(32 * side);
      if (t.steps > 0) {
        ok = bar_wait_warp(smem_u32(&acc_full[acc]), acc_phase, &dead);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t addr = tmem + acc * BN + (static_cast<uint32_t>(quarter * 32) << 16);
      // The accumulators are free for the tile after the next as soon as the warp has read its last of them, and a pair's first CTA is told
      // without waiting for what the warp has stored (that wait was most of the time of short products): 40,000 rows of eight
      // experts, 64 -> 4096: 102 -> 76 us, 32,768 of 32, 1024 -> 2048, gelu, sums kept 131 -> 127, gated, sums kept 211 -> 198.  Where rows are
      // summed, only when all is stored: 64 experts' gradients of 1024 x 2048 from 25 rows each, with those of the rows, 112 us, else 120.
      bool held = t.steps > 0;
      const auto let_go = [&] {
        if (!held) return;
        held = false;
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) bar_tell_first(smem_u32(&acc_empty[acc]));
          else bar_arrive(smem_u32(&acc_empty[acc]));
        }
      };
      if constexpr (kRows == kRowsN && kEpi == kLinear) {
        const int m = t.m0 + quarter * 32 + lane;
        const bool on = m < p.features;
        float bias = 0.0f;
        if (x.e.bias && on) bias = p.half ? value16<true>(x.e.bias[t.group * x.e.ldb + m]) : value16<false>(x.e.bias[t.group * x.e.ldb + m]);
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
          const int left = t.rows - c;
          if (left <= 0) break;
          const int64_t row = static_cast<int64_t>(t.row0) + c;
          float add[16] = {};
          if (x.e.res && on) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < left) add[j] = p.half ? value16<true>(x.e.res[(row + j) * x.e.ldr + m]) : value16<false>(x.e.res[(row + j) * x.e.ldr + m]);
          }
          float f[16] = {};
          if (t.steps > 0) tmem_load16(addr + c, f);
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] += bias;
          if (x.e.kept && on) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < left) x.e.kept[(row + j) * x.e.ldk + m] = round16(f[j], p.half);
          }
          with_act(x.e.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 16; j += 2) act_values<decltype(act)::value>(&f[j], &f[j + 1]);
          });
          if (on) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < left) result[(row + j) * p.ldo + m] = round16(f[j] + add[j], p.half);
          }
          __syncwarp();
        }
      } else if constexpr (kRows == kRowsN && kEpi == kGated) {
        const int m = t.m0 + quarter * 16 + (lane & 15);
        const bool on = m < p.features, upper = lane >= 16;  // the lanes of the second matrices
        float bias = 0.0f;
        const uint16_t* from = upper ? x.e.bias2 : x.e.bias;
        if (from && on) {
          const uint16_t v = from[t.group * (upper ? x.e.ldb2 : x.e.ldb) + m];
          bias = p.half ? value16<true>(v) : value16<false>(v);
        }
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
          const int left = t.rows - c;
          if (left <= 0) break;
          const int64_t row = static_cast<int64_t>(t.row0) + c;
          float f[16] = {};
          if (t.steps > 0) tmem_load16(addr + c, f);
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] += bias;
          uint16_t* const kept = upper ? x.e.kept2 : x.e.kept;
          if (kept && on) {
            const int64_t ld = upper ? x.e.ldk2 : x.e.ldk;
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < left) kept[(row + j) * ld + m] = round16(f[j], p.half);
          }
          // lower lanes go on with even rows, upper ones with odd ones
          float gate[8], up[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float got = __shfl_xor_sync(0xffffffffu, upper ? f[2 * j] : f[2 * j + 1], 16);
            gate[j] = upper ? got : f[2 * j];
            up[j] = upper ? f[2 * j + 1] : got;
          }
          with_act(x.e.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) act_values<decltype(act)::value>(&gate[j], &gate[j + 1]);
#pragma unroll
            for (int j = 0; j < 8; ++j) up[j] *= gate[j];
          });
          if (on) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int r = 2 * j + upper;
              if (r < left) result[(row + r) * p.ldo + m] = round16(up[j], p.half);
            }
          }
          __syncwarp();
        }
      } else if constexpr (kRows == kRowsN) {
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
        uint16_t* start = result;
        const CUtensorMap* map_to = &map_out;
        if constexpr (kRows == kRowsSum && kTwo)
          if (t.part) start = x.out, map_to = &x.second;
        uint16_t* const to = kRows == kRowsM ? result + (static_cast<int64_t>(t.row0) + quarter * 32) * p.ldo + t.n0
                                             : start + t.group * p.group_stride + (static_cast<int64_t>(t.m0) + quarter * 32) * p.ldo + t.n0;
        if constexpr (kEpi != kPlain) {
          // 32 columns at a time, the warps of a quarter by turns, each through 2 KB of its own
          constexpr int kStep = 32 * kSides;
          const int64_t row0 = static_cast<int64_t>(t.row0) + quarter * 32;
          float* const add = biases[warp - 2];
#pragma unroll 1
          for (int c = 32 * side; c < kFeaturesOf<BN, kRows, kEpi>; c += kStep) {
            const int left = columns - t.n0 - c, col = t.n0 + c;
            if (left <= 0 || lines <= 0) break;
            const bool last = c + kStep >= kFeaturesOf<BN, kRows, kEpi> || left <= kStep;
            const auto pieces_free = [&] {  // what was stored from them has been read
              if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
              __syncwarp();
            };
            const auto store = [&](uint32_t piece, const CUtensorMap* map, uint16_t* dst, int64_t ld, int vec) {
              if (vec == 16 && lines >= 32) {
                if (lane == 0) tma_store_2d(map, piece, col, static_cast<int>(row0));
              } else {
                uint16_t* to = dst + row0 * ld + col;
                if (vec >= 16) store_rows32<16>(piece, to, ld, lines, left);
                else if (vec == 8) store_rows32<8>(piece, to, ld, lines, left);
                else if (vec == 4) store_rows32<4>(piece, to, ld, lines, left);
                else store_rows32<2>(piece, to, ld, lines, left);
              }
            };
            const auto emit = [&](const uint32_t(&v)[16], const CUtensorMap* map, uint16_t* dst, int64_t ld, int vec) {
              if (vec == 32 && left >= 32) {
                if (lane < lines) store_row32(dst + (row0 + lane) * ld + col, v);
                return;
              }
              pieces_free();
              put_rows32(pieces0, v);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              store(pieces0, map, dst, ld, vec);
              if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            };
            const bool first_bias = x.e.bias != nullptr, second_bias = kEpi == kGated && x.e.bias2;
            if (first_bias || second_bias) {
              __syncwarp();
              add[lane] = any16(ahead.bias, p.half);
              if constexpr (kEpi == kGated) add[32 + lane] = any16(ahead.bias2, p.half);
              __syncwarp();
            }
            float f[32] = {};
            uint32_t w[16];  // in pairs of 16-bit values
            if constexpr (kEpi == kGated) {
              float u[32] = {};
              if (t.steps > 0) tmem_load32(addr + c, addr + BN / 2 + c, f, u);
              if (last) let_go();
              if (first_bias) add32(f, add);
              if (second_bias) add32(u, add + 32);
              if (x.e.kept) {
                pack32(f, p.half, w);
                emit(w, &x.kept, x.e.kept, x.e.ldk, x.vec_kept);
              }
              if (x.e.kept2) {
                pack32(u, p.half, w);
                emit(w, &x.kept2, x.e.kept2, x.e.ldk2, x.vec_kept);
              }
              with_act(x.e.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                  act_values<decltype(act)::value>(&f[i], &f[i + 1]);
                  split(mul2(two(f[i], f[i + 1]), two(u[i], u[i + 1])), &f[i], &f[i + 1]);
                }
              });
            } else {
              if (t.steps > 0) tmem_load32(addr + c, f);
              if (last) let_go();
              if (first_bias) add32(f, add);
              if (x.e.kept) {
                pack32(f, p.half, w);
                emit(w, &x.kept, x.e.kept, x.e.ldk, x.vec_kept);
              }
              with_act(x.e.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 32; i += 2) act_values<decltype(act)::value>(&f[i], &f[i + 1]);
              });
              if (x.e.res) add_row(f, ahead.res, p.half);
            }
            pack32(f, p.half, w);
            emit(w, &map_out, result, p.ldo, p.vec);
            look_ahead(c + kStep);  // not before the fence, which would wait for it
          }
        } else {
#pragma unroll 1
        for (int c = 0; c < BN; c += 64) {
          const int left = columns - t.n0 - c;
          if (left <= 0 || lines <= 0) break;
          float f[64] = {};
          if (t.steps > 0) tmem_load64(addr + c, f);
          if (kRows == kRowsM && (c + 64 >= BN || left <= 64)) let_go();
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
              if constexpr (kRows == kRowsSum) tma_store_3d(map_to, turn, t.n0 + c, t.m0 + quarter * 32, t.group);
              else tma_store_2d(&map_out, turn, t.n0 + c, t.row0 + quarter * 32);
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          } else {
            store_turned(p.vec, turn, to + c, p.ldo, left, [&](int row) { return row < lines; });
          }
        }
        }
      }
      let_go();
      if constexpr (kEpi != kPlain) side = (side + kSides - kTurns % kSides) % kSides;
      if (t.steps > 0 && ++acc == 2) acc = 0, acc_phase ^= 1;
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
constexpr int kFewPieces = 6;

// kGated: 16 features, each in both matrices.  kAny: rows of x and W start at any multiple of 2 bytes and are read as they are, so that W is read
// once (a copy of it to aligned rows reads and writes it besides: 64 x 2048 x 1001 in both matrices for one row each, 262 MB each,
// 347 us with copies, 170 without; rows of 1000, which are aligned, 104).
template <int kEpi>
struct ThinExtra {
  const uint16_t* second;
  int64_t ld, group_stride;
  Epilogue e;
};
template <>
struct ThinExtra<kPlain> {};

template <bool half, int kEpi, int kWide = kThinFeatures, bool kAny = false>
__global__ void __launch_bounds__(kThinThreads, 3)
    thin_kernel(const int64_t* offsets, int groups, int64_t nnz, const uint16_t* x, int64_t ldx,
                const uint16_t* W, int64_t ldw, int64_t group_stride, uint16_t* y, int64_t ldy,
                int N, int K, const ThinExtra<kEpi> more) {
  constexpr int kFeatures = kEpi == kGated ? kWide / 2 : kWide, kTiles = kWide / 16;
  __shared__ float red[kThinWarps][kWide][kThinRows + 1];
  __shared__ int scratch[32];
  __shared__ int found[3];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  if (threadIdx.x == 0) found[0] = -1;
  wait_for_last();
  const int64_t placed = offsets[groups];
  const int f0 = blockIdx.x * kFeatures;
  const auto zero_rest = [&] {  // rows behind the placed entries
    for (int64_t s = placed + static_cast<int64_t>(blockIdx.y) * kThinWarps + warp; s < nnz; s += static_cast<int64_t>(gridDim.y) * kThinWarps)
      if (lane < kFeatures && f0 + lane < N) {
        y[s * ldy + f0 + lane] = 0;
        if constexpr (kEpi != kPlain) {
          if (more.e.kept) more.e.kept[s * more.e.ldk + f0 + lane] = 0;
          if (more.e.kept2) more.e.kept2[s * more.e.ldk2 + f0 + lane] = 0;
        }
      }
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
  const uint16_t* wrow[2 * kTiles];
#pragma unroll
  for (int i = 0; i < 2 * kTiles; ++i) {
    if constexpr (kEpi == kGated) {
      const int64_t f = min(f0 + 8 * (i % kTiles) + g, N - 1);
      wrow[i] = i < kTiles ? W + e * group_stride + f * ldw : more.second + e * more.group_stride + f * more.ld;
    } else {
      wrow[i] = W + e * group_stride + min(f0 + 8 * i + g, N - 1) * ldw;
    }
  }
  const uint16_t* xrow = x + (static_cast<int64_t>(row0) + min(g, rows - 1)) * ldx;
  float acc[kTiles][4] = {};
  const auto step = [&](const uint4(&wv)[2 * kTiles], const uint4& xv) {
#pragma unroll
    for (int m = 0; m < kTiles; ++m) {
      mma16<half>(acc[m], wv[2 * m].x, wv[2 * m + 1].x, wv[2 * m].y, wv[2 * m + 1].y, xv.x, xv.y);
      mma16<half>(acc[m], wv[2 * m].z, wv[2 * m + 1].z, wv[2 * m].w, wv[2 * m + 1].w, xv.z, xv.w);
    }
  };
  const auto eight = [](const uint16_t* from) {
    if constexpr (kAny) return load8_any(from, 8);
    else return *reinterpret_cast<const uint4*>(from);
  };
  constexpr int kStep = 32 * kThinWarps, U = 4 / kTiles;  // U steps whose loads are in flight together
  int k = 32 * warp + 8 * q;
  for (; k - 8 * q + kStep * (U - 1) + 32 <= K; k += kStep * U) {
    uint4 wv[U][2 * kTiles], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 2 * kTiles; ++i) wv[u][i] = eight(wrow[i] + k + kStep * u);
      xv[u] = eight(xrow + k + kStep * u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) step(wv[u], xv[u]);
  }
#pragma unroll 1
  for (; k - 8 * q < K; k += kStep) {
    const auto rest = [&](const uint16_t* row) {
      if constexpr (kAny) return k < K ? load8_any(row + k, K - k) : make_uint4(0, 0, 0, 0);
      else return load8(row, k, K);
    };
    uint4 wv[2 * kTiles];
#pragma unroll
    for (int i = 0; i < 2 * kTiles; ++i) wv[i] = rest(wrow[i]);
    step(wv, rest(xrow));
  }
#pragma unroll
  for (int m = 0; m < kTiles; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[warp][16 * m + 8 * (i >> 1) + g][2 * q + (i & 1)] = acc[m][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kFeatures * rows; i += kThinThreads) {
    const int f = i % kFeatures, row = i / kFeatures;
    if (f0 + f >= N) continue;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThinWarps; ++w) s += red[w][f][row];
    const int64_t at = static_cast<int64_t>(row0) + row;
    if constexpr (kEpi != kPlain) {
      if (more.e.bias) s += value16<half>(more.e.bias[e * more.e.ldb + f0 + f]);
      if (more.e.kept) more.e.kept[at * more.e.ldk + f0 + f] = bits16<half>(s);
      with_act(more.e.act, [&](auto act) { s = act_value<decltype(act)::value>(s); });
      if constexpr (kEpi == kGated) {
        float u = 0.0f;
#pragma unroll
        for (int w = 0; w < kThinWarps; ++w) u += red[w][kFeatures + f][row];
        if (more.e.bias2) u += value16<half>(more.e.bias2[e * more.e.ldb2 + f0 + f]);
        if (more.e.kept2) more.e.kept2[at * more.e.ldk2 + f0 + f] = bits16<half>(u);
        s *= u;
      } else if (more.e.res) {
        s += value16<half>(more.e.res[at * more.e.ldr + f0 + f]);
      }
    }
    y[at * ldy + f0 + f] = bits16<half>(s);
  }
  zero_rest();
}

template <int kEpi, int kWide = kThinFeatures, bool kAny = false>
cudaError_t launch_thin(const GroupedRows& g, const ThinExtra<kEpi>& more, cudaStream_t s) {
  constexpr int kFeatures = kEpi == kGated ? kWide / 2 : kWide;
  const int64_t met = g.r->nnz < g.r->ncols ? g.r->nnz : g.r->ncols;
  const dim3 grid(static_cast<unsigned>((g.N + kFeatures - 1) / kFeatures),
                  static_cast<unsigned>(g.r->nnz / kThinRows + met));
  const auto kernel = g.half ? thin_kernel<true, kEpi, kWide, kAny> : thin_kernel<false, kEpi, kWide, kAny>;
  return launch_early(kernel, grid, kThinThreads, 0, s, 1, g.r->offsets, static_cast<int>(g.r->ncols), g.r->nnz,
                      static_cast<const uint16_t*>(g.x), g.ldx, static_cast<const uint16_t*>(g.w), g.ldw, g.group_stride, static_cast<uint16_t*>(g.out), g.ldo,
                      static_cast<int>(g.N), static_cast<int>(g.K), more);
}

// ---------------------------------------------------------------- a few dozen rows, few tiles: the contraction in parts
//
// As the kernel above with W's features on the lanes and 64 rows on the N side, for products whose tiles are fewer than half of the SMs: a
// cluster of 2, 4 or 8 CTAs takes a tile, each a part of the contraction.  Every CTA finishes 64 / 2, 4 or 8 of the rows: it receives the
// others' sums of them in its shared memory and adds all in the order of the parts.  33 rows, 4096 -> 4096 (33.5 MB of W, 5 us at the
// copy rate), bias and residual: 12.3 us, on 32 CTAs 24

constexpr int kSplitRows = 64, kSplitThreads = 192;
constexpr int kSplitStage = kBytesA + kSplitRows * kTileK * 2;
constexpr int kSplitStages = 8;
constexpr int kSplitReceive = 7 * 8 * kTileM * 4;  // from 7 others 8 rows of 128 features; from 3 others 16, from one 32
constexpr size_t kSplitSmem = static_cast<size_t>(kSplitStages) * kSplitStage + kSplitReceive + 1024;

template <int kEpi, int kParts>
__global__ void __launch_bounds__(kSplitThreads, 1)
    split_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const GroupedParams p,
                 const __grid_constant__ Extra<kEpi, false> x) {
  constexpr int kMine = kSplitRows / kParts;  // rows that a CTA finishes
  static_assert((kParts - 1) * kMine * kTileM * 4 <= kSplitReceive, "");
  extern __shared__ uint8_t raw[];
  __shared__ int first[kRouteMaxCols + 1];
  __shared__ int scratch[32];
  __shared__ __align__(8) uint64_t full_bar[kSplitStages], empty_bar[kSplitStages], acc_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u, receive = base + kSplitStages * kSplitStage;
  const int rank = blockIdx.x % kParts;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSplitStages; ++i) {
      bar_init(smem_u32(&full_bar[i]), 1);
      bar_init(smem_u32(&empty_bar[i]), 1);
    }
    bar_init(smem_u32(&acc_bar), 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<kSplitRows>(smem_u32(&tmem_slot));
  wait_for_last();
  int sum = 0;
  for (int e0 = 0; e0 < p.groups; e0 += kSplitThreads) {
    const int e = e0 + threadIdx.x;
    const int n = e < p.groups ? static_cast<int>((p.offsets[e + 1] - p.offsets[e] + kSplitRows - 1) / kSplitRows) : 0;
    int all = 0;
    const int before = block_exclusive_scan(n, scratch, &all);
    if (e < p.groups) first[e] = sum + before;
    sum += all;
  }
  if (threadIdx.x == 0) first[p.groups] = sum;
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  pair_sync();  // all CTAs of the cluster are there
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  may_start_next();
  Tile t;
  const bool some = tile_at<kSplitRows, kRowsN, false, kEpi, false>(p, first, blockIdx.x / kParts, 0, &t);
  const int begin = some ? rank * p.steps / kParts : 0, end = some ? (rank + 1) * p.steps / kParts : 0;
  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      for (int k = begin; k < end; ++k) {
        const int i = k - begin, stage = i % kSplitStages;
        if (i >= kSplitStages && !bar_wait(smem_u32(&empty_bar[stage]), (i / kSplitStages - 1) & 1, &dead)) {
          ok = false;
          break;
        }
        const uint32_t sa = base + stage * kSplitStage, bar = smem_u32(&full_bar[stage]);
        bar_expect(bar, kSplitStage);
        if constexpr (kEpi == kGated) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (j & 1) tma_3d(sa + j * 2048, &x.second, k * kTileK, t.m0 + 8 * (j - 1), t.group, bar);
            else tma_3d(sa + j * 2048, &map_w, k * kTileK, t.m0 + 8 * j, t.group, bar);
          }
        } else {
          tma_3d(sa, &map_w, k * kTileK, t.m0, t.group, bar);
        }
        tma_2d(sa + kBytesA, &map_x, k * kTileK, t.row0, bar);
      }
      if (!ok) {  // no copy may be in flight when the CTA leaves: time enough for any
        const unsigned long long start = now_ns();
        while (now_ns() - start < kWaitLimitNs / 100) {
        }
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = instr_desc(p.half, false, false, kTileM, kSplitRows);
      for (int k = begin; k < end; ++k) {
        const int i = k - begin, stage = i % kSplitStages;
        if (!bar_wait(smem_u32(&full_bar[stage]), i / kSplitStages & 1, &dead)) {
          ok = false;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t a = smem_desc(base + stage * kSplitStage, false), b = smem_desc(base + stage * kSplitStage + kBytesA, false);
#pragma unroll
        for (int j = 0; j < kTileK / 16; ++j) mma_f16(tmem, a + j * (32 >> 4), b + j * (32 >> 4), idesc, i > 0 || j > 0);
        mma_commit(smem_u32(&empty_bar[stage]));
      }
      mma_commit(smem_u32(&acc_bar));  // also of what was begun before a wait was given up
      if (!ok) bar_wait_short(smem_u32(&acc_bar), 0);
    }
  }
  const int quarter = warp & 3;
  const uint32_t addr = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
  const uint32_t place = (quarter * 32 + lane) * 4;  // of a row's feature in what is received
  const auto part_of = [&](int from, int row) {      // from another CTA, one of this CTA's rows
    return receive + ((from < rank ? from : from - 1) * kMine + row) * kTileM * 4 + place;
  };
  // the features and rows that a lane finishes; what it adds is asked for before the products are waited for
  const bool upper = kEpi == kGated && lane >= 16;  // the lanes of the second matrices
  const int m = !some ? 0 : kEpi == kGated ? t.m0 + quarter * 16 + (lane & 15) : t.m0 + quarter * 32 + lane;
  const bool on = some && m < p.features;
  const int64_t row0 = some ? static_cast<int64_t>(t.row0) + rank * kMine : 0;
  const int mine = some ? min(t.rows - rank * kMine, kMine) : 0;
  uint16_t bias16 = 0, res16[kEpi == kLinear ? kMine : 1] = {};
  const uint16_t* const bias_from = upper ? x.e.bias2 : x.e.bias;
  if (warp >= 2 && on) {
    if (bias_from) bias16 = bias_from[t.group * (upper ? x.e.ldb2 : x.e.ldb) + m];
    if constexpr (kEpi == kLinear)
      if (x.e.res) {
#pragma unroll
        for (int j = 0; j < kMine; ++j)
          if (j < mine) res16[j] = x.e.res[(row0 + j) * x.e.ldr + m];
      }
  }
  if (warp >= 2) {
    if (end > begin) ok = bar_wait_warp(smem_u32(&acc_bar), 0, &dead);
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
    for (int to = 0; to < kParts; ++to) {
      if (to == rank) continue;
#pragma unroll
      for (int c = 0; c < kMine; c += 8) {
        if (!some || to * kMine + c >= t.rows) break;
        float f[8] = {};
        if (end > begin) tmem_load8(addr + to * kMine + c, f);
        const uint32_t at = receive + ((rank < to ? rank : rank - 1) * kMine + c) * kTileM * 4 + place;
#pragma unroll
        for (int j = 0; j < 8; ++j) store_in(at + j * kTileM * 4, to, f[j]);
      }
    }
  }
  __syncwarp();
  pair_sync();  // all sums have come
  if (warp >= 2 && some) {
    uint16_t* const result = static_cast<uint16_t*>(p.out);
    const float bias = any16(bias16, p.half);
    uint16_t* const kept = upper ? x.e.kept2 : x.e.kept;
    const int64_t ldk = upper ? x.e.ldk2 : x.e.ldk;
#pragma unroll
    for (int c = 0; c < kMine; c += 8) {
      const int left = mine - c;
      if (left <= 0) break;
      const int64_t row = row0 + c;
      float own[8] = {}, f[8] = {};
      if (end > begin) tmem_load8(addr + rank * kMine + c, own);
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = own[j];
          if (part != rank) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(part_of(part, c + j)) : "memory");
          f[j] += v;
        }
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += bias;
      if (kept && on) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left) kept[(row + j) * ldk + m] = round16(f[j], p.half);
      }
      if constexpr (kEpi == kGated) {  // lower lanes go on with even rows, upper ones with odd ones
        float gate[4], up[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float got = __shfl_xor_sync(0xffffffffu, upper ? f[2 * j] : f[2 * j + 1], 16);
          gate[j] = upper ? got : f[2 * j];
          up[j] = upper ? f[2 * j + 1] : got;
        }
        with_act(x.e.act, [&](auto act) {
#pragma unroll
          for (int j = 0; j < 4; j += 2) act_values<decltype(act)::value>(&gate[j], &gate[j + 1]);
        });
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (on && 2 * j + upper < left) result[(row + 2 * j + upper) * p.ldo + m] = round16(up[j] * gate[j], p.half);
      } else {
        with_act(x.e.act, [&](auto act) {
#pragma unroll
          for (int j = 0; j < 8; j += 2) act_values<decltype(act)::value>(&f[j], &f[j + 1]);
        });
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (on && j < left) result[(row + j) * p.ldo + m] = round16(f[j] + any16(res16[c + j], p.half), p.half);
      }
      __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  }
  if (warp >= 2) {  // rows behind the placed entries
    uint16_t* const result = static_cast<uint16_t*>(p.out);
    for (int64_t s = p.offsets[p.groups] + 4 * static_cast<int64_t>(blockIdx.x) + quarter; s < p.nnz; s += 4 * static_cast<int64_t>(gridDim.x))
      for (int c = lane; c < p.features; c += 32) {
        result[s * p.ldo + c] = 0;
        if (x.e.kept) x.e.kept[s * x.e.ldk + c] = 0;
        if (x.e.kept2) x.e.kept2[s * x.e.ldk2 + c] = 0;
      }
  }
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0 && dead) atomicOr(p.status, 1);
  if (warp == 1) tmem_free<kSplitRows>(tmem);
}

// ---------------------------------------------------------------- host

template <int BN, int kRows, bool kWMN, bool kPair = false, int kEpi = kPlain, bool kTwo = false>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const GroupedParams& p, int64_t tiles, int num_sms,
                   cudaStream_t s, const Extra<kEpi, kTwo>& x = {}) {
  using S = Shape<BN, kRows, kPair, kEpi>;
  const auto kernel = grouped_kernel<BN, kRows, kWMN, kPair, kEpi, kTwo>;
  static std::atomic<uint64_t> allowed{0};
  const int64_t teams = kPair ? num_sms / 2 : num_sms;
  const unsigned grid = static_cast<unsigned>((tiles < teams ? tiles : teams) * (kPair ? 2 : 1));
  return with_smem(reinterpret_cast<const void*>(kernel), S::kSmem, &allowed, [&] {
    return launch_early(kernel, dim3(grid), kThreadsOf<BN, kRows, kPair, kEpi>, S::kSmem, s, kPair ? 2 : 1, a, b, out, p, x);
  });
}

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

int row_alignment(uint64_t bits) { return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2; }

// What a product with an epilogue, or of two parts, has beyond one alone.
struct Fused {
  const void* second;  // the second matrices
  int64_t ld, stride;
  Epilogue e;
  bool any;  // few rows: rows start at any multiple of 2 bytes
};

// kWMN: the rows' gradient.
template <bool kWMN, int kEpi = kPlain, bool kTwo = false>
cudaError_t launch_rows(const GroupedRows& g, int num_sms, cudaStream_t s, bool* encoded, const Fused& fused = {}) {
  const int64_t features = kWMN ? g.K : g.N, depth = kWMN ? g.N : g.K;
  GroupedParams p{};
  p.offsets = g.r->offsets;
  p.groups = static_cast<int>(g.r->ncols);
  p.nnz = g.r->nnz;
  p.features = static_cast<int>(features);
  p.steps = static_cast<int>(up(depth, kTileK)) * (kTwo ? 2 : 1);
  p.out = g.out;
  p.ldo = g.ldo;
  p.half = g.half;
  const uint64_t bits = reinterpret_cast<uintptr_t>(g.out) | static_cast<uint64_t>(g.ldo * 2);
  Extra<kEpi, kTwo> extra{};
  if constexpr (kEpi != kPlain) {
    extra.e = fused.e;
    uint64_t kept = 0;
    if (fused.e.kept) kept |= reinterpret_cast<uintptr_t>(fused.e.kept) | static_cast<uint64_t>(fused.e.ldk * 2);
    if (fused.e.kept2) kept |= reinterpret_cast<uintptr_t>(fused.e.kept2) | static_cast<uint64_t>(fused.e.ldk2 * 2);
    extra.vec_kept = kept % 32 == 0 ? 32 : row_alignment(kept);
  }
  p.vec = kEpi != kPlain && bits % 32 == 0 ? 32 : row_alignment(bits);
  p.status = g.r->status;
  CUtensorMap x{}, w{}, out{};
  const int64_t wide = features * (kEpi == kGated ? 2 : 1);  // features counted as often as they are multiplied
  const int64_t met = g.r->nnz < g.r->ncols ? g.r->nnz : g.r->ncols;  // groups that can have rows
  const double mean = static_cast<double>(g.r->nnz) / static_cast<double>(g.r->ncols);
  const auto run = [&](auto bn, auto side, auto pair) {
    constexpr int BN = decltype(bn)::value, kRows = decltype(side)::value;
    constexpr bool kPair = decltype(pair)::value;
    constexpr int kRowTile = kRowTileOf<BN, kRows>;
    constexpr int kFeat = kFeaturesOf<BN, kRows, kEpi>;
    constexpr int kBox = kWMN ? 64 : kEpi == kGated ? (kRows == kRowsN ? 16 : kFeat) : kPair ? kFeat / 2 : kFeat;
    if constexpr (kEpi != kPlain) {
      if (fused.e.res || (kEpi == kGated && kPair && p.steps > kDirectSteps)) {
        if (p.vec == 32) p.vec = 16;
        if (extra.vec_kept == 32) extra.vec_kept = 16;
      }
    }
    if constexpr (kRows == kRowsM) {  // results that the copy engine stores
      if (p.vec == 16 && !encode(&out, g.out, g.half, features, g.r->nnz, g.ldo, 0, 0, 32, kEpi == kPlain ? 64 : 32)) p.vec = 8;
      if constexpr (kEpi != kPlain)
        if (extra.vec_kept == 16 &&
            ((fused.e.kept && !encode(&extra.kept, fused.e.kept, g.half, features, g.r->nnz, fused.e.ldk, 0, 0, 32, 32)) ||
             (fused.e.kept2 && !encode(&extra.kept2, fused.e.kept2, g.half, features, g.r->nnz, fused.e.ldk2, 0, 0, 32, 32))))
          extra.vec_kept = 8;
    }
    if (depth > 0) {  // else no stage is fetched
      *encoded = encode(&x, g.x, g.half, kTwo ? p.steps * kTileK : depth, g.r->nnz, g.ldx, 0, 0, kRowTile) &&
                 encode(&w, g.w, g.half, g.K, g.N, g.ldw, g.r->ncols, g.group_stride, kBox);
      if constexpr (kTwo || kEpi == kGated)
        *encoded = *encoded && encode(&extra.second, fused.second, g.half, g.K, g.N, fused.ld, g.r->ncols, fused.stride, kBox);
      if (!*encoded) return cudaSuccess;
    }
    const int64_t tiles = (g.r->nnz / (kPair ? 2 * kRowTile : kRowTile) + met) * up(features, kFeat);
    return launch<BN, kRows, kWMN, kPair, kEpi, kTwo>(kRows == kRowsM ? x : w, kRows == kRowsM ? w : x, out, p, tiles, num_sms, s, extra);
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
    if (few_rows(g.r->nnz, g.r->ncols, wide, num_sms)) {
      ThinExtra<kEpi> more{};
      if constexpr (kEpi != kPlain) more = {static_cast<const uint16_t*>(fused.second), fused.ld, fused.stride, fused.e};
      if constexpr (kEpi != kPlain)
        if (fused.any) return launch_thin<kEpi, kThinFeatures, true>(g, more, s);
      if constexpr (kEpi != kPlain)  // pieces half as wide where an SM has only a few, so that all SMs end together
        if ((g.r->nnz / kThinRows + met) * up(wide, kThinFeatures) <= kFewPieces * num_sms) return launch_thin<kEpi, kThinFeatures / 2>(g, more, s);
      return launch_thin<kEpi>(g, more, s);
    }
  }
  if constexpr (kEpi != kPlain) {
    // At least four stages for every part.  Rows of more than one tile read W as often, so up to 128 of them.
    const int64_t pieces = (g.r->nnz / kSplitRows + met) * up(features, kFeaturesOf<64, kRowsN, kEpi>);
    for (int parts = 8; parts >= 2; parts /= 2)
      if (mean <= 128 && pieces * parts <= num_sms && p.steps >= 4 * parts) {
        constexpr int kBox = kEpi == kGated ? 16 : kTileM;
        *encoded = encode(&x, g.x, g.half, depth, g.r->nnz, g.ldx, 0, 0, kSplitRows) &&
                   encode(&w, g.w, g.half, g.K, g.N, g.ldw, g.r->ncols, g.group_stride, kBox) &&
                   (kEpi != kGated || encode(&extra.second, fused.second, g.half, g.K, g.N, fused.ld, g.r->ncols, fused.stride, kBox));
        if (!*encoded) return cudaSuccess;
        const auto kernel = parts == 8 ? split_kernel<kEpi, 8> : parts == 4 ? split_kernel<kEpi, 4> : split_kernel<kEpi, 2>;
        static std::atomic<uint64_t> allowed[3]{};
        return with_smem(reinterpret_cast<const void*>(kernel), kSplitSmem, &allowed[parts >> 2], [&] {
          return launch_early(kernel, dim3(static_cast<unsigned>(pieces * parts)), kSplitThreads, kSplitSmem, s, parts, w, x, p, extra);
        });
      }
  }
  // Tiles of 64 rows | of 128, the rows on the lanes: 64 experts as above, mean 24 48, 45 | 49, 48, mean 48 49.5, 46.5 | 49.9, 49.2, mean
  // 64 50.2, 47.3 | 49.9, 48.5, mean 96 59, 61 | 52, 51; 16 experts, K = 4096, N = 2048, mean 24 45.4, 45.8 | 48.7, 44.9, mean 48 46.6,
  // 46.8 | 49.2, 45.9, mean 96 62, 56 | 50, 46.
  if (mean <= 48) return run(integral_constant<int, 64>(), integral_constant<int, kRowsN>(), std::false_type());
  // Pairs of row tiles where experts have enough of them that the odd one left over costs less than pairs gain.  2048 -> 4096, TFLOP/s
  // in pairs | one by one: 256 rows an expert 1060 | 1073, 512 1327 | 1277, 1024 1490 | 1364, 4096 1692 | 1536; with gradients 256
  // 634 | 679, 512 1029 | 1039, 1024 1318 | 1238, 4096 1615 | 1517.
  if (mean >= kPairRows && (g.r->nnz / (2 * kTileM) + up(met, 2)) * up(wide, 256) >= num_sms / 2)
    return run(integral_constant<int, 256>(), integral_constant<int, kRowsM>(), std::true_type());
  // A tile of 128 features takes two thirds of the time of one of 256 (bound by its operands' way from L2), so the wider one is
  // taken unless the narrower fills the SMs' last turn so much better.
  const int64_t row_tiles = g.r->nnz / kTileM + up(met, 2);
  if (3 * up(row_tiles * up(wide, 256), num_sms) <= 2 * up(row_tiles * up(wide, 128), num_sms))
    return run(integral_constant<int, 256>(), integral_constant<int, kRowsM>(), std::false_type());
  return run(integral_constant<int, 128>(), integral_constant<int, kRowsM>(), std::false_type());
}

}  // namespace
}  // namespace wsk
