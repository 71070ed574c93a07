// Products by column of a routing matrix with an epilogue, and their gradients (kernels of the products in grouped.cuh):
//   linear   ys[s] = act(W[e] xs[s] + b[e]) + residual[s]
//   gated    h[s]  = act(Wg[e] xs[s] + bg[e]) * (Wu[e] xs[s] + bu[e])
// Forward each is one kernel: the sums are finished where they leave tensor memory, in 32 bits, and rounded once.
//
// Backward the sums' gradients come first, gz = gys act'(z), or dg = gh up act'(gate) and du = gh act(gate) side by side, from the kept
// sums, and with them those of the biases; then the products' kernels take them as any other rows.  gxs = dg Wg + du Wu is one
// product whose contraction goes on over the second matrices, so that it is summed in 32 bits and rounded once.  The sums kept
// (z, gate, up) and their gradients are rounded to the 16 bits that the tensor cores read: to keep them in 32 would double
// what this step moves, and a product of them would still be one of 16-bit values.
#include "grouped.cuh"

namespace wsk {
namespace {

// ---------------------------------------------------------------- gradients of the sums

// Bound by memory.  A CTA takes a tile of rows of an expert and 256 columns, a warp a row at a time, a lane eight columns (16 bytes).
// Sums over rows for the biases stay in registers; the warps' meet in shared memory, the tiles' in a second kernel,
// both in a fixed order.
constexpr int kSlopeThreads = 256;
constexpr int kSlopePerSm = 8;  // CTAs launched
constexpr int kAtOnce = 2;  // rows that a warp has in flight

struct SlopeParams {
  const int64_t* offsets;
  int groups;
  int width, padded;          // columns; those of a row of `out` (16-byte rows; behind the width zeros)
  const uint16_t *g, *z, *up;
  int64_t ldg, ldz, ldup;
  bool vecg, vecz, vecup;     // rows start at multiples of 16 bytes
  uint16_t* out;              // rows of 1 or 2 x padded; NULL: sums only
  float* sums;                // tiles x (1 or 2) x padded
  int act;
  int tile;                   // rows
};

// Row tiles before every group, in shared memory; the same in both kernels.
__device__ __forceinline__ void count_tiles(const int64_t* offsets, int groups, int rows, int* first, int* scratch) {
  int sum = 0;
  for (int e0 = 0; e0 < groups; e0 += kSlopeThreads) {
    const int e = e0 + threadIdx.x;
    const int n = e < groups ? static_cast<int>((offsets[e + 1] - offsets[e] + rows - 1) / rows) : 0;
    int all = 0;
    const int before = block_exclusive_scan(n, scratch, &all);
    if (e < groups) first[e] = sum + before;
    sum += all;
  }
  if (threadIdx.x == 0) first[groups] = sum;
  __syncthreads();
}

template <bool half>
__device__ __forceinline__ void unpack8(const uint4& w, float (&f)[8]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = value16<half>(static_cast<uint16_t>(v[i] & 0xffff));
    f[2 * i + 1] = value16<half>(static_cast<uint16_t>(v[i] >> 16));
  }
}
template <bool half>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pair16<half>(f[0], f[1]), pair16<half>(f[2], f[3]), pair16<half>(f[4], f[5]), pair16<half>(f[6], f[7]));
}

template <bool half, bool kBoth, bool kSums>
__global__ void __launch_bounds__(kSlopeThreads, kBoth && kSums ? 3 : 0) slope_kernel(const SlopeParams p) {
  constexpr int kParts = kBoth ? 2 : 1, kWarps = kSlopeThreads / 32;
  __shared__ int first[kSums ? kRouteMaxCols + 1 : 1];
  __shared__ int scratch[32];
  __shared__ float red[kSums ? kParts * kWarps : 1][kSums ? kSlopeColumns : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = blockIdx.x * kSlopeColumns + 8 * lane;
  wait_for_last();
  int64_t tiles;
  const int64_t placed = p.offsets[p.groups];
  if constexpr (kSums) {
    count_tiles(p.offsets, p.groups, p.tile, first, scratch);
    tiles = first[p.groups];
  } else {
    tiles = (placed + p.tile - 1) / p.tile;
  }
  may_start_next();
  with_act(p.act, [&](auto act) {
  constexpr bool kSame = !kBoth && decltype(act)::value == WS_ACT_NONE;  // the sums' gradient is the result's
  for (int64_t tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
    int64_t row0 = tile * p.tile, rows = placed - row0;
    if constexpr (kSums) {
      int lo = 0, hi = p.groups - 1;  // the last group with first[e] <= tile
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= tile) lo = mid;
        else hi = mid - 1;
      }
      const int64_t before = (tile - first[lo]) * p.tile;
      row0 = p.offsets[lo] + before;
      rows = p.offsets[lo + 1] - row0;
    }
    if (rows > p.tile) rows = p.tile;
    [[maybe_unused]] float sum[kParts][8] = {};
    if (col < p.padded) {
      for (int r0 = warp; r0 < rows; r0 += kWarps * kAtOnce) {
        [[maybe_unused]] uint4 wg[kAtOnce], wz[kAtOnce], wu[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const int64_t row = row0 + min(static_cast<int64_t>(r0 + j * kWarps), rows - 1);
          wg[j] = load8(p.g + row * p.ldg, col, p.width, p.vecg);
          if constexpr (!kSame) wz[j] = load8(p.z + row * p.ldz, col, p.width, p.vecz);
          if constexpr (kBoth) wu[j] = load8(p.up + row * p.ldup, col, p.width, p.vecup);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          if (r0 + j * kWarps >= rows) break;
          const int64_t row = row0 + r0 + j * kWarps;
          [[maybe_unused]] float g[8], z[8], up[8], dz[8], du[8];
          unpack8<half>(wg[j], g);
          if constexpr (kBoth) unpack8<half>(wu[j], up);
          if constexpr (kSame) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dz[i] = g[i];
          } else {
            unpack8<half>(wz[j], z);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              float value[2];
              act_slopes<decltype(act)::value>(&z[i], &z[i + 1], &value[0], &value[1]);
              const Two gi = two(g[i], g[i + 1]);
              Two d = mul2(gi, two(z[i], z[i + 1]));
              if constexpr (kBoth) {
                d = mul2(d, two(up[i], up[i + 1]));
                split(mul2(gi, two(value[0], value[1])), &du[i], &du[i + 1]);
              }
              split(d, &dz[i], &dz[i + 1]);
            }
          }
          if (p.out) {
            uint16_t* to = p.out + row * kParts * p.padded + col;
            *reinterpret_cast<uint4*>(to) = pack8<half>(dz);
            if constexpr (kBoth) *reinterpret_cast<uint4*>(to + p.padded) = pack8<half>(du);
          }
          if constexpr (kSums) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              sum[0][i] += dz[i];
              if constexpr (kBoth) sum[kParts - 1][i] += du[i];
            }
          }
        }
      }
    }
    if constexpr (kSums) {
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int i = 0; i < 8; ++i) red[part * kWarps + warp][8 * lane + i] = sum[part][i];
      __syncthreads();
      const int c = blockIdx.x * kSlopeColumns + threadIdx.x;
      if (c < p.padded) {
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          float s = 0.0f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) s += red[part * kWarps + w][threadIdx.x];
          p.sums[(tile * kParts + part) * p.padded + c] = s;
        }
      }
      __syncthreads();
    }
  }
  });
}

// The biases' gradients from the tiles' sums: a CTA takes 32 columns of an expert, its warps every eighth tile.
struct BiasParams {
  const int64_t* offsets;
  int groups, width, padded, parts, tile;
  const float* sums;
  uint16_t* out[2];
  int64_t ld[2];
};

template <bool half>
__global__ void __launch_bounds__(kSlopeThreads) bias_kernel(const BiasParams p) {
  constexpr int kWarps = kSlopeThreads / 32;
  __shared__ int first[kRouteMaxCols + 1];
  __shared__ int scratch[32];
  __shared__ float red[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.y, part = blockIdx.z;
  const int col = blockIdx.x * 32 + lane;
  wait_for_last();
  count_tiles(p.offsets, p.groups, p.tile, first, scratch);
  may_start_next();
  float s = 0.0f;
  if (col < p.width)
#pragma unroll 4
    for (int tile = first[e] + warp; tile < first[e + 1]; tile += kWarps) s += p.sums[(static_cast<int64_t>(tile) * p.parts + part) * p.padded + col];
  red[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || col >= p.width || !p.out[part]) return;
  s = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += red[w][lane];
  p.out[part][e * p.ld[part] + col] = bits16<half>(s);
}

template <bool kBoth, bool kSums>
cudaError_t launch_slope(const SlopeParams& p, bool half, int64_t tiles, int num_sms, cudaStream_t s) {
  const int64_t wide = up(p.padded, kSlopeColumns), most = up(static_cast<int64_t>(kSlopePerSm) * num_sms, wide);
  const dim3 grid(static_cast<unsigned>(wide), static_cast<unsigned>(tiles < most ? tiles : most));
  return launch_early(half ? slope_kernel<true, kBoth, kSums> : slope_kernel<false, kBoth, kSums>, grid, kSlopeThreads, 0, s, 1, p);
}

bool rows16(const void* p, int64_t ld, int64_t rows) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld % 8 == 0); }

}  // namespace

ws_status_t launch_fused(const GroupedRows& g, const FusedRows& f, int num_sms, cudaStream_t s) {
  if (!encoder()) return routing_fail(WS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  Fused x{f.second, f.ld2, f.stride2, {}, f.any};
  const auto half16 = [](const void* p) { return static_cast<const uint16_t*>(p); };
  x.e.act = f.act;
  x.e.bias = half16(f.bias), x.e.ldb = f.ldb;
  x.e.bias2 = half16(f.bias2), x.e.ldb2 = f.ldb2;
  const uint64_t res = reinterpret_cast<uintptr_t>(f.res) | (g.r->nnz > 1 ? static_cast<uint64_t>(f.ldr * 2) : 0);
  x.e.res = half16(f.res), x.e.ldr = f.ldr, x.e.res_vec = res % 32 == 0 ? 32 : row_alignment(res);
  x.e.kept = static_cast<uint16_t*>(f.kept), x.e.ldk = f.ldk;
  x.e.kept2 = static_cast<uint16_t*>(f.kept2), x.e.ldk2 = f.ldk2;
  bool encoded = true;
  const cudaError_t e = f.gated ? launch_rows<false, kGated>(g, num_sms, s, &encoded, x) : launch_rows<false, kLinear>(g, num_sms, s, &encoded, x);
  if (!encoded) return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "grouped product: %s", cudaGetErrorString(e));
}

ws_status_t launch_two_products(const GroupedRows& g, const void* second, int64_t ld2, int64_t stride2, int num_sms, cudaStream_t s) {
  if (!encoder()) return routing_fail(WS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  bool encoded = true;
  const cudaError_t e = launch_rows<true, kPlain, true>(g, num_sms, s, &encoded, {second, ld2, stride2, {}, false});
  if (!encoded) return routing_fail(WS_ERR_INVALID_ARG, "a matrix cannot be described to the copy engine");
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "grouped product: %s", cudaGetErrorString(e));
}

ws_status_t launch_slopes(const SlopeRows& r, int num_sms, cudaStream_t s) {
  const int64_t nnz = r.r->nnz;
  SlopeParams p{};
  p.offsets = r.r->offsets;
  p.groups = static_cast<int>(r.r->ncols);
  p.width = static_cast<int>(r.width);
  p.padded = static_cast<int>(r.padded);
  p.g = static_cast<const uint16_t*>(r.g), p.ldg = r.ldg, p.vecg = rows16(r.g, r.ldg, nnz);
  p.z = static_cast<const uint16_t*>(r.z), p.ldz = r.ldz, p.vecz = rows16(r.z, r.ldz, nnz);
  p.up = static_cast<const uint16_t*>(r.up), p.ldup = r.ldup, p.vecup = rows16(r.up, r.ldup, nnz);
  p.out = static_cast<uint16_t*>(r.out);
  p.sums = r.sums;
  p.act = r.z ? r.act : WS_ACT_NONE;
  const bool both = r.up != nullptr, sums = r.sums != nullptr;
  p.tile = slope_rows(nnz, p.padded, sums);
  const int64_t tiles = sums ? slope_tiles(nnz, p.groups, p.padded) : up(nnz, p.tile);
  cudaError_t e = both ? (sums ? launch_slope<true, true>(p, r.half, tiles, num_sms, s) : launch_slope<true, false>(p, r.half, tiles, num_sms, s))
                       : (sums ? launch_slope<false, true>(p, r.half, tiles, num_sms, s) : launch_slope<false, false>(p, r.half, tiles, num_sms, s));
  if (e == cudaSuccess && sums) {
    BiasParams b{};
    b.offsets = p.offsets, b.groups = p.groups, b.width = p.width, b.padded = p.padded, b.parts = both ? 2 : 1, b.sums = p.sums, b.tile = p.tile;
    for (int i = 0; i < 2; ++i) b.out[i] = static_cast<uint16_t*>(r.gbias[i]), b.ld[i] = r.ldgbias[i];
    const dim3 grid(static_cast<unsigned>(up(p.width, 32)), static_cast<unsigned>(p.groups), static_cast<unsigned>(b.parts));
    e = launch_early(r.half ? bias_kernel<true> : bias_kernel<false>, grid, kSlopeThreads, 0, s, 1, b);
  }
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "gradients of the sums: %s", cudaGetErrorString(e));
}

}  // namespace wsk
