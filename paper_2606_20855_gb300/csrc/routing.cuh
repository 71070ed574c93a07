// Declarations shared by the operators on sparse routing matrices: route.cu
// (rows of R chosen from logits), routing.cu (R transposed; rows gathered and
// summed), grouped.cu (products by column of R), adapters.cu, routing_api.cu.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "ws_spgemm.h"

namespace wsk {

constexpr int kRouteMaxCols = 1024;  // columns of a routing matrix: a warp of the choice holds a row, 32 logits a lane
constexpr int kRouteMaxK = 32;       // entries chosen in a row: one a lane

// Message of ws_last_error() on the calling thread (api.cu); never throws.
ws_status_t routing_fail(ws_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N consecutive values of T, moved as one access.
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void unpack(const Pack<T, N>& p, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = to_f32<T>(p.v[i]);
}
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> pack(const float (&f)[N]) {
  Pack<T, N> p;
#pragma unroll
  for (int i = 0; i < N; ++i) p.v[i] = from_f32<T>(f[i]);
  return p;
}

// Stored entries of row i, whatever rowptr holds: a range inside [0, nnz].
__device__ __forceinline__ void entry_range(const int64_t* rowptr, int64_t i, int64_t nnz, int* begin, int* end) {
  const int64_t b = rowptr[i], e = rowptr[i + 1];
  const int64_t bc = b < 0 ? 0 : b > nnz ? nnz : b;
  *begin = static_cast<int>(bc);
  *end = static_cast<int>(e < bc ? bc : e > nnz ? nnz : e);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// A 16-bit value (half or bfloat16) and a float.
template <bool half>
__device__ __forceinline__ float value16(uint16_t u) {
  if constexpr (half) return __half2float(__ushort_as_half(u));
  else return __uint_as_float(static_cast<uint32_t>(u) << 16);
}
template <bool half>
__device__ __forceinline__ uint16_t bits16(float f) {
  if constexpr (half) return __half_as_ushort(__float2half_rn(f));
  else return __bfloat16_as_ushort(__float2bfloat16_rn(f));
}
// Two of them, a in the lower half.
template <bool half>
__device__ __forceinline__ uint32_t pair16(float a, float b) {
  if constexpr (half) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
// The warp-level matrix instruction: d (16 x 8) += a (16 x 16) b (16 x 8).  Lane 4 g + q holds rows g (a0, a2) and g + 8 (a1,
// a3) of a and column g of b; a0, a1, b0 are one pair of the contraction index, a2, a3, b1 another, the same pairs for all
// lanes of a q.  d: rows g (d0, d1) and g + 8, columns 2 q and 2 q + 1.
template <bool half>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
  if constexpr (half)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Values k .. k + 7 of a row of K, zero past its end; vec: the row is 16-byte aligned.
__device__ __forceinline__ uint4 load8(const uint16_t* row, int k, int K, bool vec = true) {
  if (vec && k + 8 <= K) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t w[4] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < K) w[i >> 1] |= static_cast<uint32_t>(row[k + i]) << (16 * (i & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// A kernel that may start while the one before it on the stream still runs (as soon as all of that one's CTAs have called
// may_start_next, or are done) and calls wait_for_last before it touches what that one writes or reads.  Every CTA calls it, so that the
// kernel's end comes after the end of the one before.  `together`: CTAs of a cluster.
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, int together, A... args) {
  cudaLaunchAttribute attrs[2]{};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = together;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(threads);
  config.dynamicSmemBytes = smem;
  config.stream = s;
  config.attrs = attrs;
  config.numAttrs = together > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&config, kernel, static_cast<P>(args)...);
}
__device__ __forceinline__ void may_start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Launchers.  They queue kernels on s and leave errors to cudaGetLastError.
void launch_topk_route(const void* logits, int64_t rows, int cols, int64_t ld, ws_dtype_t dt, int k, bool normalize,
                       int64_t* rowptr, int32_t* colidx, float* vals, cudaStream_t s);
void launch_topk_route_backward(const void* logits, int64_t rows, int cols, int64_t ld, ws_dtype_t dt, int k,
                                bool normalize, const int32_t* colidx, const float* vals, const float* gvals,
                                void* glogits, int64_t ldg, cudaStream_t s);
int64_t routing_chunks(int64_t nrows, int64_t ncols, int num_sms);  // chunks of rows counted apart (1: one launch does it all)
void launch_routing_build(const ws_routing& r, int32_t* counts, int num_sms, cudaStream_t s);
void launch_dispatch(const ws_routing& r, const void* x, int64_t ldx, void* xs, int64_t ldxs, int64_t width,
                     ws_dtype_t dt, cudaStream_t s);
void launch_combine(const ws_routing& r, bool weighted, const void* ys, int64_t ldys, void* y, int64_t ldy,
                    int64_t width, ws_dtype_t dt, int num_sms, cudaStream_t s);
void launch_combine_backward(const ws_routing& r, const void* gy, int64_t ldgy, const void* ys, int64_t ldys,
                             void* gys, int64_t ldgys, float* gvals, int64_t width, ws_dtype_t dt, cudaStream_t s);

// `groups` matrices of `rows` rows of 16-bit values, copied to contiguous rows of `packs` 16-byte pieces (zeros past the width).
struct AlignedCopy {
  const uint16_t* src;
  int64_t ld, stride, groups, rows;
  int width;
  int64_t packs;
  uint16_t* dst;
  const int64_t* offsets;  // group g is copied if offsets[g] != offsets[g + 1] (NULL: always)
};
struct AlignedCopies {
  AlignedCopy m[3];
  int count;
};
void launch_align(const AlignedCopies& c, cudaStream_t s);

// Products by column of R (grouped.cu).  x: nnz rows in slot order; w: ncols matrices N x K; 16-bit values, addresses
// and strides multiples of 16 bytes.  out is not aligned further than its type.
struct GroupedRows {
  const ws_routing* r;
  bool half;
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw, group_stride;
  void* out;
  int64_t ldo;
  int64_t N, K;
};
// transposed: out = rows of x (N values) times W, else rows of x (K values) times W^T.
ws_status_t launch_grouped(const GroupedRows& g, bool transposed, int num_sms, cudaStream_t s);
// out[e] (N x K, ldo, group_stride) = sum over the rows of e of gys row (N) times x row (K).
ws_status_t launch_grouped_weights(const GroupedRows& g, const void* gys, int64_t ldgys, int num_sms, cudaStream_t s);

// Ranks kept for an entry of S: h is padded with zeros.
inline int adapters_rank(int64_t r) { return static_cast<int>((r + 15) / 16 * 16); }
// Whether tokens go one by one.  That reads A and B for every token (from L2), 2 rank (K + N) bytes each; a tile of 128 tokens
// reads x once for every few adapters it meets.  K = N = 4096, bfloat16, us of the kernels where all tokens share an adapter, where
// each has its own, one by one | in tiles: 512 tokens of rank 16 26, 37 | 16.5, 411, 256 of rank 32 31, 40 | 16.5, 554, 128 of
// rank 64 47, 57 | 21, 993, 1024 of rank 16 48, 70 | 17.5, 458, 256 of rank 64 84, 100 | 21, 1025.  How many adapters the tokens
// have is known on the device only: above the limit many tokens that each have their own take six to ten times as long as they
// would one by one, below it tokens that share one take up to 2.3 times as long as in tiles.  Rank 0 (base alone) goes by tokens as rank 16 does: one by one is a launch with a row of CTAs a token, of
// which there may be 65535.
inline bool adapters_step(int64_t nrows, int64_t r) { return nrows * (r > 0 ? adapters_rank(r) : 16) <= 8192; }
// scratch: a status word (16 bytes), then up to four parts of h.
ws_status_t launch_adapters(const ws_adapters_call& c, void* scratch, int num_sms, cudaStream_t s);

}  // namespace wsk
