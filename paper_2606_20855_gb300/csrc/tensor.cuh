// Barriers, copies and matrix instructions of sm_103a (PTX), shared by the kernels on the tcgen05 tensor cores, and the
// descriptions of matrices for the copy engine.
//
// Every wait has a limit in time, after which the CTA's roles give up together: `dead` in shared memory is set, copies and
// products in flight are waited for, tensor memory is given back, and an error word tells the host.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace wsk {

constexpr unsigned long long kWaitLimitNs = 2000000000ull;

// One lane of a warp, all of whose lanes are here, the same one at every call: the compiler then knows that a single thread runs
// what follows, and does not wrap each copy and matrix instruction in a loop over lanes.
__device__ __forceinline__ bool elect_one() {
  uint32_t on;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(on));
  return on != 0;
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// The same for arrivals from the other CTA of a pair.
__device__ __forceinline__ bool bar_try_pair(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Whether the phase is over, asked without a wait.
__device__ __forceinline__ bool bar_ask(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// An answer of bar_try takes more than 200 cycles (measured), about half of what a stage's products take: the loops of the kernels
// ask for the next stage, without a wait, before they work on this one, and wait only if the answer was no.
//
// Waits for a phase; gives up after kWaitLimitNs or when another role gave up (*dead).
template <bool kPair = false>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
  const auto there = [&] { return kPair ? bar_try_pair(bar, parity) : bar_try(bar, parity); };
  if (there()) return true;
  const unsigned long long start = now_ns();
  for (unsigned i = 1;; ++i) {
    if (there()) return true;
    if ((i & 31) == 0) {
      if (*dead) return false;
      if (now_ns() - start > kWaitLimitNs) {
        *dead = 1;
        return false;
      }
    }
  }
}

// The same for a whole warp: one lane asks.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int* dead) {
  const bool got = (threadIdx.x & 31) != 0 || bar_wait(bar, parity, dead);
  return __shfl_sync(0xffffffffu, got, 0);
}
// The same for what is waited for on the way out.
__device__ __forceinline__ void bar_wait_short(uint32_t bar, uint32_t parity) {
  const unsigned long long start = now_ns();
  while (!bar_try(bar, parity) && now_ns() - start < kWaitLimitNs / 10) {
  }
}

// Columns of tensor memory, by a whole warp; the address is written to shared memory.
template <int kCols, bool kPair = false>
__device__ __forceinline__ void tmem_alloc(uint32_t slot) {
  if constexpr (kPair) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <int kCols, bool kPair = false>
__device__ __forceinline__ void tmem_free(uint32_t tmem) {
  if constexpr (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
}

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// Copies to this CTA whose bytes are counted at a barrier of the pair's CTA of rank 0.
__device__ __forceinline__ void tma_2d_first(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_3d_first(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::
          "r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
// Where the CTA of rank 0 has what lies at `at` here.
__device__ __forceinline__ uint32_t at_first(uint32_t at) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(at));
  return r;
}
// Both CTAs of a pair (a cluster of two) meet.
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y),
               "r"(src)
               : "memory");
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z),
               "r"(src)
               : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: 8-row groups of
// 1024 bytes follow each other.  MN-major: blocks of 64 (M or N) x 64 (K), in
// which 8 steps of K take 1024 bytes; blocks are 8192 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn_major) {
  const uint64_t lbo = mn_major ? 8192 >> 4 : 1, sbo = 1024 >> 4;
  return (static_cast<uint64_t>(addr >> 4) & 0x3fff) | lbo << 16 | sbo << 32 | 1ull << 46 | 2ull << 61;
}
// K-major with 64 bytes a row (64-byte swizzle): 8-row groups of 512 bytes.
__device__ __forceinline__ uint64_t smem_desc64(uint32_t addr) {
  return (static_cast<uint64_t>(addr >> 4) & 0x3fff) | 1ull << 16 | static_cast<uint64_t>(512 >> 4) << 32 | 1ull << 46 | 4ull << 61;
}
// Instruction descriptor: D in 32 bits, A and B half or bfloat16, M rows and N columns.
__device__ __forceinline__ uint32_t instr_desc(bool half, bool a_mn, bool b_mn, int M, int N) {
  return 1u << 4 | (half ? 0u : 1u << 7 | 1u << 10) | static_cast<uint32_t>(a_mn) << 15 | static_cast<uint32_t>(b_mn) << 16 |
         static_cast<uint32_t>(N >> 3) << 17 | static_cast<uint32_t>(M >> 4) << 24;
}

__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// A product of a pair: A's upper and lower 128 rows and the halves of B's columns lie in the two CTAs' shared memory at the same
// places, each CTA's tensor memory receives its rows.  Issued by the CTA of rank 0.
__device__ __forceinline__ void mma_f16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
// The arrival at the barriers of both.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"(static_cast<uint16_t>(3))
               : "memory");
}
// Arrival at the barrier of the pair's CTA of rank 0 that lies where `bar` does in this one.
__device__ __forceinline__ void bar_arrive_first(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_first(bar)) : "memory");
}

// 16 consecutive 32-bit columns of the warp's 32 lanes.
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&f)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(r[i]);
}


// 64 consecutive columns.
__device__ __forceinline__ void tmem_load64(uint32_t addr, float (&f)[64]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr + 32 * h)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) f[32 * h + i] = __uint_as_float(r[i]);
  }
}

// ---------------------------------------------------------------- host

using EncodeFn = CUresult(CUDAAPI*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

// Rows of 16-bit values; groups > 0: `groups` matrices of `rows` rows.  Boxes of box_width (64: 128-byte swizzle, 32: 64-byte
// swizzle) values x box_rows.
inline bool encode(CUtensorMap* map, const void* p, bool half, int64_t width, int64_t rows, int64_t ld, int64_t groups,
                   int64_t group_stride, int box_rows, int box_width = 64) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(groups)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2,
                                 static_cast<cuuint64_t>(groups > 1 ? group_stride : ld * rows) * 2};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_width), static_cast<cuuint32_t>(box_rows), 1}, step[3] = {1, 1, 1};
  return encoder()(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, groups > 0 ? 3 : 2,
                   const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   box_width == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace wsk
