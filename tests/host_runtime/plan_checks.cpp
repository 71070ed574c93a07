// The launches of a routing matrix's plan (csrc/routing.cu) on a fake CUDA runtime: a kernel's limit of dynamic shared memory
// belongs to the kernel, so a plan that another thread builds between a launch and the call that raised the limit may not lower it.
// No kernel runs; nothing of the arrays is read.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <map>
#include <utility>

#include <cuda_runtime_api.h>

#include "ws_spgemm.h"

namespace wsk {
void launch_routing_build(const ws_routing& r, int32_t* counts, int num_sms, cudaStream_t s);
}

namespace {

constexpr size_t kDefault = 48 * 1024;
std::map<const void*, size_t> limit;
int launches = 0, refused = 0;
std::function<void()> between;  // what another thread does before the next launch

cudaError_t launch(const void* kernel, size_t smem) {
  if (between) {
    const std::function<void()> f = std::move(between);
    between = nullptr;
    f();
  }
  ++launches;
  const auto at = limit.find(kernel);
  if (smem <= (at == limit.end() ? kDefault : at->second)) return cudaSuccess;
  ++refused;
  return cudaErrorInvalidValue;
}

void build(int64_t rows, int64_t cols, int64_t nnz) {
  ws_routing r{};
  r.nrows = rows, r.ncols = cols, r.nnz = nnz;
  wsk::launch_routing_build(r, nullptr, 152, nullptr);
}

struct Size {
  int64_t rows, cols, nnz;
};

}  // namespace

extern "C" {
cudaError_t cudaFuncSetAttribute(const void* kernel, cudaFuncAttribute, int value) {
  limit[kernel] = static_cast<size_t>(value);
  return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void* kernel, dim3, dim3, void**, size_t smem, cudaStream_t) { return launch(kernel, smem); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* kernel, void**) { return launch(kernel, c->dynamicSmemBytes); }
cudaError_t cudaGetLastError() { return cudaSuccess; }

static struct {
  dim3 grid, block;
  size_t smem;
  cudaStream_t s;
} call;
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t smem, CUstream_st* s) {
  call = {grid, block, smem, s};
  return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3* grid, dim3* block, size_t* smem, void* s) {
  *grid = call.grid, *block = call.block, *smem = call.smem, *static_cast<cudaStream_t*>(s) = call.s;
  return cudaSuccess;
}
cudaError_t __cudaGetKernel(cudaKernel_t* k, const void* f) {
  *k = reinterpret_cast<cudaKernel_t>(const_cast<void*>(f));
  return cudaSuccess;
}
cudaError_t __cudaLaunchKernel(cudaKernel_t k, dim3, dim3, void**, size_t smem, cudaStream_t) { return launch(k, smem); }
void** __cudaRegisterFatBinary(void*) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
char __cudaInitModule(void**) { return 1; }
}

int main() {
  // large plans of each kernel, and smaller ones that need more than the default limit too
  const Size one_large{1024, 1024, 4096}, one_small{300, 1024, 600}, two_large{2000, 1024, 4000}, two_small{2000, 900, 4000},
      many_large{100'000, 1024, 200'000}, many_small{100'000, 500, 200'000}, staged{1000, 64, 40'000}, staged_small{900, 64, 12'000};
  const Size pairs[][2] = {{one_large, one_small}, {two_large, two_small}, {many_large, many_small}, {staged, staged_small},
                           {one_large, staged_small}};
  for (const auto& p : pairs)
    for (int turn = 0; turn < 2; ++turn) {
      limit.clear();
      between = [&] { build(p[1].rows, p[1].cols, p[1].nnz); };
      build(p[0].rows, p[0].cols, p[0].nnz);
      for (int i = 0; i < 2; ++i) build(p[i].rows, p[i].cols, p[i].nnz);
    }
  std::printf("%d launches, %d refused\n", launches, refused);
  return launches > 0 && refused == 0 ? 0 : 1;
}
