// C entry points of the operations on routing matrices (declared in
// include/ws_spgemm.h): argument checks, then the launchers.  Nothing here
// allocates, waits or throws.
#include <climits>
#include <initializer_list>

#include "routing.cuh"

using namespace wsk;

namespace {

constexpr int64_t kMaxWidth = 1 << 24;

bool row_type(ws_dtype_t dt) { return dt == WS_F32 || dt == WS_BF16 || dt == WS_F16; }

cudaStream_t cuda_stream(ws_stream_t s) { return reinterpret_cast<cudaStream_t>(s); }

ws_status_t launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

ws_status_t sm_count(int* n) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "device query: %s", cudaGetErrorString(e));
}

// Sizes and arrays of a routing matrix; `built`: its transpose is there too.
ws_status_t check(const ws_routing* r) {
  if (!r) return routing_fail(WS_ERR_INVALID_ARG, "NULL routing matrix");
  if (r->nrows < 0 || r->ncols < 0 || r->nnz < 0) return routing_fail(WS_ERR_INVALID_ARG, "negative size");
  if (r->nrows > INT32_MAX || r->nnz > INT32_MAX || r->ncols > kRouteMaxCols)
    return routing_fail(WS_ERR_OVERFLOW, "routing matrix %lld x %lld with %lld entries: at most %d columns and %d rows and entries",
                        static_cast<long long>(r->nrows), static_cast<long long>(r->ncols),
                        static_cast<long long>(r->nnz), kRouteMaxCols, INT32_MAX);
  if (r->nnz > 0 && (r->nrows == 0 || r->ncols == 0))
    return routing_fail(WS_ERR_SHAPE, "entries in a routing matrix without rows or columns");
  if (!r->rowptr || !r->offsets || !r->status || (r->nnz > 0 && (!r->colidx || !r->rows || !r->entries || !r->slots)))
    return routing_fail(WS_ERR_INVALID_ARG, "NULL array in a routing matrix");
  return WS_OK;
}

struct Dense {
  const void* p;
  int64_t rows, ld;
};

// The dense operands of a call that moves rows of `width` values.
ws_status_t check_rows(const ws_routing* r, int64_t width, ws_dtype_t dt, std::initializer_list<Dense> all) {
  if (const ws_status_t st = check(r)) return st;
  if (!row_type(dt)) return routing_fail(WS_ERR_DTYPE, "dense rows are float, bfloat16 or half");
  if (width < 0) return routing_fail(WS_ERR_INVALID_ARG, "negative width");
  if (width > kMaxWidth || r->nrows * ((width + 31) / 32) / 8 >= INT32_MAX)
    return routing_fail(WS_ERR_OVERFLOW, "rows of %lld values", static_cast<long long>(width));
  const uintptr_t size = dt == WS_F32 ? 4 : 2;
  for (const Dense& d : all) {
    if (d.rows > 0 && width > 0 && !d.p) return routing_fail(WS_ERR_INVALID_ARG, "NULL dense matrix");
    if (d.ld < width && d.rows > 1) return routing_fail(WS_ERR_INVALID_ARG, "row stride smaller than the row");
    if (reinterpret_cast<uintptr_t>(d.p) % size) return routing_fail(WS_ERR_INVALID_ARG, "misaligned dense matrix");
  }
  return WS_OK;
}

// A 16-bit matrix that the copy engine reads, or (read false) a result.
struct Operand {
  const void* p;
  int64_t rows, width, ld;
  bool read;
};

ws_status_t check_product(const ws_routing* r, int64_t N, int64_t K, ws_dtype_t dt, int64_t group_stride,
                          std::initializer_list<Operand> all) {
  if (const ws_status_t st = check(r)) return st;
  if (dt != WS_BF16 && dt != WS_F16) return routing_fail(WS_ERR_DTYPE, "products are of bfloat16 or half matrices");
  if (N < 0 || K < 0) return routing_fail(WS_ERR_INVALID_ARG, "negative size");
  if (N > kMaxWidth || K > kMaxWidth) return routing_fail(WS_ERR_OVERFLOW, "rows of more than 2^24 values");
  for (const Operand& d : all) {
    if (d.rows == 0 || d.width == 0) continue;
    if (!d.p || (d.rows > 1 && d.ld < d.width)) return routing_fail(WS_ERR_INVALID_ARG, "NULL matrix, or row stride smaller than the row");
    if (reinterpret_cast<uintptr_t>(d.p) % (d.read ? 16 : 2) || (d.read && (d.ld % 8 || d.ld >= int64_t{1} << 36)))
      return routing_fail(WS_ERR_INVALID_ARG, "operands of a product start and have row strides at multiples of 16 bytes");
  }
  if (r->ncols > 1 && (group_stride % 8 || group_stride < 0 || group_stride >= int64_t{1} << 36))
    return routing_fail(WS_ERR_INVALID_ARG, "matrices of a product are a multiple of 16 bytes apart");
  return WS_OK;
}

// Rows of 16-bit zeros: a sum over nothing.
ws_status_t zero_rows(void* p, int64_t rows, int64_t width, int64_t ld, ws_stream_t stream) {
  const cudaError_t e = ld == width || rows == 1
                            ? cudaMemsetAsync(p, 0, static_cast<size_t>(rows) * width * 2, cuda_stream(stream))
                            : cudaMemset2DAsync(p, static_cast<size_t>(ld) * 2, 0, static_cast<size_t>(width) * 2,
                                                static_cast<size_t>(rows), cuda_stream(stream));
  return e == cudaSuccess ? WS_OK : routing_fail(WS_ERR_CUDA, "memset: %s", cudaGetErrorString(e));
}

}  // namespace

extern "C" {

ws_status_t ws_topk_route(const void* logits, int64_t rows, int64_t cols, int64_t ld, ws_dtype_t dtype, int k,
                          int normalize, int64_t* rowptr, int32_t* colidx, float* vals, ws_stream_t stream) {
  if (rows < 0 || cols < 1 || k < 1 || k > cols || k > kRouteMaxK)
    return routing_fail(WS_ERR_INVALID_ARG, "k must be in 1..min(cols, %d)", kRouteMaxK);
  if (!row_type(dtype)) return routing_fail(WS_ERR_DTYPE, "logits are float, bfloat16 or half");
  if (cols > kRouteMaxCols || rows > INT32_MAX / k)
    return routing_fail(WS_ERR_OVERFLOW, "at most %d columns and %d entries", kRouteMaxCols, INT32_MAX);
  if (!rowptr || (rows > 0 && (!logits || !colidx || !vals)) || (rows > 1 && ld < cols) ||
      reinterpret_cast<uintptr_t>(logits) % (dtype == WS_F32 ? 4 : 2))
    return routing_fail(WS_ERR_INVALID_ARG, "NULL or misaligned pointer, or row stride smaller than the row");
  if (rows == 0) {
    cudaMemsetAsync(rowptr, 0, sizeof(int64_t), cuda_stream(stream));
    return launched("ws_topk_route");
  }
  launch_topk_route(logits, rows, static_cast<int>(cols), ld, dtype, k, normalize != 0, rowptr, colidx, vals, cuda_stream(stream));
  return launched("ws_topk_route");
}

ws_status_t ws_topk_route_backward(const void* logits, int64_t rows, int64_t cols, int64_t ld, ws_dtype_t dtype,
                                   int k, int normalize, const int32_t* colidx, const float* vals,
                                   const float* gvals, void* glogits, int64_t ldg, ws_stream_t stream) {
  if (rows < 0 || cols < 1 || k < 1 || k > cols || k > kRouteMaxK)
    return routing_fail(WS_ERR_INVALID_ARG, "k must be in 1..min(cols, %d)", kRouteMaxK);
  if (!row_type(dtype)) return routing_fail(WS_ERR_DTYPE, "logits are float, bfloat16 or half");
  if (cols > kRouteMaxCols || rows > INT32_MAX / k)
    return routing_fail(WS_ERR_OVERFLOW, "at most %d columns and %d entries", kRouteMaxCols, INT32_MAX);
  const uintptr_t size = dtype == WS_F32 ? 4 : 2;
  if ((rows > 0 && (!colidx || !vals || !gvals || !glogits || (!normalize && !logits))) || (rows > 1 && ldg < cols) ||
      (rows > 1 && !normalize && ld < cols) || reinterpret_cast<uintptr_t>(glogits) % size ||
      (!normalize && reinterpret_cast<uintptr_t>(logits) % size))
    return routing_fail(WS_ERR_INVALID_ARG, "NULL or misaligned pointer, or row stride smaller than the row");
  if (rows == 0) return WS_OK;
  launch_topk_route_backward(logits, rows, static_cast<int>(cols), ld, dtype, k, normalize != 0, colidx, vals, gvals,
                             glogits, ldg, cuda_stream(stream));
  return launched("ws_topk_route_backward");
}

int64_t ws_routing_scratch(int64_t nrows, int64_t ncols) {
  int sms = 0;
  if (nrows < 0 || ncols < 0 || sm_count(&sms) != WS_OK) return 0;
  const int64_t chunks = routing_chunks(nrows, sms);
  return chunks == 1 ? 0 : chunks * ((ncols + 3) & ~int64_t{3}) * static_cast<int64_t>(sizeof(int32_t));
}

ws_status_t ws_routing_build(const ws_routing* r, void* scratch, int64_t scratch_bytes, ws_stream_t stream) {
  if (const ws_status_t st = check(r)) return st;
  if (r->nnz == 0) {
    cudaMemsetAsync(r->status, 0, sizeof(int32_t), cuda_stream(stream));
    cudaMemsetAsync(r->offsets, 0, static_cast<size_t>(r->ncols + 1) * sizeof(int64_t), cuda_stream(stream));
    return launched("ws_routing_build");
  }
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  const int64_t chunks = routing_chunks(r->nrows, sms);
  if (chunks > 1 && (!scratch || reinterpret_cast<uintptr_t>(scratch) % 16 ||
                     scratch_bytes < chunks * ((r->ncols + 3) & ~int64_t{3}) * static_cast<int64_t>(sizeof(int32_t))))
    return routing_fail(WS_ERR_INVALID_ARG, "scratch smaller than ws_routing_scratch, or misaligned");
  launch_routing_build(*r, static_cast<int32_t*>(scratch), sms, cuda_stream(stream));
  return launched("ws_routing_build");
}

ws_status_t ws_routing_dispatch(const ws_routing* r, const void* x, int64_t ldx, void* xs, int64_t ldxs,
                                int64_t width, ws_dtype_t dtype, ws_stream_t stream) {
  if (const ws_status_t st = check_rows(r, width, dtype, {{x, r ? r->nrows : 0, ldx}, {xs, r ? r->nnz : 0, ldxs}})) return st;
  if (r->nnz == 0 || width == 0) return WS_OK;
  launch_dispatch(*r, x, ldx, xs, ldxs, width, dtype, cuda_stream(stream));
  return launched("ws_routing_dispatch");
}

ws_status_t ws_routing_dispatch_backward(const ws_routing* r, const void* gxs, int64_t ldgxs, void* gx, int64_t ldgx,
                                         int64_t width, ws_dtype_t dtype, ws_stream_t stream) {
  if (const ws_status_t st = check_rows(r, width, dtype, {{gxs, r ? r->nnz : 0, ldgxs}, {gx, r ? r->nrows : 0, ldgx}})) return st;
  if (r->nrows == 0 || width == 0) return WS_OK;
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  launch_combine(*r, false, gxs, ldgxs, gx, ldgx, width, dtype, sms, cuda_stream(stream));
  return launched("ws_routing_dispatch_backward");
}

ws_status_t ws_routing_combine(const ws_routing* r, const void* ys, int64_t ldys, void* y, int64_t ldy,
                               int64_t width, ws_dtype_t dtype, ws_stream_t stream) {
  if (const ws_status_t st = check_rows(r, width, dtype, {{ys, r ? r->nnz : 0, ldys}, {y, r ? r->nrows : 0, ldy}})) return st;
  if (r->nnz > 0 && !r->vals) return routing_fail(WS_ERR_INVALID_ARG, "NULL values");
  if (r->nrows == 0 || width == 0) return WS_OK;
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  launch_combine(*r, true, ys, ldys, y, ldy, width, dtype, sms, cuda_stream(stream));
  return launched("ws_routing_combine");
}

ws_status_t ws_routing_combine_backward(const ws_routing* r, const void* gy, int64_t ldgy, const void* ys,
                                        int64_t ldys, void* gys, int64_t ldgys, float* gvals, int64_t width,
                                        ws_dtype_t dtype, ws_stream_t stream) {
  if (const ws_status_t st = check_rows(r, width, dtype, {{gy, r ? r->nrows : 0, ldgy}, {ys, r ? r->nnz : 0, ldys},
                                                          {gys, r ? r->nnz : 0, ldgys}}))
    return st;
  if (r->nnz > 0 && (!r->vals || !gvals)) return routing_fail(WS_ERR_INVALID_ARG, "NULL values");
  if (r->nnz == 0) return WS_OK;
  if (width == 0) {
    cudaMemsetAsync(gvals, 0, static_cast<size_t>(r->nnz) * sizeof(float), cuda_stream(stream));
    return launched("ws_routing_combine_backward");
  }
  launch_combine_backward(*r, gy, ldgy, ys, ldys, gys, ldgys, gvals, width, dtype, cuda_stream(stream));
  return launched("ws_routing_combine_backward");
}

ws_status_t ws_routing_matmul(const ws_routing* r, const void* xs, int64_t ldxs, const void* W, int64_t ldw,
                              int64_t stride, int64_t N, int64_t K, void* ys, int64_t ldys, ws_dtype_t dtype,
                              ws_stream_t stream) {
  if (const ws_status_t st = check_product(r, N, K, dtype, stride, {{xs, r ? r->nnz : 0, K, ldxs, true}, {W, N, K, ldw, true},
                                                                    {ys, r ? r->nnz : 0, N, ldys, false}}))
    return st;
  if (r->nnz == 0 || N == 0) return WS_OK;
  if (K == 0) return zero_rows(ys, r->nnz, N, ldys, stream);
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  return launch_grouped({r, dtype == WS_F16, xs, ldxs, W, ldw, stride, ys, ldys, N, K}, false, sms, cuda_stream(stream));
}

ws_status_t ws_routing_matmul_rows(const ws_routing* r, const void* gys, int64_t ldgys, const void* W, int64_t ldw,
                                   int64_t stride, int64_t N, int64_t K, void* gxs, int64_t ldgxs, ws_dtype_t dtype,
                                   ws_stream_t stream) {
  if (const ws_status_t st = check_product(r, N, K, dtype, stride, {{gys, r ? r->nnz : 0, N, ldgys, true}, {W, N, K, ldw, true},
                                                                    {gxs, r ? r->nnz : 0, K, ldgxs, false}}))
    return st;
  if (r->nnz == 0 || K == 0) return WS_OK;
  if (N == 0) return zero_rows(gxs, r->nnz, K, ldgxs, stream);
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  return launch_grouped({r, dtype == WS_F16, gys, ldgys, W, ldw, stride, gxs, ldgxs, N, K}, true, sms, cuda_stream(stream));
}

ws_status_t ws_routing_matmul_weights(const ws_routing* r, const void* gys, int64_t ldgys, const void* xs,
                                      int64_t ldxs, int64_t N, int64_t K, void* gW, int64_t ldgw, int64_t stride,
                                      ws_dtype_t dtype, ws_stream_t stream) {
  if (const ws_status_t st = check_product(r, N, K, dtype, 0, {{gys, r ? r->nnz : 0, N, ldgys, true}, {xs, r ? r->nnz : 0, K, ldxs, true},
                                                               {gW, N, K, ldgw, false}}))
    return st;
  if (r->ncols == 0 || N == 0 || K == 0) return WS_OK;
  if (r->nnz == 0) {
    for (int64_t e = 0; e < r->ncols; ++e)
      if (const ws_status_t st = zero_rows(static_cast<char*>(gW) + 2 * e * stride, N, K, ldgw, stream)) return st;
    return WS_OK;
  }
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  return launch_grouped_weights({r, dtype == WS_F16, xs, ldxs, nullptr, 0, stride, gW, ldgw, N, K}, gys, ldgys, sms, cuda_stream(stream));
}

int64_t ws_adapters_scratch(int64_t nnz, int64_t r) {
  return 16 + (nnz <= 0 || r <= 0 ? 0 : nnz * adapters_rank(r) * 4 * static_cast<int64_t>(sizeof(float)));
}

ws_status_t ws_adapters(const ws_adapters_call* call, void* scratch, int64_t scratch_bytes, ws_stream_t stream) {
  if (!call) return routing_fail(WS_ERR_INVALID_ARG, "NULL arguments");
  const ws_adapters_call& c = *call;
  if (c.nrows < 0 || c.ncols < 0 || c.nnz < 0 || c.K < 0 || c.r < 0 || c.N < 0)
    return routing_fail(WS_ERR_INVALID_ARG, "negative size");
  if (c.dtype != WS_BF16 && c.dtype != WS_F16) return routing_fail(WS_ERR_DTYPE, "adapters are bfloat16 or half");
  if (c.nrows > INT32_MAX || c.ncols > INT32_MAX || c.nnz > INT32_MAX || c.K > kMaxWidth || c.N > kMaxWidth || c.r > 4096)
    return routing_fail(WS_ERR_OVERFLOW, "at most %d rows, columns and entries, rows of 2^24 values, rank 4096", INT32_MAX);
  if (c.nnz > 0 && (c.nrows == 0 || c.ncols == 0)) return routing_fail(WS_ERR_SHAPE, "entries in a matrix without rows or columns");
  const bool used = c.nrows > 0 && c.N > 0, prompt = !adapters_step(c.nrows, c.r);
  const bool inner = used && c.nnz > 0 && c.r > 0 && c.K > 0;
  if (!c.rowptr || (c.nnz > 0 && (!c.colidx || !c.vals)) || (used && (!c.y || !scratch)) || (inner && (!c.x || !c.A || !c.B)))
    return routing_fail(WS_ERR_INVALID_ARG, "NULL pointer");
  if (used && c.nrows > 1 && (c.ldy < c.N || (c.base && c.ldbase < c.N)))
    return routing_fail(WS_ERR_INVALID_ARG, "row stride smaller than the row");
  if (inner) {
    const auto off16 = [](const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 != 0 || ld % 8 != 0; };
    if (off16(c.x, c.nrows > 1 ? c.ldx : 0) || off16(c.A, c.r > 1 ? c.lda : 0) || (c.ncols > 1 && c.strideA % 8))
      return routing_fail(WS_ERR_INVALID_ARG, "x and A start and have strides at multiples of 16 bytes");
    if (prompt && (off16(c.B, c.N > 1 ? c.ldb : 0) || (c.ncols > 1 && c.strideB % 8)))
      return routing_fail(WS_ERR_INVALID_ARG, "for many tokens B starts and has strides at multiples of 16 bytes");
    if ((c.nrows > 1 && c.ldx < c.K) || (c.r > 1 && c.lda < c.K) || (c.N > 1 && c.ldb < c.r) || c.strideA < 0 || c.strideB < 0)
      return routing_fail(WS_ERR_INVALID_ARG, "row stride smaller than the row");
  }
  if (used && (scratch_bytes < ws_adapters_scratch(inner ? c.nnz : 0, c.r) || reinterpret_cast<uintptr_t>(scratch) % 16))
    return routing_fail(WS_ERR_INVALID_ARG, "scratch smaller than ws_adapters_scratch, or misaligned");
  if ((reinterpret_cast<uintptr_t>(c.y) | reinterpret_cast<uintptr_t>(c.base) | reinterpret_cast<uintptr_t>(c.B)) % 2)
    return routing_fail(WS_ERR_INVALID_ARG, "misaligned matrix");
  if (!used) return WS_OK;
  ws_adapters_call run = c;
  if (!inner) run.nnz = 0;  // nothing to add: entry ranges are cut to [0, 0]
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  if (const ws_status_t st = launch_adapters(run, scratch, sms, cuda_stream(stream))) return st;
  return launched("ws_adapters");
}

}  // extern "C"
