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

// A stack of 16-bit matrices that a kernel reads in 16-byte pieces, or (read false) writes.
struct Operand {
  const void* p;
  int64_t groups, rows, width, ld, stride;
  bool read;
  bool aligned() const {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld % 8 == 0) && (groups <= 1 || stride % 8 == 0);
  }
};

ws_status_t check_operands(std::initializer_list<Operand> all) {
  constexpr int64_t kMost = int64_t{1} << 36;
  for (const Operand& d : all) {
    if (d.groups == 0 || d.rows == 0 || d.width == 0) continue;
    if (!d.p) return routing_fail(WS_ERR_INVALID_ARG, "NULL matrix");
    if ((d.rows > 1 && (d.ld < (d.read ? 0 : d.width) || d.ld >= kMost)) || (d.groups > 1 && (d.stride < 0 || d.stride >= kMost)))
      return routing_fail(WS_ERR_INVALID_ARG, "row stride smaller than the row, negative or too large");
    if (reinterpret_cast<uintptr_t>(d.p) % 2) return routing_fail(WS_ERR_INVALID_ARG, "misaligned matrix");
  }
  return WS_OK;
}

// Replaces operands whose rows do not start at multiples of 16 bytes by copies in `scratch` (one launch).
class Aligner {
 public:
  Aligner(void* scratch, int64_t bytes) : at_(static_cast<char*>(scratch)), left_(bytes) {}
  bool add(Operand* d, const int64_t* offsets = nullptr) {
    if (d->groups == 0 || d->rows == 0 || d->width == 0) return true;
    const int64_t packs = (d->width + 7) / 8;
    if (d->aligned() && (d->rows <= 1 || d->ld >= d->width)) {
      if (d->rows <= 1) d->ld = 8 * packs;
      if (d->groups <= 1) d->stride = d->ld * d->rows;
      return true;
    }
    const int64_t need = d->groups * d->rows * packs * 16;
    if (!at_ || need > left_ || reinterpret_cast<uintptr_t>(at_) % 16) return false;
    copies_.m[copies_.count++] = {static_cast<const uint16_t*>(d->p), d->ld, d->stride, d->groups, d->rows,
                                  static_cast<int>(d->width), packs, reinterpret_cast<uint16_t*>(at_), offsets};
    d->p = at_;
    d->ld = 8 * packs;
    d->stride = d->ld * d->rows;
    at_ += need;
    left_ -= need;
    return true;
  }
  void run(cudaStream_t s) {
    if (copies_.count) launch_align(copies_, s);
  }

 private:
  char* at_;
  int64_t left_;
  AlignedCopies copies_{};
};

ws_status_t short_scratch() {
  return routing_fail(WS_ERR_INVALID_ARG, "no room in scratch for copies of operands that are not 16-byte aligned");
}

ws_status_t check_product(const ws_routing* r, int64_t N, int64_t K, ws_dtype_t dt) {
  if (const ws_status_t st = check(r)) return st;
  if (dt != WS_BF16 && dt != WS_F16) return routing_fail(WS_ERR_DTYPE, "products are of bfloat16 or half matrices");
  if (N < 0 || K < 0) return routing_fail(WS_ERR_INVALID_ARG, "negative size");
  if (N > kMaxWidth || K > kMaxWidth) return routing_fail(WS_ERR_OVERFLOW, "rows of more than 2^24 values");
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
  if (nrows < 0 || ncols < 0) return 0;
  if (sm_count(&sms) != WS_OK) return -1;
  const int64_t chunks = routing_chunks(nrows, ncols, sms);
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
  const int64_t chunks = routing_chunks(r->nrows, r->ncols, sms);
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
                              void* scratch, int64_t scratch_bytes, ws_stream_t stream) {
  if (const ws_status_t st = check_product(r, N, K, dtype)) return st;
  Operand x{xs, 1, r->nnz, K, ldxs, 0, true}, w{W, r->ncols, N, K, ldw, stride, true};
  if (const ws_status_t st = check_operands({x, w, {ys, 1, r->nnz, N, ldys, 0, false}})) return st;
  if (r->nnz == 0 || N == 0) return WS_OK;
  if (K == 0) return zero_rows(ys, r->nnz, N, ldys, stream);
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  Aligner align(scratch, scratch_bytes);
  if (!align.add(&x) || !align.add(&w, r->offsets)) return short_scratch();
  align.run(cuda_stream(stream));
  return launch_grouped({r, dtype == WS_F16, x.p, x.ld, w.p, w.ld, w.stride, ys, ldys, N, K}, false, sms, cuda_stream(stream));
}

ws_status_t ws_routing_matmul_backward(const ws_routing* r, const void* gys, int64_t ldgys, const void* xs, int64_t ldxs,
                                       const void* W, int64_t ldw, int64_t stride, int64_t N, int64_t K, void* gxs,
                                       int64_t ldgxs, void* gW, int64_t ldgw, int64_t gstride, ws_dtype_t dtype,
                                       void* scratch, int64_t scratch_bytes, ws_stream_t stream) {
  if (const ws_status_t st = check_product(r, N, K, dtype)) return st;
  Operand g{gys, 1, r->nnz, N, ldgys, 0, true};
  Operand x{xs, 1, gW ? r->nnz : 0, K, ldxs, 0, true}, w{W, gxs ? r->ncols : 0, N, K, ldw, stride, true};
  if (const ws_status_t st = check_operands({g, x, w, {gxs, 1, gxs ? r->nnz : 0, K, ldgxs, 0, false},
                                             {gW, gW ? r->ncols : 0, N, K, ldgw, gstride, false}}))
    return st;
  const bool rows = gxs && r->nnz > 0 && K > 0, weights = gW && r->ncols > 0 && N > 0 && K > 0;
  if (rows && N == 0)
    if (const ws_status_t st = zero_rows(gxs, r->nnz, K, ldgxs, stream)) return st;
  if (weights && r->nnz == 0)
    for (int64_t e = 0; e < r->ncols; ++e)
      if (const ws_status_t st = zero_rows(static_cast<char*>(gW) + 2 * e * gstride, N, K, ldgw, stream)) return st;
  if (r->nnz == 0 || N == 0 || (!rows && !weights)) return WS_OK;
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  Aligner align(scratch, scratch_bytes);
  if (!align.add(&g) || !align.add(&x) || !align.add(&w, r->offsets)) return short_scratch();
  align.run(cuda_stream(stream));
  if (rows)
    if (const ws_status_t st = launch_grouped({r, dtype == WS_F16, g.p, g.ld, w.p, w.ld, w.stride, gxs, ldgxs, N, K}, true, sms,
                                              cuda_stream(stream)))
      return st;
  return weights ? launch_grouped_weights({r, dtype == WS_F16, x.p, x.ld, nullptr, 0, gstride, gW, ldgw, N, K}, g.p, g.ld, sms,
                                          cuda_stream(stream))
                 : WS_OK;
}

int64_t ws_adapters_scratch(int64_t nnz, int64_t r) {
  return 16 + (nnz <= 0 || r <= 0 ? 0 : nnz * adapters_rank(r) * 4 * static_cast<int64_t>(sizeof(float)));
}

int ws_adapters_many(int64_t nrows, int64_t r) { return nrows >= 0 && r >= 0 && !adapters_step(nrows, r); }

ws_status_t ws_adapters(const ws_adapters_call* call, void* scratch, int64_t scratch_bytes, ws_stream_t stream) {
  if (!call) return routing_fail(WS_ERR_INVALID_ARG, "NULL arguments");
  const ws_adapters_call& c = *call;
  if (c.nrows < 0 || c.ncols < 0 || c.nnz < 0 || c.K < 0 || c.r < 0 || c.N < 0)
    return routing_fail(WS_ERR_INVALID_ARG, "negative size");
  if (c.dtype != WS_BF16 && c.dtype != WS_F16) return routing_fail(WS_ERR_DTYPE, "adapters are bfloat16 or half");
  if (c.nrows > INT32_MAX || c.ncols > INT32_MAX || c.nnz > INT32_MAX || c.K > kMaxWidth || c.N > kMaxWidth || c.r > 4096)
    return routing_fail(WS_ERR_OVERFLOW, "at most %d rows, columns and entries, rows of 2^24 values, rank 4096", INT32_MAX);
  if (c.nnz > 0 && (c.nrows == 0 || c.ncols == 0)) return routing_fail(WS_ERR_SHAPE, "entries in a matrix without rows or columns");
  const bool used = c.nrows > 0 && c.N > 0;
  const bool inner = used && c.nnz > 0 && c.r > 0 && c.K > 0;
  if (!c.rowptr || (c.nnz > 0 && (!c.colidx || !c.vals)) || (used && !scratch))
    return routing_fail(WS_ERR_INVALID_ARG, "NULL pointer");
  Operand x{c.x, 1, inner ? c.nrows : 0, c.K, c.ldx, 0, true}, A{c.A, inner ? c.ncols : 0, c.r, c.K, c.lda, c.strideA, true},
      B{c.B, inner ? c.ncols : 0, c.N, c.r, c.ldb, c.strideB, true};
  if (const ws_status_t st = check_operands({x, A, B, {c.y, 1, c.nrows, c.N, c.ldy, 0, false},
                                             {c.base, 1, c.base ? c.nrows : 0, c.N, c.ldbase, 0, false}}))
    return st;
  const int64_t own = ws_adapters_scratch(inner ? c.nnz : 0, c.r);
  if (used && (scratch_bytes < own || reinterpret_cast<uintptr_t>(scratch) % 16))
    return routing_fail(WS_ERR_INVALID_ARG, "scratch smaller than ws_adapters_scratch, or misaligned");
  if (!used) return WS_OK;
  ws_adapters_call run = c;
  if (!inner) run.nnz = 0;  // nothing to add: entry ranges are cut to [0, 0]
  if (inner && !adapters_step(c.nrows, c.r)) {
    Aligner align(static_cast<char*>(scratch) + own, scratch_bytes - own);
    if (!align.add(&x) || !align.add(&A) || !align.add(&B)) return short_scratch();
    align.run(cuda_stream(stream));
    run.x = x.p, run.ldx = x.ld, run.A = A.p, run.lda = A.ld, run.strideA = A.stride, run.B = B.p, run.ldb = B.ld, run.strideB = B.stride;
  }
  int sms = 0;
  if (const ws_status_t st = sm_count(&sms)) return st;
  if (const ws_status_t st = launch_adapters(run, scratch, sms, cuda_stream(stream))) return st;
  return launched("ws_adapters");
}

}  // extern "C"
