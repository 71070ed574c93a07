/*
 * ws_spgemm.h -- C ABI of the GB300 (sm_103a) sparse x sparse -> sparse
 * matrix multiply, C = A * B, with A, B and C in CSR.
 *
 * The operation is the sparse product whose parallel form is Gustavson's
 * algorithm (Sec. 5.1, Fig. "SpGEMM implemented in WingSpan"): every output
 * row C[i,:] = sum over stored A[i,k] of A[i,k] * B[k,:] is owned by exactly
 * one worker, which accumulates it in a private workspace and then writes its
 * own, disjoint segment of C (the shard level of Sec. 4, used for SpGEMM in
 * Sec. 5.1).  The output must satisfy the compressed-format invariants the
 * paper singles out (Sec. 1 and Sec. 3.1: monotone prefix-sum position
 * arrays over contiguous buffers).  The calls follow the tensor lifecycle of
 * Sec. 4 (declare -> update -> freeze): a symbolic pass sizes C and fills its
 * row pointer, the caller allocates C's index and value arrays, and a numeric
 * pass fills them.
 *
 * CSR layout used by every call (0-based):
 *   rowptr  int64_t[nrows + 1], rowptr[0] = 0, non-decreasing, rowptr[nrows] = nnz
 *   colidx  int32_t[nnz], strictly increasing within each row, in [0, ncols)
 *   vals    float[nnz] or double[nnz] (ws_dtype_t)
 * All array pointers are DEVICE pointers on the current CUDA device and are
 * borrowed: the library never frees them, and the caller keeps them alive
 * until the last call that uses the handle has completed on its stream.
 *
 * Result semantics:
 *   - structure: C holds (i, j) iff some stored A[i,k] meets a stored B[k,j]
 *     (structural product; an entry whose sum is exactly zero is kept, stored
 *     zeros in A or B count as entries);
 *   - column indices of every row of C are strictly increasing;
 *   - values are accumulated in the value type of A and B; the order of the
 *     additions is unspecified (results agree with an ordered sequential sum
 *     up to rounding).
 *
 * Errors: every call returns a ws_status_t; no call throws or aborts.
 * Argument, shape and dtype errors are detected on the host before any work
 * is queued.  Failures detected by a kernel are recorded in a status word
 * that the library reads at its next synchronisation point (the end of
 * ws_spgemm_symbolic, or ws_spgemm_wait).  Kernels never trap and every
 * device loop is bounded.  ws_last_error() gives a one-line description of
 * the most recent failure on the calling thread.
 *
 * Threading: handles are not thread-safe.  One output handle serves one
 * product at a time; use separate output handles for products that run
 * concurrently.
 */
#ifndef WS_SPGEMM_H
#define WS_SPGEMM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Same type as cudaStream_t; NULL is the legacy default stream. */
typedef struct CUstream_st* ws_stream_t;

typedef struct ws_csr_s* ws_csr_t;

typedef enum {
  WS_F32 = 1,  /* float  */
  WS_F64 = 2,  /* double */
  WS_BF16 = 3, /* bfloat16: dense rows and matrices of the routing operations only */
  WS_F16 = 4   /* half:     the same */
} ws_dtype_t;

typedef enum {
  WS_OK = 0,
  WS_ERR_INVALID_ARG = 1, /* NULL handle/pointer, negative size, bad enum        */
  WS_ERR_INVALID_CSR = 2, /* validation found broken CSR invariants              */
  WS_ERR_SHAPE = 3,       /* operand or output shapes do not fit the operation    */
  WS_ERR_DTYPE = 4,       /* A, B and C do not share one value type              */
  WS_ERR_OVERFLOW = 5,    /* a size exceeds what the index types can hold         */
  WS_ERR_ALLOC = 6,       /* device or pinned-host allocation failed             */
  WS_ERR_CUDA = 7,        /* a CUDA runtime call failed                          */
  WS_ERR_DEVICE = 8,      /* a kernel gave up (bounded loop ran out) -- internal  */
  WS_ERR_STATE = 9        /* calls out of order (numeric before symbolic, ...)   */
} ws_status_t;

/*
 * ws_csr_create -- wraps borrowed device CSR arrays in a handle.
 *   out      receives the handle (set to NULL on failure)
 *   nrows, ncols  matrix shape, 0 <= nrows, 0 <= ncols <= INT32_MAX
 *   nnz      number of stored entries (ignored for an output handle, pass 0)
 *   rowptr   int64[nrows + 1] device array (required, also for C: the
 *            symbolic pass writes C's row pointer into it)
 *   colidx   int32[nnz] device array; may be NULL when nnz == 0 or for an
 *            output handle before ws_spgemm_numeric
 *   vals     value array of type dtype; same NULL rule as colidx
 *   dtype    WS_F32 or WS_F64
 *   validate non-zero: check the CSR invariants listed above on the device
 *            (O(nrows + nnz) work, synchronises `stream`); a violation gives
 *            WS_ERR_INVALID_CSR and no handle.  Pass 0 for an output handle.
 *   stream   stream for the validation kernel
 * The handle owns only library scratch (released by ws_csr_destroy).
 * Passage: the compressed-format invariants of Sec. 1 ("Complex Data
 * Structure Invariants": CSR is prefix sums over contiguous buffers) and
 * Sec. 3.1 (position arrays are cumulative sums that must stay monotonically
 * non-decreasing); validation checks exactly those plus sorted, in-range
 * column indices.
 */
ws_status_t ws_csr_create(ws_csr_t* out, int64_t nrows, int64_t ncols, int64_t nnz, int64_t* rowptr,
                          int32_t* colidx, void* vals, ws_dtype_t dtype, int validate,
                          ws_stream_t stream);

/*
 * ws_spgemm_symbolic -- structure pass of C = A * B.
 * Computes, for every row i, the number of distinct columns of
 * sum_k A[i,k] B[k,:], writes C.rowptr (exclusive prefix sum, C.rowptr[0] = 0)
 * into the rowptr array given to C's handle, and returns nnz(C) in *nnz_out
 * (host pointer).  C must be an output handle of shape A.nrows x B.ncols and
 * the same dtype.  Work is queued on `stream`; the call returns after the
 * stream has reached the end of the pass (it synchronises `stream`), because
 * the caller needs nnz(C) to allocate C's arrays.  Independent row kernels of
 * a pass may run side by side on streams of the library that have the
 * priority of `stream`; they start after what `stream` holds and end before
 * what is queued on it later.  While `stream` is being captured,
 * and if it is confined to a part of the GPU (a green context), everything
 * stays on it.  The row plan (row classes,
 * per-row workspaces) is kept in C's handle for ws_spgemm_numeric.
 * Device scratch is allocated stream-ordered on `stream` and cached in C's
 * handle across calls.  The first call on a device sets the release
 * threshold of that device's default stream-ordered memory pool to its
 * maximum, so memory freed by destroyed handles stays in the pool for the
 * next ones (it is returned to the system when the process exits).
 * Passage: Sec. 5.1 (Gustavson's SpGEMM, parallel over output fibers: the
 * count of row i is the number of distinct fibers that row's worker will
 * write under the shard level) and the `declare` step of the lifecycle in
 * Sec. 4 ("Building on Finch": the output is initialised and sized before it
 * is updated).
 */
ws_status_t ws_spgemm_symbolic(ws_csr_t A, ws_csr_t B, ws_csr_t C, int64_t* nnz_out, ws_stream_t stream);

/*
 * ws_spgemm_numeric -- value pass of C = A * B.
 *   c_colidx  device int32[nnz(C)] written with C's column indices
 *   c_vals    device value array [nnz(C)] of C's dtype
 * Requires a completed ws_spgemm_symbolic for the same A, B and C (and A, B
 * unchanged since).  Asynchronous: work is queued on `stream` (row kernels
 * side by side, as in the symbolic pass) and the call
 * returns without waiting; device-side failures are reported by
 * ws_spgemm_wait.  The two arrays are recorded in C's handle.
 * Passage: Sec. 5.1 (Gustavson's loop: w[j] += A[i,k] * B[k,j] in a per-row
 * workspace, then row i of C is written from w in sorted column order) and
 * the `update` -> `freeze` steps of Sec. 4 (the pass updates C's disjoint row
 * segments and leaves C in read mode).
 */
ws_status_t ws_spgemm_numeric(ws_csr_t A, ws_csr_t B, ws_csr_t C, int32_t* c_colidx, void* c_vals,
                              ws_stream_t stream);

/*
 * ws_spgemm_outer_symbolic / ws_spgemm_outer_numeric -- C = A * B as the
 * outer-product SpGEMM (Sec. 5.1, Fig. "SpGEMM implemented in WingSpan",
 * outer product, with the merge level and its coalesce step of Sec. 4): the
 * k range is split into `parts` contiguous blocks K_p; block p contributes the
 * partial product A[:, K_p] * B[K_p, :] (a worker's own copy of C) and the
 * copies are coalesced by pairwise sparse additions.  C's structure equals
 * the row-wise product's (a sum of exactly 0.0 is kept); values agree up to
 * summation order (sums per block, then block sums).
 *   parts  >= 1 (clamped to the number of columns of A; 1 is the row-wise
 *          product itself), else WS_ERR_INVALID_ARG
 * Same two-pass contract as ws_spgemm_symbolic / ws_spgemm_numeric: the
 * symbolic call writes C.rowptr, returns nnz(C) and synchronises `stream`;
 * it computes every block's partial product and every merge except the value
 * pass of the last one, in library-owned scratch allocated stream-ordered on
 * `stream` (B's row blocks are views of B, A's column blocks share one buffer
 * of nnz(A) entries).  The numeric call (asynchronous) writes C's column
 * indices and values and releases that scratch stream-ordered.  A and B must
 * stay unchanged in between.  Errors as for the row-wise calls; a device-side
 * failure in any step gives WS_ERR_DEVICE.
 */
ws_status_t ws_spgemm_outer_symbolic(ws_csr_t A, ws_csr_t B, ws_csr_t C, int parts, int64_t* nnz_out,
                                     ws_stream_t stream);
ws_status_t ws_spgemm_outer_numeric(ws_csr_t A, ws_csr_t B, ws_csr_t C, int32_t* c_colidx, void* c_vals,
                                    ws_stream_t stream);

/* Elementwise operations (Sec. 5.2, "Sparse Linear Algebra": C = A op B). */
typedef enum {
  WS_EWISE_ADD = 1, /* SpAdd: C = A + B on the union of the two patterns            */
  WS_EWISE_MUL = 2  /* Hadamard product: C = A .* B on the intersection of the two */
} ws_ewise_op_t;

/*
 * ws_ewise_symbolic -- structure pass of the elementwise operation C = A op B
 * (Sec. 5.2, "Sparse Linear Algebra", where SpAdd and the Hadamard product
 * use the sharded sparse list: distinct rows of C go to distinct workers).
 *   op   WS_EWISE_ADD: C holds (i, j) iff A or B stores (i, j), with
 *        C[i,j] = A[i,j] + B[i,j] (a missing entry contributes nothing; a sum
 *        of exactly 0.0 is kept);
 *        WS_EWISE_MUL: C holds (i, j) iff both store (i, j), with
 *        C[i,j] = A[i,j] * B[i,j].
 * A and B have the same shape and dtype; C is an output handle of that shape
 * and dtype.  Writes C.rowptr into the rowptr array of C's handle and returns
 * nnz(C) in *nnz_out (host pointer).  Work is queued on `stream` and the call
 * synchronises it (the caller needs nnz(C) to allocate C).  The tile plan
 * (the merged entries of all rows cut into equal tiles) is kept in C's handle
 * for ws_ewise_numeric; device scratch is allocated stream-ordered on
 * `stream` and cached in the handle.  Errors: WS_ERR_SHAPE, WS_ERR_DTYPE,
 * WS_ERR_INVALID_ARG (NULL pointer, unknown op), WS_ERR_DEVICE (a kernel found
 * inconsistent input, e.g. unsorted columns).
 */
ws_status_t ws_ewise_symbolic(ws_csr_t A, ws_csr_t B, ws_csr_t C, int op, int64_t* nnz_out, ws_stream_t stream);

/*
 * ws_ewise_numeric -- value pass of C = A op B.
 *   c_colidx  device int32[nnz(C)] written with C's column indices
 *   c_vals    device value array [nnz(C)] of C's dtype
 * Requires a completed ws_ewise_symbolic for the same A, B and C (A and B
 * unchanged since).  Asynchronous on `stream`; device-side failures are
 * reported by ws_spgemm_wait.  Values are computed in the value type: one
 * rounding per entry.
 */
ws_status_t ws_ewise_numeric(ws_csr_t A, ws_csr_t B, ws_csr_t C, int32_t* c_colidx, void* c_vals,
                             ws_stream_t stream);

/*
 * ws_spmspv -- sparse matrix - sparse vector product y = A x (Sec. 5.2,
 * "Sparse Linear Algebra": SpMSpV, where x's stored entries select columns of
 * A and the columns are accumulated into a sparse byte-map over y that a
 * merge level protects).
 *   At      handle of A^T in CSR, i.e. A by columns: At is n x m for an m x n
 *           A, and row j of At lists the rows i of A's entries in column j
 *           (ascending) with their values
 *   nnz_x   stored entries of x, 0 <= nnz_x <= n
 *   x_idx   device int32[nnz_x], strictly increasing, in [0, n)
 *   x_vals  device values [nnz_x] of At's dtype
 *   y_idx   device int32[m] (capacity m): receives y's indices, increasing
 *   y_vals  device values [m] of At's dtype: receives y's values
 *   nnz_y   host pointer: receives the number of stored entries of y
 * y holds i iff some stored A[i,j] has j stored in x (structural: a sum of
 * exactly 0.0 is kept), y[i] = sum of A[i,j] x[j] accumulated in the value
 * type in unspecified order.  Work is queued on `stream` and the call
 * synchronises it (to return nnz_y).  Device scratch (an accumulator and a
 * byte-map of length m, offsets per x entry) is allocated stream-ordered and
 * cached in At's handle.  Errors: WS_ERR_INVALID_ARG (NULL pointers, nnz_x out
 * of range), WS_ERR_DEVICE (an index of x or of At out of range: those entries
 * are skipped and flagged).
 */
ws_status_t ws_spmspv(ws_csr_t At, int64_t nnz_x, const int32_t* x_idx, const void* x_vals, int32_t* y_idx,
                      void* y_vals, int64_t* nnz_y, ws_stream_t stream);

/*
 * ws_csr_submatrix_symbolic / ws_csr_submatrix_numeric -- S = A[r0:r1, c0:c1]
 * as a CSR matrix of shape (r1 - r0) x (c1 - c0) with columns shifted by -c0.
 * This is the layout step of the outer-product SpGEMM (Sec. 5.1, Fig.
 * "SpGEMM implemented in WingSpan": the k loop split over workers, worker p
 * multiplying the column block A[:, K_p] by the row block B[K_p, :] into its
 * own copy of C before a merge level coalesces the copies).
 *   0 <= r0 <= r1 <= A.nrows, 0 <= c0 <= c1 <= A.ncols (else WS_ERR_INVALID_ARG)
 *   S   output handle of shape (r1 - r0) x (c1 - c0) and A's dtype
 * The symbolic call writes S.rowptr and returns nnz(S) (it synchronises
 * `stream`); the numeric call (asynchronous) fills the caller's s_colidx
 * (int32[nnz(S)]) and s_vals from the same A, unchanged in between.
 */
ws_status_t ws_csr_submatrix_symbolic(ws_csr_t A, int64_t r0, int64_t r1, int64_t c0, int64_t c1, ws_csr_t S,
                                      int64_t* nnz_out, ws_stream_t stream);
ws_status_t ws_csr_submatrix_numeric(ws_csr_t A, ws_csr_t S, int32_t* s_colidx, void* s_vals, ws_stream_t stream);

/*
 * ws_spgemm_wait -- synchronises `stream` and returns the device status
 * recorded by the last symbolic/numeric pass of C (WS_OK if none failed);
 * serves the elementwise passes too.
 */
ws_status_t ws_spgemm_wait(ws_csr_t C, ws_stream_t stream);

/*
 * ws_csr_destroy -- releases the handle and the scratch it owns (never the
 * borrowed arrays).  NULL-safe.  Synchronises the handle's device (whichever
 * is current) if the handle owns scratch, so pending work that uses it completes
 * first.  Scratch of up to 32 MiB is kept for the next handles of the device, of
 * up to eight handles in the process; other device scratch goes back to the
 * stream-ordered pool and the pinned host summary to a process-wide free list.
 * Passage: the end of the lifecycle of Sec. 4 ("Building on Finch"): once C is
 * frozen, the workspaces the passes declared are no longer needed.  The
 * paper has no explicit release call; this one frees the library's share.
 */
ws_status_t ws_csr_destroy(ws_csr_t handle);

/* Short static description of a status code. */
const char* ws_status_string(ws_status_t status);

/* One-line description of the most recent failure on the calling thread ("" if none). */
const char* ws_last_error(void);

/*
 * ws_csr_nnz -- number of entries of a handle (for C: nnz(C) after symbolic,
 * -1 before).  Returns WS_ERR_INVALID_ARG for a NULL handle or pointer.
 */
ws_status_t ws_csr_nnz(ws_csr_t handle, int64_t* nnz_out);

/*
 * ws_spgemm_plan_info -- counts from the last symbolic pass of C, for
 * diagnostics and tests: info[0] empty rows, info[1] single-entry (direct
 * copy) rows, info[2] hash rows, info[3] hash rows ranked by a sort,
 * info[4] dense-window rows, info[5] dense-window slices,
 * info[6] total products (sum over rows of the product count),
 * info[7] number of kernel launches queued by the last symbolic pass,
 * info[8] number queued by the last numeric pass, info[9] bitmap rows,
 * info[10] heavy rows on the dense path (value windows), info[11] heavy rows
 * on the wide-bitmap path.
 * `n` is the length of `info` (at most 12 values are written).
 */
ws_status_t ws_spgemm_plan_info(ws_csr_t C, int64_t* info, int n);

/*
 * ws_set_tuning -- test/diagnostic knob, process-wide.
 *   key 1: largest product count of a row that uses the shared-memory hash
 *          path (default 4096; smaller values send more rows to the
 *          dense-window path, 0 sends every multi-entry row there)
 *   key 2: most products a bucket of a hash row may hold (default 63; a row
 *          with a fuller bucket is sorted; smaller values send more rows
 *          there, larger ones, up to 4096, act as 63)
 *   key 3: dense-window slice width in columns (default 8192 for double,
 *          16384 for float; must be a multiple of 1024, 0 = default)
 *   key 4: widest column range of a row that uses the bitmap path
 *          (default and maximum 65536; 0 disables the bitmap path)
 *   key 5: most stored A entries of a row that uses the one-warp register
 *          bitmap path (default and maximum 16; 0 disables that path)
 *   key 6: most stored A entries of a heavy row that uses the dense
 *          path (value windows) (default and maximum 8192; 0 disables it)
 *   key 7: widest column range of a heavy row that uses the wide-bitmap path
 *          (default and maximum 1048576; 0 disables it)
 *   key 8 (-1, 0, 1, 2, 4, 8, 16, 32 or 64; default -1) and key 9 ([2,
 *          1048576]; default 64): accepted, without effect (the elementwise
 *          operations once had several paths; they have one)
 *   key 10: most bytes that the ranks of hash rows, the bitmaps of dense heavy
 *          rows and those of wide heavy rows may each take between the passes
 *          (default and maximum 2^32; beyond it the numeric pass works them
 *          out again, dense heavy rows in batches of at least 1024)
 * Returns WS_ERR_INVALID_ARG for an unknown key or out-of-range value.
 */
ws_status_t ws_set_tuning(int key, int64_t value);

/*
 * ws_rowptr_scan_static -- builds a CSR row pointer from per-row counts
 * without allocating any memory.  (The paper has no counterpart: this is a
 * service for callers of this library that cannot allocate device memory at
 * this point, for example code inside a framework that owns all device
 * memory and forbids outside allocations, or a latency-critical loop where
 * cudaMalloc/cudaFree would block on the whole device.)
 *   rowptr  device int64[nrows + 1]; on entry rowptr[i + 1] holds the entry
 *           count of row i (rowptr[0] is ignored); on exit rowptr[0] = 0 and
 *           rowptr[i + 1] = rowptr[i] + count_i, so rowptr[nrows] = nnz.
 *   nrows   0 <= nrows <= 16,777,216 (the fixed scratch holds one partial
 *           sum per 4096 rows); larger values return WS_ERR_OVERFLOW.
 *   stream  the work is queued on it; the call does not wait.
 * Scratch lives in a fixed array compiled into the library (about 33 KB),
 * which every GPU that loads the library keeps until the process exits.  The
 * call itself calls no cudaMalloc, cudaFree or other allocating routine.
 * The first call on a device looks up that array's device address and
 * keeps it for the life of the process; make that first call before any
 * stream capture, and do not call this function again on a device after
 * cudaDeviceReset (or anything else that destroys the device's primary
 * context), because the kept address then names freed memory.  All calls
 * share the array:
 * calls that may run at the same time on the GPU (on unordered streams) race
 * and give wrong results.  Returns WS_ERR_INVALID_ARG for a NULL rowptr or a
 * negative nrows, WS_ERR_CUDA if a CUDA call fails.
 */
ws_status_t ws_rowptr_scan_static(int64_t* rowptr, int64_t nrows, ws_stream_t stream);

/*
 * Routing matrices.  An nrows x ncols CSR matrix R with a row per token and a
 * column per expert (or adapter), float values, few entries a row.  (The paper
 * has no counterpart: these calls serve layers that send rows of dense
 * matrices along a sparse matrix.)  The calls below take device pointers, queue
 * their work on `stream` and return without waiting; they allocate nothing
 * and can be captured in a graph.  Argument errors are found on the host
 * before anything is queued.  Dense matrices are row-major with unit stride
 * within a row and `ld` values from row to row.  ncols <= 1024, nrows, nnz and
 * the number of dense rows <= INT32_MAX, rows of at most 2^24 values.
 * Entries whose column is not in [0, ncols), and those before rowptr[0] and from
 * rowptr[nrows] on, take no part: they have slot -1 and gradient 0, and the
 * slots they leave over come last and hold zero rows.
 * rowptr is read within [0, nnz] whatever it holds: where it decreases results
 * are unspecified, but nothing outside the arrays is read or written, and
 * offsets never exceed nnz.
 *
 * ws_topk_route -- R from logits (rows x cols, float, bfloat16 or half): row i
 * holds the k largest logits of row i (ties to the lowest column), by
 * ascending column, with the weights exp(l - max) / sum of exp(l - max), the sum over the k chosen
 * (normalize != 0) or over all columns (0), in 32 bits.  A logit of -inf has
 * weight 0 and is chosen last; a row of nothing else has weights 0.  NaN counts
 * as the largest value and makes the row's weights NaN.  Writes rowptr
 * (int64[rows + 1] = 0, k, 2 k, ...), colidx and vals ([rows * k]).
 * 1 <= k <= min(cols, 32), cols <= 1024.
 *
 * ws_topk_route_backward -- gradient of the logits (rows x cols, their type,
 * row stride ldg) from the gradient gvals of vals; colidx and vals as
 * ws_topk_route wrote them.  The choice of columns counts as fixed.  logits
 * are read only where normalize is 0 (may be NULL otherwise).
 */
ws_status_t ws_topk_route(const void* logits, int64_t rows, int64_t cols, int64_t ld, ws_dtype_t dtype, int k,
                          int normalize, int64_t* rowptr, int32_t* colidx, float* vals, ws_stream_t stream);
ws_status_t ws_topk_route_backward(const void* logits, int64_t rows, int64_t cols, int64_t ld, ws_dtype_t dtype,
                                   int k, int normalize, const int32_t* colidx, const float* vals,
                                   const float* gvals, void* glogits, int64_t ldg, ws_stream_t stream);

/* A routing matrix and its transpose: all arrays are the caller's. */
typedef struct ws_routing {
  int64_t nrows, ncols, nnz;
  const int64_t* rowptr; /* [nrows + 1] */
  const int32_t* colidx; /* [nnz], strictly increasing within a row */
  const float* vals;     /* [nnz]; read by combine and its gradient only */
  int64_t* offsets;      /* [ncols + 1]: first slot of every column (the row pointer of R^T) */
  int32_t* rows;         /* [nnz]: row of every slot (the columns of R^T, ascending within a column) */
  int32_t* entries;      /* [nnz]: entry of R in every slot */
  int32_t* slots;        /* [nnz]: slot of every entry of R */
  int32_t* status;       /* [1]: cleared by ws_routing_build; nonzero after a product whose bounded waits ran out */
} ws_routing;

/*
 * ws_routing_build -- fills offsets, rows, entries and slots: the entries of R
 * sorted by column, rows in order within a column.  `scratch` holds
 * ws_routing_scratch(nrows, ncols) bytes, 16-byte aligned (0 for few rows: NULL
 * then; -1 if the device cannot be asked, with the reason in ws_last_error).
 */
int64_t ws_routing_scratch(int64_t nrows, int64_t ncols);
ws_status_t ws_routing_build(const ws_routing* r, void* scratch, int64_t scratch_bytes, ws_stream_t stream);

/*
 * Dense rows along R, each row `width` values of `dtype` (float, bfloat16, half):
 *   dispatch           xs[slot] = x[row]                     x: nrows rows, xs: nnz rows in slot order
 *   dispatch_backward  gx[i] = sum over row i of gxs[slot]
 *   combine            y[i] = sum over row i of value * ys[slot]
 *   combine_backward   gys[slot] = value * gy[row],  gvals[entry] = <gy[row], ys[slot]>
 * Sums are held in 32 bits, in the order of the entries, and rounded once; rows
 * of R without entries give zero rows.  Outputs may not overlap inputs.
 */
ws_status_t ws_routing_dispatch(const ws_routing* r, const void* x, int64_t ldx, void* xs, int64_t ldxs,
                                int64_t width, ws_dtype_t dtype, ws_stream_t stream);
ws_status_t ws_routing_dispatch_backward(const ws_routing* r, const void* gxs, int64_t ldgxs, void* gx, int64_t ldgx,
                                         int64_t width, ws_dtype_t dtype, ws_stream_t stream);
ws_status_t ws_routing_combine(const ws_routing* r, const void* ys, int64_t ldys, void* y, int64_t ldy,
                               int64_t width, ws_dtype_t dtype, ws_stream_t stream);
ws_status_t ws_routing_combine_backward(const ws_routing* r, const void* gy, int64_t ldgy, const void* ys,
                                        int64_t ldys, void* gys, int64_t ldgys, float* gvals, int64_t width,
                                        ws_dtype_t dtype, ws_stream_t stream);

/*
 * Products by column of R: column e has a matrix W[e], N x K, row-major (ldw
 * values from row to row, `stride` from matrix to matrix), and the rows of its
 * slots.  bfloat16 or half, sums in 32 bits, one rounding.
 *   matmul            ys[s] = W[e] xs[s]                     xs: nnz x K, ys: nnz x N
 *   matmul_backward   gxs[s] = W[e]^T gys[s]                 gys: nnz x N, gxs: nnz x K; NULL: not wanted, W is not read
 *                     gW[e] = sum over s of gys[s] xs[s]^T   zero for columns without entries; NULL: not wanted, xs is not read
 * Rows behind the placed entries are zero (ys, gxs).  N, K <= 2^24.
 * An input whose address or strides are not multiples of 16 bytes is first
 * copied to `scratch` (16-byte aligned), which has to have room for 16 bytes for every 8 values, or part of
 * them, of its rows; scratch may be NULL where all inputs are aligned.
 */
ws_status_t ws_routing_matmul(const ws_routing* r, const void* xs, int64_t ldxs, const void* W, int64_t ldw,
                              int64_t stride, int64_t N, int64_t K, void* ys, int64_t ldys, ws_dtype_t dtype,
                              void* scratch, int64_t scratch_bytes, ws_stream_t stream);
ws_status_t ws_routing_matmul_backward(const ws_routing* r, const void* gys, int64_t ldgys, const void* xs, int64_t ldxs,
                                       const void* W, int64_t ldw, int64_t stride, int64_t N, int64_t K, void* gxs,
                                       int64_t ldgxs, void* gW, int64_t ldgw, int64_t gstride, ws_dtype_t dtype,
                                       void* scratch, int64_t scratch_bytes, ws_stream_t stream);

/*
 * Products by column of R with an epilogue, in one kernel: the sums are held in 32 bits, and so is what follows, rounded once.
 *   linear   ys[s] = act(z) + residual[s],   z = W[e] xs[s] + bias[e]               W[e]: N x K
 *   gated    h[s]  = act(gate) * up,         gate = Wg[e] xs[s] + bg[e],  up = Wu[e] xs[s] + bu[e]   Wg[e], Wu[e]: F x K
 * bfloat16 or half, biases (one row an expert) and residual (rows in slot order) in the same type.  bias, bg, bu, residual may be NULL
 * (none).  z, or gate and up, receive the sums rounded to that type, for the backward calls; NULL: not wanted.
 * act: WS_ACT_NONE is z itself, a gated block's gate too; silu = z / (1 + exp(-z)), gelu = z (1 + erf(z / sqrt 2)) / 2, gelu_tanh its form
 * with tanh, the derivative of relu at 0 is 0.
 * At infinities values and derivatives are the limits; values below 2^-119 and derivatives below 2^-118 may be 0.
 * Backward, from gys or gh and the kept sums:
 *   linear   gz = gys act'(z);  gxs[s] = W[e]^T gz[s],  gW[e] = sum of gz[s] xs[s]^T,  gbias[e] = sum of gz[s]   (residual: gys)
 *   gated    dg = gh up act'(gate), du = gh act(gate);  gxs[s] = Wg[e]^T dg[s] + Wu[e]^T du[s],  gWg, gWu, gbg, gbu likewise
 * z may be NULL where act is WS_ACT_NONE.  Each of gxs, gW, gbias, gWg, gWu, gbg, gbu may be NULL: not wanted.  gz, dg and du are rounded to
 * the rows' type before they are multiplied; the biases' gradients are summed before that, in a fixed order.  Columns without
 * entries have gradients 0.  Rows behind the placed entries are zero in ys, z, h, gate, up and gxs.
 * Strides, limits and scratch are those of ws_routing_matmul: 16 bytes for every 8 values, or part of them, of the rows of each of xs, the
 * matrices and, in linear_backward where act is WS_ACT_NONE, gys, whose address or strides are not multiples of 16 bytes; the
 * backward calls need their _scratch besides (-1: a size is negative).  Outputs may overlap no input.
 */
typedef enum ws_act {
  WS_ACT_NONE = 0,
  WS_ACT_RELU = 1,
  WS_ACT_SILU = 2,
  WS_ACT_GELU = 3,
  WS_ACT_GELU_TANH = 4,
  WS_ACT_SIGMOID = 5
} ws_act_t;

typedef struct ws_linear_call {
  int64_t N, K;
  const void* xs;
  int64_t ldxs;
  const void* W;
  int64_t ldw, stride;
  const void* bias;
  int64_t ldbias;
  const void* residual;
  int64_t ldresidual;
  void* ys;
  int64_t ldys;
  void* z;
  int64_t ldz;
  ws_dtype_t dtype;
  ws_act_t act;
} ws_linear_call;

typedef struct ws_linear_backward_call {
  int64_t N, K;
  const void* gys;
  int64_t ldgys;
  const void* z;
  int64_t ldz;
  const void* xs;
  int64_t ldxs;
  const void* W;
  int64_t ldw, stride;
  void* gxs;
  int64_t ldgxs;
  void* gW;
  int64_t ldgw, gstride;
  void* gbias;
  int64_t ldgbias;
  ws_dtype_t dtype;
  ws_act_t act;
} ws_linear_backward_call;

typedef struct ws_gated_call {
  int64_t F, K;
  const void* xs;
  int64_t ldxs;
  const void* Wg;
  int64_t ldwg, strideg;
  const void* Wu;
  int64_t ldwu, strideu;
  const void* bg;
  int64_t ldbg;
  const void* bu;
  int64_t ldbu;
  void* h;
  int64_t ldh;
  void* gate;
  int64_t ldgate;
  void* up;
  int64_t ldup;
  ws_dtype_t dtype;
  ws_act_t act;
} ws_gated_call;

typedef struct ws_gated_backward_call {
  int64_t F, K;
  const void* gh;
  int64_t ldgh;
  const void* gate;
  int64_t ldgate;
  const void* up;
  int64_t ldup;
  const void* xs;
  int64_t ldxs;
  const void* Wg;
  int64_t ldwg, strideg;
  const void* Wu;
  int64_t ldwu, strideu;
  void* gxs;
  int64_t ldgxs;
  void* gWg;
  int64_t ldgwg, gstrideg;
  void* gWu;
  int64_t ldgwu, gstrideu;
  void* gbg;
  int64_t ldgbg;
  void* gbu;
  int64_t ldgbu;
  ws_dtype_t dtype;
  ws_act_t act;
} ws_gated_backward_call;

ws_status_t ws_routing_linear(const ws_routing* r, const ws_linear_call* call, void* scratch, int64_t scratch_bytes, ws_stream_t stream);
int64_t ws_routing_linear_backward_scratch(int64_t nnz, int64_t ncols, int64_t N, ws_act_t act, int bias);
ws_status_t ws_routing_linear_backward(const ws_routing* r, const ws_linear_backward_call* call, void* scratch, int64_t scratch_bytes,
                                       ws_stream_t stream);
ws_status_t ws_routing_gated(const ws_routing* r, const ws_gated_call* call, void* scratch, int64_t scratch_bytes, ws_stream_t stream);
int64_t ws_routing_gated_backward_scratch(int64_t nnz, int64_t ncols, int64_t F, int bias);
ws_status_t ws_routing_gated_backward(const ws_routing* r, const ws_gated_backward_call* call, void* scratch, int64_t scratch_bytes,
                                      ws_stream_t stream);

/*
 * ws_adapters -- low-rank adapters of many requests beside a projection they
 * share: y[t] = base[t] + sum over row t of S of value * B[a] (A[a] x[t]).
 * S is an nrows x ncols CSR matrix, tokens x adapters (columns strictly
 * increasing within a row; rows may be empty; entries whose column is out of
 * range take no part).  bfloat16 or half; inner products A[a] x[t] are summed in
 * 32 bits, for many tokens kept, times the value, as pairs of 16-bit values
 * (bfloat16: 16 significant bits; half: off by 2^-23 of them and at most 2^-25 of
 * the largest of 32 ranks of the token, over the range of floats), the result is
 * summed in 32 bits and rounded once.  "Many tokens": ws_adapters_many(nrows, r)
 * is not 0.  base may be NULL (zero) and may be y itself; y may overlap no other input.
 * `scratch` holds ws_adapters_scratch(nnz, r) bytes, 16-byte aligned, and for
 * many tokens 16 bytes more for every 8 values, or part of them, of the rows of
 * each of x, A and B whose address or strides are not multiples of 16 bytes.  For
 * many tokens its first int is 0 after the call, or nonzero if a kernel's bounded
 * waits ran out.  Queued on `stream`; nothing is allocated.
 */
typedef struct ws_adapters_call {
  int64_t nrows, ncols, nnz;
  const int64_t* rowptr;
  const int32_t* colidx;
  const float* vals;
  int64_t K, r, N; /* A[a]: r x K, B[a]: N x r */
  const void* x;
  int64_t ldx;
  const void* A;
  int64_t lda, strideA;
  const void* B;
  int64_t ldb, strideB;
  const void* base;
  int64_t ldbase;
  void* y;
  int64_t ldy;
  ws_dtype_t dtype;
} ws_adapters_call;

int64_t ws_adapters_scratch(int64_t nnz, int64_t r);
int ws_adapters_many(int64_t nrows, int64_t r);
ws_status_t ws_adapters(const ws_adapters_call* call, void* scratch, int64_t scratch_bytes, ws_stream_t stream);

/*
 * ws_adamw -- one AdamW step over `count` tensors, those whose gradient is not NULL.  For every value, t = steps done + 1:
 *   g = grad * scale;  m' = beta1 m + (1 - beta1) g;  v' = beta2 v + (1 - beta2) g^2;
 *   p' = p (1 - lr decay) - lr / (1 - beta1^t) * m' / (sqrt(v' / (1 - beta2^t)) + eps);  copy = p' rounded to 16 bits.
 * p: float[n], in place.  grads: `count` arrays of grad_dtype (float, bfloat16, half).  copy: copy_dtype (bfloat16 or half), or
 * NULL.  All arithmetic is in 32 bits.  eps: 0, or at least 2^-126.
 * bits 32: m, v float[n]; m_scale, v_scale are not read.
 * bits 8: m, v uint8[n], e4m3 codes of m and of r = sqrt(v); m_scale, v_scale float[(n + 255) / 256], the scales of blocks of 256
 * values: the largest magnitude / 448, 0 below 1e-30.  Codes are rounded up with their share of the way to the next one as
 * probability, by a hash of seed, step, the tensor's index and the value's: equal inputs give equal bits.  A root above zero (2^-63 and
 * above) has no code of zero; smaller ones count as 0, so that eps has to be at least 1e-15.  Infinities and NaN become NaN and stay with
 * their value.
 * step: int64[1] on the device, steps done, one count for all tensors, whether they had a gradient in every step or not: the call adds one.
 * done: int32[1] on the device, 0 between calls.  lr_at, scale, skip: one value on the device, read when the step runs (NULL: lr, 1, 0);
 * where *skip is not 0 nothing changes, steps done neither.  Tensors may overlap neither one another nor the gradients.
 * tensors and grads are read before the call returns.  Calls with the same tensors or step array must not overlap on the GPU.
 */
typedef struct ws_adamw_tensor {
  void* p;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
  float decay;
} ws_adamw_tensor;

typedef struct ws_adamw_call {
  const ws_adamw_tensor* tensors;
  const void* const* grads;
  int64_t count;
  int64_t* step;
  int32_t* done;
  const float* lr_at;
  const float* scale;
  const int32_t* skip;
  double lr, beta1, beta2, eps;
  uint32_t seed;
  int bits;
  ws_dtype_t grad_dtype, copy_dtype;
} ws_adamw_call;

ws_status_t ws_adamw(const ws_adamw_call* call, ws_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WS_SPGEMM_H */
