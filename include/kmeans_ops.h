/*
 * kmeans_ops.h -- C ABI of the operators of a layer conditioned on clusters
 * (MI355X, gfx950), in libkmeans_mti.so beside kmeans_mti.h.
 *
 * The assignment that k-means gives every row routes the rows of a model
 * (tokens, embeddings) to small experts of their clusters.  The operators:
 *   kmeans_sort_*     rows sorted by cluster and back with weights, and the
 *                     gradients of both;
 *   kmeans_norm_*     layer norm of rows and its gradients;
 *   kmeans_adapter_*  a shared projection with one low-rank adapter per
 *                     cluster, and the gradients of rows and adapters;
 *   kmeans_linear_*   products with one weight per cluster, and the gradients
 *                     of rows and weights;
 *   kmeans_fp8_*      rows in 8-bit floating point with a scale for each 128
 *                     elements, and products of them with one weight per
 *                     cluster;
 *   kmeans_table_*    rows of a table by their ids, and the table's gradient;
 *   kmeans_clip_*     the norm over many tensors, and scaling them to a limit.
 *
 * Common to all.  Status codes and kmeans_mti_last_hip_error() are those of
 * kmeans_mti.h; no entry point throws, allocates device memory or
 * synchronizes, and all may be recorded into a HIP graph.  Device work is
 * ordered on hip_stream (NULL = the null stream).  All array arguments are
 * DEVICE pointers on the current device; a pointer may be NULL where its
 * array is empty.  Rows are `d` contiguous elements, `ld` elements apart
 * (ld >= d) where an argument ld* is given, else d apart.  Outputs must not
 * overlap inputs (kmeans_clip_norm may work in place).  Rows have at most 2^28
 * elements.  Workspaces are the caller's: device memory of at least the bytes
 * that the *_workspace_bytes function gives, 256-byte aligned, contents on entry
 * of no matter, not to be used by another call until this one's work completes.
 * Sums, statistics and gradients are formed in float32 and rounded once to the type
 * of the output (kmeans_fp8_forward says what its results of 16 bits keep); equal
 * inputs give bitwise equal outputs.
 */
#ifndef KMEANS_OPS_H
#define KMEANS_OPS_H

#include "kmeans_mti.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of rows. */
enum { KM_F32 = 0, KM_BF16 = 1, KM_F16 = 2 };
/* e4m3 values (1 sign, 4 exponent, 3 mantissa bits, largest 448, one NaN): kmeans_fp8_forward alone. */
enum { KM_E4M3 = 3 };

/*
 * The plan that sorts rows by cluster.  ids: n x m int32, row i's m clusters
 * (m = 1: the assignment of kmeans_mti_run); slot p = i * m + j.  A slot
 * whose id is outside [0, k) is empty.
 *   order      n m int32: the slots by (cluster, slot), empty slots last in
 *              slot order; place s of the sorted rows holds slot order[s]
 *   pos        n x m int32: the inverse, order[pos[p]] = p
 *   sorted_ids n m int32: the cluster of every place, -1 for empty slots
 *   offsets    k + 1 int32: cluster c has places offsets[c] .. offsets[c+1];
 *              offsets[k] = slots in use
 * Requires n >= 0, m >= 1, k >= 1, n m < 2^31.
 */
size_t kmeans_sort_workspace_bytes(int64_t n, int32_t m, int32_t k);   /* 0 for bad sizes */
int kmeans_sort_plan(const int32_t* ids, int64_t n, int32_t m, int32_t k, int32_t* order, int32_t* pos,
                     int32_t* sorted_ids, int32_t* offsets, void* workspace, size_t workspace_bytes,
                     void* hip_stream);

/*
 * Xs[s] = X[order[s] / m] (n m rows; zero rows for empty slots), from pos and
 * offsets of a plan of (n, m, k).  type: KM_F32, KM_BF16 or KM_F16.  Its
 * gradient is kmeans_sort_combine of dXs with w = NULL.
 */
int kmeans_sort_gather(const void* X, int64_t ldx, int64_t n, int32_t m, int32_t k, int32_t d, int32_t type,
                       const int32_t* pos, const int32_t* offsets, void* Xs, void* hip_stream);

/*
 * Y[i] = sum over row i's slots in use of w[i,j] Z[pos[i,j]], j ascending (a
 * row with none: zero).  Z: n m sorted rows; w: n x m float32 or NULL (ones).
 * Rows of Z and weights of empty slots are not read.
 */
int kmeans_sort_combine(const void* Z, int64_t ldz, int64_t n, int32_t m, int32_t k, int32_t d, int32_t type,
                        const int32_t* pos, const int32_t* offsets, const float* w, void* Y, void* hip_stream);

/*
 * Gradients of kmeans_sort_combine: dZ[pos[i,j]] = w[i,j] dY[i] (n m rows,
 * zero rows for empty slots) and, if dw is not NULL, dw[i,j] =
 * <dY[i], Z[pos[i,j]]> (n x m float32, 0 for empty slots).  Z may be NULL
 * with dw.
 */
int kmeans_sort_combine_backward(const void* dY, int64_t lddy, const void* Z, int64_t ldz, int64_t n, int32_t m,
                                 int32_t k, int32_t d, int32_t type, const int32_t* pos, const int32_t* offsets,
                                 const float* w, void* dZ, float* dw, void* hip_stream);

/*
 * Layer norm: y = (x - mu) rs gamma + beta for every row, mu its mean, rs =
 * 1 / sqrt(v + eps), v its mean square deviation.  gamma, beta: d values or
 * NULL (ones, zeros), float32 if param_f32 is not 0, else of the rows' type.
 * Y: n x d of the rows' type; mean, rstd: n float32.  Requires n >= 0,
 * d >= 1, eps >= 0.
 */
int kmeans_norm_forward(const void* X, int64_t ldx, int64_t n, int32_t d, int32_t type, const void* gamma,
                        const void* beta, int32_t param_f32, float eps, void* Y, float* mean, float* rstd,
                        void* hip_stream);

/*
 * Gradients of kmeans_norm_forward from dY, X and its mean and rstd: dX
 * (n x d of the rows' type), dgamma and dbeta (d float32; either may be NULL;
 * zeros for n = 0).
 */
size_t kmeans_norm_workspace_bytes(int64_t n, int32_t d, int32_t type);   /* 0 for bad sizes */
int kmeans_norm_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, int64_t n, int32_t d,
                         int32_t type, const float* mean, const float* rstd, const void* gamma, int32_t param_f32,
                         void* dX, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

/*
 * A shared projection with one low-rank adapter per cluster: for every row x
 * of cluster c
 *   h = A_c x,  y = W x + scale_c B_c h;
 * a row whose id is outside [0, k) has h = 0 and y = W x.
 *   X      n rows of din, ldx apart      W  dout x din
 *   A      k x r x din                   B  k x dout x r
 *   scale  k float32 or NULL (ones)
 *   Y      n x dout                      H  n x r (for the backward pass)
 * all of one type; the result H is h rounded to it, scale_c h keeps its float32
 * value into the second product (to 2^-16 of it in bfloat16 and 2^-22 in
 * float16, whose range it may leave).  The clusters come as
 *   ids    n int32, with sorted_ids = offsets = order = NULL: the rows are
 *          sorted in the workspace where the form for many rows takes them;
 *   or a plan of kmeans_sort_plan with n slots (ids is not read): sorted_ids,
 *          offsets and order (m = 1), or order = NULL for rows that are in
 *          the plan's order already (the output of kmeans_sort_gather).
 * Requires n >= 0, din, dout, k, r >= 1; KM_ERR_UNSUPPORTED beyond r = 128,
 * n = 2^27 and din, dout = 2^24.  backward: the workspace of the backward
 * pass, else of the forward pass.
 */
size_t kmeans_adapter_workspace_bytes(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type,
                                      int32_t backward);   /* 0 for bad sizes */

/*
 * The form that the shared product of such a call takes where its rows and
 * weights can be read 16 bytes at a time: tiles of *tile x *tile results (256,
 * 128 or 64; 0: the form for few rows), the contraction in *splits parts.
 * Returns KM_OK, or KM_ERR_* for bad sizes.
 */
int kmeans_adapter_tile(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type, int32_t backward,
                        int32_t* tile, int32_t* splits);

int kmeans_adapter_forward(const void* X, int64_t ldx, int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r,
                           int32_t type, const void* W, const void* A, const void* B, const float* scale,
                           const int32_t* ids, const int32_t* order, const int32_t* sorted_ids,
                           const int32_t* offsets, void* Y, void* H, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/*
 * Gradients of kmeans_adapter_forward from dY (n rows of dout), X and H, with
 * a plan (as above, order or rows in its order):
 *   g = scale_c B_c^T dy,  dX = W^T dy + A_c^T g  (n x din),
 *   dA_c = sum g x^T  (k x r x din),  dB_c = scale_c sum dy h^T  (k x dout x r)
 * over the rows of each cluster (zeros for a cluster with none), all of the
 * rows' type; g keeps its float32 value as scale_c h does, and h is H as it is
 * given, rounded as a stored activation is.  W has no gradient here: it is frozen
 * where adapters are trained.
 */
int kmeans_adapter_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, const void* H, int64_t n,
                            int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type, const void* W,
                            const void* A, const void* B, const float* scale, const int32_t* order,
                            const int32_t* sorted_ids, const int32_t* offsets, void* dX, void* dA, void* dB,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Products with one weight per cluster: y = W_c x for every row x of cluster c,
 * zeros for a row of no cluster.
 *   X  n rows of din, ldx apart     W  k x dout x din     Y  n x dout
 * all of one type.  The clusters come as a plan of kmeans_sort_plan with n
 * slots: sorted_ids, offsets and order (m = 1), or order = NULL for rows that
 * are in the plan's order already.  Requires n >= 0, din, dout, k >= 1;
 * KM_ERR_UNSUPPORTED beyond n = 2^27, din, dout = 2^24 and some 2^31 tiles of 64
 * rows and columns.  backward: the workspace of the backward pass, else of the
 * forward pass.
 */
size_t kmeans_linear_workspace_bytes(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t type,
                                     int32_t backward);   /* 0 for bad sizes */
int kmeans_linear_forward(const void* X, int64_t ldx, int64_t n, int32_t din, int32_t dout, int32_t k, int32_t type,
                          const void* W, const int32_t* order, const int32_t* sorted_ids, const int32_t* offsets,
                          void* Y, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradients of kmeans_linear_forward from dY (n rows of dout): dX = W_c^T dy
 * (n x din, zeros for a row of no cluster) and dW_c = sum dy x^T over the
 * cluster's rows (k x dout x din, zeros for a cluster with none).  Either may be
 * NULL; X is read for dW alone, W for dX alone.
 */
int kmeans_linear_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, int64_t n, int32_t din,
                           int32_t dout, int32_t k, int32_t type, const void* W, const int32_t* order,
                           const int32_t* offsets, void* dX, void* dW, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/*
 * Rows in 8-bit floating point.  Of each 128 elements of a row (the last ones
 * fewer), a being the largest finite magnitude: e = max(-126, the least whole
 * number with a <= 448 2^e), exponents = e + 127 (n x ceil(d / 128) bytes),
 * values = x 2^-e rounded to the nearest e4m3 value, ties to even (n x d
 * bytes); infinities and NaN become NaN.  dequantize: X = values 2^e, rounded to
 * its type.  An exponent byte of 255, which quantize never writes, stands for NaN
 * in all of its elements.  Requires 0 <= n <= 2^40, d >= 1.
 */
int kmeans_fp8_quantize(const void* X, int64_t ldx, int64_t n, int32_t d, int32_t type, void* values,
                        uint8_t* exponents, void* hip_stream);
int kmeans_fp8_dequantize(const void* values, const uint8_t* exponents, int64_t n, int32_t d, int32_t type, void* X,
                          void* hip_stream);

/*
 * kmeans_linear_forward with both operands in 8 bits: y = sum of the products of
 * the values that they stand for, rounded to y_type (KM_F32, KM_BF16 or KM_F16).
 * Sums: for KM_F32 all float32.  For KM_BF16 and KM_F16 the products of each 8
 * consecutive elements (from a multiple of 8 on) are aligned to the one of the
 * largest exponent, and what lies more than 13 bits below it is dropped: less than
 * 2^-10 2^m of the 8 together, m being the largest sum of two values' exponents
 * (their powers of two counted; an e4m3 value below 2^-6 has that exponent); these sums
 * of 8 are added in float32.  That is below a bfloat16 result's own rounding where
 * products do not cancel, but may be two of a float16 one's: for float32 sums take
 * KM_F32 and round its results.  W: k x dout x din values with k x dout x ceil(din / 128)
 * exponents.  X: of type KM_E4M3 with its exponents (n x ceil(din / 128) bytes),
 * or of another type with exponents = NULL: quantised in the workspace.
 */
size_t kmeans_fp8_workspace_bytes(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t type);   /* 0 for bad sizes */
int kmeans_fp8_forward(const void* X, int64_t ldx, const uint8_t* exponents, int64_t n, int32_t din, int32_t dout,
                       int32_t k, int32_t type, const void* W, const uint8_t* w_exponents, const int32_t* order,
                       const int32_t* sorted_ids, const int32_t* offsets, void* Y, int32_t y_type, void* workspace,
                       size_t workspace_bytes, void* hip_stream);

/*
 * Rows of a table by their ids: Y[i] = scale table[ids[i]] (n x d), zeros for an
 * id outside [0, k).  table: k rows of d, ld apart.  Requires n >= 0, d >= 1,
 * k >= 1 and a finite scale.
 */
int kmeans_table_forward(const int32_t* ids, int64_t n, int32_t k, int32_t d, int32_t type, const void* table,
                         int64_t ld, float scale, void* Y, void* hip_stream);

/*
 * Gradient of kmeans_table_forward: dTable[c] = scale times the sum of dY over
 * the slots of id c (k x d of the rows' type, zeros for an id without slots),
 * from dY (n rows) and a plan of kmeans_sort_plan of the ids (n slots).
 */
size_t kmeans_table_workspace_bytes(int64_t n, int32_t k, int32_t d, int32_t type);   /* 0 for bad sizes */
int kmeans_table_backward(const void* dY, int64_t lddy, int64_t n, int32_t k, int32_t d, int32_t type,
                          const int32_t* order, const int32_t* sorted_ids, const int32_t* offsets, float scale,
                          void* dTable, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The norm g over `count` tensors: the square root of the sum of all squares,
 * formed in float64, to *norm (device, float32; infinity beyond its range).  With
 * out, not NULL, out[i] = tensors[i] f rounded once, f = min(1, limit / g) in
 * float32; where g is infinite or NaN, as it is if an input is, out[i] = tensors[i]
 * (beyond float32's range g is not: values are scaled).  tensors, out, sizes (elements)
 * and types are HOST arrays, read before the call returns; out[i] is tensors[i]
 * (in place) or does not overlap any tensor.  Requires at most 2^40 elements in
 * all and a positive limit.
 */
size_t kmeans_clip_workspace_bytes(const int64_t* sizes, int32_t count);   /* 0 for bad sizes */
int kmeans_clip_norm(const void* const* tensors, void* const* out, const int64_t* sizes, const int32_t* types,
                     int32_t count, double limit, float* norm, void* workspace, size_t workspace_bytes,
                     void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* KMEANS_OPS_H */
