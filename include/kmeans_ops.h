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
 *                     cluster, and the gradients of rows and adapters.
 *
 * Common to all.  Status codes and kmeans_mti_last_hip_error() are those of
 * kmeans_mti.h; no entry point throws, allocates device memory or
 * synchronizes, and all may be recorded into a HIP graph.  Device work is
 * ordered on hip_stream (NULL = the null stream).  All array arguments are
 * DEVICE pointers on the current device; a pointer may be NULL where its
 * array is empty.  Rows are `d` contiguous elements, `ld` elements apart
 * (ld >= d) where an argument ld* is given, else d apart.  Outputs must not
 * overlap inputs.  Rows have at most 2^28 elements.  Workspaces are the caller's: device memory of at least
 * the bytes that the *_workspace_bytes function gives, 256-byte aligned,
 * contents on entry of no matter, not to be used by another call until this
 * one's work completes.  Sums, statistics and gradients are formed in
 * float32 and rounded once to the type of the output; equal inputs give
 * bitwise equal outputs.
 */
#ifndef KMEANS_OPS_H
#define KMEANS_OPS_H

#include "kmeans_mti.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of rows. */
enum { KM_F32 = 0, KM_BF16 = 1, KM_F16 = 2 };

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

#ifdef __cplusplus
}
#endif

#endif /* KMEANS_OPS_H */
