/*
 * kunlun_layers.h - the operators in front of attention, on packed event rows (part of the same library as kunlun.h).
 *
 *   kunlun_embedding_fwd / _bwd       rows of a table by event id, scaled; the table's gradient, summed over equal
 *                                     ids in a fixed order (ids sorted, no atomics on sums)
 *   kunlun_layer_norm_fwd / _bwd      layer normalisation of every row (the Norm of Eq. (seed-level attention) and of
 *                                     the rows in front of an attention block) and its gradients
 *   kunlun_grouped_linear_fwd / _bwd  one linear map per group of consecutive rows, groups of any sizes: projections
 *                                     that differ by event type (event-level personalisation), the products of experts
 *
 * Memory, streams, workspaces, data types and errors as in kunlun.h: device pointers, aligned to their values (rows of odd
 * widths are taken as they lie; the grouped linear maps: tensors 16-byte aligned), row-major and contiguous; nothing is allocated, kept or synchronised; kernels only
 * (no memset), so that calls can be captured; statuses instead of exceptions; `workspace` 256-byte aligned, scratch.  The
 * device that is current at the call must be the device of `stream` and of the tensors.  Outputs must not overlap
 * inputs.  Sums are held in fp32 and rounded once; equal calls give equal bits.
 */
#ifndef KUNLUN_LAYERS_H_
#define KUNLUN_LAYERS_H_

#include "kunlun.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KUNLUN_MAX_CHANNELS 16384 /* values per row of any operator here */
#define KUNLUN_MAX_GROUPS 4096

/*
 * Embedding lookup:  out[r] = scale * table[ids[r]]  for r < n;  an id outside [0, rows) (padding: -1) gives a row of zeros.
 *   table  in,  device, [rows, D]       rows < 2^31; may be NULL when rows == 0
 *   ids    in,  device, [n] int32 (id_bytes = 4) or int64 (id_bytes = 8)
 *   out    out, device, [n, D]
 * 1 <= D <= KUNLUN_MAX_CHANNELS, n < 2^31, scale finite.  n == 0 is legal and does nothing.
 */
int kunlun_embedding_fwd(const void* table, const void* ids, void* out, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                         int dtype, void* stream);

/*
 * Gradient of the table:  d_table[v] = scale * sum of d_out[r] over the r with ids[r] = v, every row written (zeros where no
 * id names it); ids outside [0, rows) add nothing.
 *   d_out    in,  device, [n, D];   d_table  out, device, [rows, D]
 * The ids are sorted with their positions; runs of equal ids are added in the order of their positions within fixed ranges,
 * the ranges' fp32 sums in order.  workspace: kunlun_embedding_bwd_workspace_bytes(...) bytes.  n == 0: d_table is set
 * to zero.  rows == 0 does nothing.
 */
int kunlun_embedding_bwd(const void* d_out, const void* ids, void* d_table, int64_t n, int64_t rows, int D, float scale, int id_bytes,
                         int dtype, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace for kunlun_embedding_bwd with these sizes (0 for invalid ones); a workspace for some n also serves a
 * smaller n with the same rows, D and dtype. */
size_t kunlun_embedding_bwd_workspace_bytes(int64_t n, int64_t rows, int D, int dtype);

/*
 * Layer normalisation of every row:  y = (x - mean) * rstd * weight + bias,  mean and variance (biased) over the D values
 * of the row, rstd = 1 / sqrt(variance + eps).
 *   x       in,  device, [rows, D];  y  out, device, [rows, D]
 *   weight  in,  device, [D] or NULL (ones);  bias  in, device, [D] or NULL (zeros)
 *   mean, rstd  out, device, float [rows]; each may be NULL
 * The variance is the mean of (x - mean)^2 with the row in registers (no difference of two large sums).
 * 1 <= D <= KUNLUN_MAX_CHANNELS, eps >= 0 and finite.  rows == 0 is legal and does nothing.
 */
int kunlun_layer_norm_fwd(const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd, int64_t rows, int D,
                          float eps, int dtype, void* stream);

/*
 * Gradients of <y, dy>:  with h = (x - mean) rstd and g = dy * weight,
 *     dx = rstd (g - mean(g) - h mean(g h)),   dw = sum over the rows of dy h,   db = sum over the rows of dy.
 *   x, weight  in,  as in the forward call;   dy  in, device, [rows, D];   mean, rstd  in, device: of the forward call
 *   dx  out, device, [rows, D];   dw, db  out, device, [D]; each of the three may be NULL (not computed)
 * dw and db: fp32 sums over fixed sets of rows, added in a fixed order and rounded once.  rows == 0: dw and db are set to
 * zero.  workspace: kunlun_layer_norm_bwd_workspace_bytes(...) bytes; not needed when dw and db are NULL.
 */
int kunlun_layer_norm_bwd(const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, void* dx, void* dw,
                          void* db, int64_t rows, int D, int dtype, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace for kunlun_layer_norm_bwd with these sizes (0 for invalid ones); it also serves fewer rows. */
size_t kunlun_layer_norm_bwd_workspace_bytes(int64_t rows, int D, int dtype);

/*
 * One linear map per group of rows:  y[r] = x[r] w[g]  for the rows r = offsets[g] .. offsets[g + 1] - 1 of group g.
 *   x  in,  device, [total, K];   w  in, device, [G, K, N] (applied from the right: rows = input channel)
 *   y  out, device, [total, N];   offsets  in, device int32 [G + 1]: offsets[0] = 0, non-decreasing, offsets[G] <= total
 * Groups may be empty.  Rows from offsets[G] on belong to no group (a padded batch): they are not read, and their rows of y are
 * left as they are (fill_rest = 0) or set to zero (fill_rest = 1).
 * K and N: whole 16-byte pieces (multiples of 8 in bf16, of 4 in fp32) up to KUNLUN_MAX_CHANNELS; 1 <= G <= KUNLUN_MAX_GROUPS;
 * total < 2^31.  total == 0 does nothing.
 */
int kunlun_grouped_linear_fwd(const void* x, const void* w, void* y, const int32_t* offsets, int G, int64_t total, int K, int N,
                              int fill_rest, int dtype, void* stream);

/*
 * Gradients of <y, dy>:  dx[r] = dy[r] w[g]^T;  dw[g] = sum over the rows of group g of x[r]^T dy[r] (zeros for an empty group).
 *   dy  in,  device, [total, N];   dx  out, device, [total, K] or NULL;   dw  out, device, [G, K, N] or NULL
 * w may be NULL when dx is, x when dw is; fill_rest: as above, for the rows of dx.  Long groups are cut into ranges of rows whose fp32 sums go to the workspace
 * (kunlun_grouped_linear_bwd_workspace_bytes(...) bytes; not needed when dw is NULL) and are added in row order.
 */
int kunlun_grouped_linear_bwd(const void* x, const void* w, const void* dy, void* dx, void* dw, const int32_t* offsets, int G,
                              int64_t total, int K, int N, int fill_rest, int dtype, void* workspace, size_t workspace_bytes,
                              void* stream);

/* Bytes of workspace for kunlun_grouped_linear_bwd with these sizes (0 for invalid ones). */
size_t kunlun_grouped_linear_bwd_workspace_bytes(int G, int64_t total, int K, int N, int dtype);

#ifdef __cplusplus
}
#endif
#endif /* KUNLUN_LAYERS_H_ */
