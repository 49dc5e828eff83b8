/*
 * dl.h - C ABI of the dense layer (same library, libsc_mi355x.so).
 *
 * What a model of arXiv 2504.10700 has beside its equivariant kernels: the radial weights
 * R[edge][path][channel] of the tensor product (Section 4.1, input of Algorithm 1) are the output
 * of a small stack of such layers on functions of the edge length, and the readout of the
 * invariant channels is another (Section 2.2).  For every row i
 *
 *   Z[i,n] = sum_k X[i,k] * W[k,n] + b[n]          Y[i,n] = act(Z[i,n]) + residual[i,n]
 *
 * with bias and residual optional.  Forces are derivatives of the energy and reach a loss through
 * the layer's dX, so there is a second-order pass as well (as sc_double_backward, tp_double_backward).
 *
 * Types.  SC_F32: everything fp32; SC_F64: everything fp64; SC_BF16: the tensors with a row
 * per edge or atom (X, Y, Z, residual, dY, dX, HX, ddY, X2) bfloat16, the weights and their
 * gradients (W, b, dW, db, W2, b2) fp32.  Products and sums in fp64 for SC_F64; otherwise sums are
 * fp32 and products have the exactness of fp32 ones: rows of bfloat16 are rounded once, at the end.
 *
 * Strides.  Rows of X, dX, HX, X2 are ld_in elements apart, rows of Y, Z, residual, dY, ddY ld_out
 * (0: dense, k_in and k_out), so that a layer can read the invariant channels of features laid
 * out [atom][component][channel].  Elements between the rows are neither read nor written.
 *
 * Other conventions as in sc.h: device pointers, row-major, 16-byte aligned; calls enqueue on the
 * given HIP stream and never synchronise; outputs are overwritten and share no memory with inputs
 * or each other; sums have a fixed order (bitwise reproducible results); errors by return code
 * with sc_last_error().
 */
#ifndef DL_MI355X_H
#define DL_MI355X_H

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* DL_SILU: z / (1 + exp(-z)).  DL_GELU: z / (1 + exp(-2 a (z + 0.044715 z^3))), a = sqrt(2 / pi), the form with
 * the hyperbolic tangent.  DL_RELU: max(z, 0), its derivative at 0 taken as 0. */
typedef enum { DL_NONE = 0, DL_RELU = 1, DL_SILU = 2, DL_GELU = 3 } dl_activation;

#define DL_MAX_WIDTH 65536     /* largest k_in and k_out   */
#define DL_MAX_STRIDE 33554432 /* largest ld_in and ld_out */

typedef struct {
  int32_t struct_size; /* = sizeof(dl_config), ABI guard        */
  int32_t k_in;        /* 1..DL_MAX_WIDTH                       */
  int32_t k_out;       /* 1..DL_MAX_WIDTH                       */
  int32_t activation;  /* dl_activation                         */
  int32_t dtype;       /* sc_dtype                              */
  int32_t device;      /* HIP device ordinal                    */
  int64_t ld_in;       /* elements between rows of X, dX, HX, X2; 0: k_in       */
  int64_t ld_out;      /* ... of Y, Z, residual, dY, ddY; 0: k_out              */
} dl_config;

/* Forward.  X [n_rows][k_in], W [k_in][k_out]; b [k_out], residual [n_rows][k_out] or NULL;
 * Y [n_rows][k_out].  Z [n_rows][k_out]: what the backward calls need, or NULL (always NULL-able; with
 * DL_NONE the backward calls do not read it).  n_rows == 0 does nothing. */
sc_status dl_forward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* b,
                     const void* residual, void* Y, void* Z, void* hip_stream);

/* Bytes of device workspace that dl_backward and dl_double_backward need. */
sc_status dl_workspace_bytes(const dl_config* cfg, int64_t n_rows, size_t* bytes);

/* Backward for an upstream gradient dY [n_rows][k_out], with G = dY * act'(Z):
 *   dX [n_rows][k_in]   = sum_n W[k,n] G[.,n]
 *   dW [k_in][k_out]    = sum over the rows of X[.,k] G[.,n]
 *   db [k_out]          = sum over the rows of G
 * (the gradient of the residual is dY itself).  Each of dX, dW, db may be NULL: then it is not computed.
 * Z: as dl_forward wrote it; NULL with DL_NONE.  workspace: device memory, 256-byte aligned, at
 * least dl_workspace_bytes().  n_rows == 0 zeroes dW and db. */
sc_status dl_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z, const void* dY,
                      void* dX, void* dW, void* db, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Second-order pass: the gradients of sum(HX * dX) with respect to the arguments of dl_backward, for a cotangent
 * HX [n_rows][k_in] of dX.  With V = HX W and S = V * dY * act''(Z):
 *   ddY [n_rows][k_out] = V * act'(Z)
 *   X2  [n_rows][k_in]  = sum_n W[k,n] S[.,n]
 *   W2  [k_in][k_out]   = sum over the rows of X[.,k] S[.,n] + HX[.,k] G[.,n]
 *   b2  [k_out]         = sum over the rows of S
 * X2, W2 and b2 include the path through Z = X W + b.  With DL_NONE and DL_RELU S is zero, and so are X2 and b2.
 * X2, W2, b2 may be NULL.  Workspace as for dl_backward.  n_rows == 0 zeroes W2 and b2. */
sc_status dl_double_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z,
                             const void* dY, const void* HX, void* ddY, void* X2, void* W2, void* b2, void* workspace,
                             size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DL_MI355X_H */
