/*
 * gp.h - C ABI of the products by element (same library, libsc_mi355x.so).
 *
 * Weights that belong to an atom's chemical element, as those of the contraction do (Section 2.2 of
 * arXiv 2504.10700), but mixing its channels: the self connection of an interaction layer.  For every atom i and
 * component c
 *
 *   Y[i,c,n] = sum_k X[i,c,k] * W[z_i,k,n] + residual[i,c,n]
 *
 * with the residual optional.  The components of one order l have 2l+1 rows; every order has its own W and its own
 * call.  With types of sites or experts in the place of elements and one component it is their layer.
 * The batch is ragged: any number of atoms of each element, none included.
 *
 * An index outside 0..num_elements-1 (padding) has no product: its rows of Y are the residual or zero, its rows of
 * dX zero, and it has no part in dW.
 *
 * Grouping.  The kernels walk over the atoms element by element.  gp_group makes that order, once for a batch: it depends
 * on z and num_elements alone, and serves every call on that batch, whatever its widths, components and type are.
 *
 * Strides.  Component c of atom i has its k_in elements at X + i * ld_in + c * k_in (dX the same; Y, residual, dY with
 * ld_out and k_out), so that the call reads one order's block of features laid out [atom][component][channel].
 * Elements between the blocks are neither read nor written.
 *
 * Types.  SC_F32: everything fp32; SC_F64: everything fp64; SC_BF16: the tensors with a row per atom (X, Y, residual,
 * dY, dX) bfloat16, W and dW fp32.  Products and sums in fp64 for SC_F64; otherwise sums are fp32 and
 * products have the exactness of fp32 ones: rows of bfloat16 are rounded once, at the end.
 *
 * Other conventions as in sc.h: device pointers, row-major; calls enqueue on the given HIP stream and never synchronise; outputs are
 * overwritten and share no memory with inputs or each other, but that Y may be the residual; sums have a fixed order (bitwise
 * reproducible results); errors by return code with sc_last_error().  Tensors are aligned to their element, grouping and
 * workspace to 256 bytes.
 */
#ifndef GP_MI355X_H
#define GP_MI355X_H

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GP_MAX_ELEMENTS 1024
#define GP_MAX_WIDTH 65536     /* largest k_in and k_out                           */
#define GP_MAX_COMPONENTS 64
#define GP_MAX_STRIDE 33554432 /* largest ld_in and ld_out                         */
#define GP_MAX_ROWS 536870912  /* largest n_nodes * components                      */
#define GP_UNGROUPED 64        /* batches of at most so many atoms need no grouping */

typedef struct {
  int32_t struct_size;  /* = sizeof(gp_config), ABI guard                          */
  int32_t num_elements; /* 1..GP_MAX_ELEMENTS                                      */
  int32_t k_in;         /* 1..GP_MAX_WIDTH                                         */
  int32_t k_out;        /* 1..GP_MAX_WIDTH                                         */
  int32_t components;   /* rows of an atom, 1..GP_MAX_COMPONENTS                   */
  int32_t dtype;        /* sc_dtype                                                */
  int32_t device;       /* HIP device ordinal                                      */
  int32_t reserved;     /* 0                                                       */
  int64_t ld_in;        /* elements between atoms of X, dX; 0: components * k_in   */
  int64_t ld_out;       /* ... of Y, residual, dY; 0: components * k_out           */
} gp_config;

/* Bytes of device memory of a batch's grouping: 0 up to GP_UNGROUPED atoms. */
sc_status gp_grouping_bytes(const gp_config* cfg, int64_t n_nodes, size_t* bytes);

/* Writes the grouping of z [n_nodes] (int32).  Of cfg it reads num_elements and device.  The grouping is ordinary
 * data: valid until it is overwritten, read by any number of calls.  Up to GP_UNGROUPED atoms it does nothing. */
sc_status gp_group(const gp_config* cfg, int64_t n_nodes, const int32_t* z, void* grouping, size_t grouping_bytes, void* hip_stream);

/* Bytes of device workspace that gp_forward and gp_backward need.  What a batch of more than GP_UNGROUPED atoms needs is enough for every batch of up to as many.  (Batches without a grouping whose
 * rows are many or wide are grouped by the call itself, there.) */
sc_status gp_workspace_bytes(const gp_config* cfg, int64_t n_nodes, size_t* bytes);

/* Forward.  z [n_nodes]; grouping: as gp_group wrote it for this z (NULL up to GP_UNGROUPED atoms); X [n_nodes][components][k_in];
 * W [num_elements][k_in][k_out]; residual [n_nodes][components][k_out] or NULL; Y [n_nodes][components][k_out].
 * workspace: device memory of at least gp_workspace_bytes().  n_nodes == 0 does nothing.
 * With the grouping of another z for as many elements the results are wrong (never an access outside the buffers of this call). */
sc_status gp_forward(const gp_config* cfg, int64_t n_nodes, const int32_t* z, const void* grouping, const void* X, const void* W,
                     const void* residual, void* Y, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Backward for an upstream gradient dY [n_nodes][components][k_out]:
 *   dX [n_nodes][components][k_in]  = sum_n W[z_i,k,n] dY[i,c,n]
 *   dW [num_elements][k_in][k_out]  = sum over the atoms of element z and their components of X[i,c,k] dY[i,c,n]
 * (zero for elements that are absent; the gradient of the residual is dY itself).  dX or dW may be NULL: then it is not
 * computed, and X (of dW) or W (of dX) may be NULL too.  n_nodes == 0 zeroes dW.
 * The second-order pass, for a cotangent HX of dX, is made of the same calls: the gradient with respect to dY is gp_forward
 * of HX (without residual), the one with respect to W is this dW with HX in the place of X. */
sc_status gp_backward(const gp_config* cfg, int64_t n_nodes, const int32_t* z, const void* grouping, const void* X, const void* W,
                      const void* dY, void* dX, void* dW, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GP_MI355X_H */
