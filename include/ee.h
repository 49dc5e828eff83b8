/*
 * ee.h - C ABI of the element embedding (same library, libsc_mi355x.so).
 *
 * The features a first layer starts from (Section 2.2 of arXiv 2504.10700: node features are
 * initialised from the chemical element): a row of a trainable table per atom,
 *
 *   Y[i,k] = scale * T[z_i,k]            dT[z,k] = scale * sum over the atoms with z_i = z of dY[i,k]
 *
 * Y is h [node][channel][1] of the tensor product with l_h = 0 (tp.h).  Tables may be much longer than a list of
 * elements (types of sites, of molecules): up to EE_MAX_ELEMENTS rows.
 *
 * An index outside 0..num_elements-1 (padding) has a zero row of Y and no part in dT.
 *
 * The gradient groups the rows by index first (a stable sort) and then sums each group in the order of
 * the batch, in pieces of fixed length: no atomics, bitwise reproducible.
 *
 * Types: SC_F32, SC_F64: all tensors of that type; SC_BF16: Y and dY bfloat16, T and dT fp32.  Sums in fp32, for SC_F64 in
 * fp64.  Other conventions as in sc.h: device pointers, dense row-major, 16-byte aligned; calls
 * enqueue on the given HIP stream and never synchronise; outputs are overwritten and alias nothing.
 */
#ifndef EE_MI355X_H
#define EE_MI355X_H

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EE_MAX_ELEMENTS 1000000 /* rows of the table  */
#define EE_MAX_CHANNELS 65536

typedef struct {
  int32_t struct_size;  /* = sizeof(ee_config), ABI guard       */
  int32_t num_elements; /* 1..EE_MAX_ELEMENTS                   */
  int32_t num_channels; /* 1..EE_MAX_CHANNELS                   */
  int32_t dtype;        /* sc_dtype                             */
  int32_t device;       /* HIP device ordinal                   */
  int32_t reserved;     /* 0                                    */
  double scale;         /* finite, in fp32 too but for SC_F64   */
} ee_config;

/* z [n_nodes] int32, T [num_elements][num_channels], Y [n_nodes][num_channels].  n_nodes == 0 does nothing. */
sc_status ee_forward(const ee_config* cfg, int64_t n_nodes, const int32_t* z, const void* T, void* Y, void* hip_stream);

/* Bytes of device workspace that ee_backward needs (the sorted order, sums of pieces). */
sc_status ee_workspace_bytes(const ee_config* cfg, int64_t n_nodes, size_t* bytes);

/* dY [n_nodes][num_channels], dT [num_elements][num_channels] (overwritten; zero rows for absent elements).
 * workspace: device memory, 256-byte aligned, at least ee_workspace_bytes().  n_nodes == 0 zeroes dT. */
sc_status ee_backward(const ee_config* cfg, int64_t n_nodes, const int32_t* z, const void* dY, void* dT, void* workspace,
                      size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EE_MI355X_H */
