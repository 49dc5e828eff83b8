/*
 * ou.h - C ABI of the orthogonalised update (same library, libsc_mi355x.so).
 *
 * A step of an optimizer for weight matrices, after the backward pass (and gc.h).  For every matrix of a list
 * of tensors [count][rows][cols], with m = min(rows, cols)
 *
 *   M <- mu M + G             U = G + mu M  (OU_NESTEROV),  M without it,  G where there is no momentum
 *   X = U / (|U| + eps)       |U|: the root of the sum of the squares of U's elements
 *   steps times               X <- a X + (b S + c S S) X    with S = X X^T   (rows <= cols)
 *                             X <- a X + X (b S + c S S)    with S = X^T X   (rows > cols)
 *   update = X                W <- (1 - rate * decay) W - rate * scale * X
 *
 * With the usual coefficients the iteration brings every singular value of U that is not much smaller than
 * the largest near 1: the update has the directions of U, all about equally long.  `scale` is the caller's, per tensor
 * (for a matrix [k_in][k_out] usually sqrt(max(1, k_out / k_in))).
 *
 * Types.  SC_F32: everything fp32; SC_F64: everything fp64; SC_BF16: G and the update bfloat16, M and W fp32.  M, U, W are
 * computed element by element in fp32 (SC_F64: fp64), the norm in fp64 (of finite elements of any size); an update of bfloat16 is rounded once, at the end.
 * The products of matrices are, seen over a whole matrix (the norm of the error), as exact as fp32 ones (SC_F64: fp64).  Their operands have 22 bits relative to the largest singular value
 * there can be after the step, and fewer below 2^-16 of it: rows or columns far smaller than the others are relatively less exact (1e-4 of them as in fp32, 1e-6 to 6e-5, 1e-8 to 6e-3 of their size).
 * Coefficients that need more (|b| t^2 + |c| t^4 > 64 |a| in a step, t the largest singular value there can be before it) take fp32 instructions.
 *
 * A matrix of zeros (an element that is absent) stays zero, for every eps.  Where U has an element that is not finite, the matrix's X is NaN (steps 0, infinite elements: these
 * are, the others zero); no other matrix sees it.
 *
 * ou_tensor is a HOST array that the call reads before it returns (its contents travel to the device as kernel arguments: no copy, no
 * allocation, usable in a captured graph).  Tensors are dense, row-major, aligned to at least their element, and
 * share no memory.  Sums have a fixed order: the same list gives the same bits (which kernel a matrix takes, and so its last bits, may depend on what else is in the
 * list).  Other conventions as in sc.h.
 */
#ifndef OU_MI355X_H
#define OU_MI355X_H

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OU_MAX_TENSORS 16384
#define OU_MAX_SIDE 65536   /* largest rows and cols             */
#define OU_MAX_STEPS 32
#define OU_MAX_TILES 8388608 /* of all matrices together: ceil(rows / 64) * ceil(cols / 64) each */
#define OU_MAX_GROWTH 1024  /* see ou_config: coefficients       */

#define OU_NESTEROV 1 /* ou_config.flags */

typedef struct {
  const void* grad; /* dev: G                                                         */
  void* momentum;   /* dev: M, updated in place; NULL: none                           */
  void* weight;     /* dev: W, updated in place; NULL: only the update is wanted      */
  void* update;     /* dev: X, overwritten; NULL: only the weight is wanted           */
  double scale;     /* finite, as rate * scale, rate * decay, momentum; in fp32 too but for SC_F64 */
  int64_t count;    /* matrices, 0 is valid                                           */
  int32_t rows;     /* 1..OU_MAX_SIDE                                                 */
  int32_t cols;     /* 1..OU_MAX_SIDE                                                 */
  int32_t dtype;    /* sc_dtype                                                       */
  int32_t reserved; /* 0                                                              */
} ou_tensor;

/* Coefficients: from |x| <= 1 on, the polynomial a x + b x^3 + c x^5 may grow to at most OU_MAX_GROWTH in any step
 * (otherwise the call fails with SC_ERR_UNSUPPORTED). */
typedef struct {
  int32_t struct_size; /* = sizeof(ou_config), ABI guard     */
  int32_t device;      /* HIP device ordinal                 */
  int32_t steps;       /* 0..OU_MAX_STEPS                    */
  uint32_t flags;      /* OU_NESTEROV                        */
  double a, b, c;      /* finite                             */
  double momentum;     /* mu, finite                         */
  double rate;         /* finite                             */
  double decay;        /* finite                             */
  double eps;          /* > 0, finite                        */
} ou_config;

/* Bytes of device workspace that ou_step needs for this list.  (A matrix whose shorter side is at most 64 or 128 and whose longer one is more takes there what squares of 64 x 64 or 128 x 128 along
 * its longer side take, however short the shorter one is: 100 000 of 1 x 200 9.8 GB.) */
sc_status ou_workspace_bytes(const ou_config* cfg, int64_t n_tensors, const ou_tensor* tensors, size_t* bytes);

/* workspace: device memory, 256-byte aligned, at least ou_workspace_bytes(). */
sc_status ou_step(const ou_config* cfg, int64_t n_tensors, const ou_tensor* tensors, void* workspace, size_t workspace_bytes,
                  void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* OU_MI355X_H */
