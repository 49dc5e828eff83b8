/*
 * gc.h - C ABI of the global gradient norm and clipping (same library, libsc_mi355x.so).
 *
 * Between the backward pass and the step of the optimizer: over a list of tensors x_1..x_m
 *
 *   norm = sqrt(sum over all tensors and elements of x^2)
 *   coefficient = max_norm / (norm + eps) where that is below 1, otherwise 1 (a NaN norm: NaN)
 *   dst_j = coefficient * src_j
 *
 * Sums in fp64 in a fixed order: bitwise reproducible, and fp32 gradients of any finite size neither
 * overflow nor vanish in the square (fp64 gradients beyond 1e154 do overflow).  fp32 and bfloat16 elements are multiplied in
 * fp32, in fp64 where the coefficient is below 1e-30.  An infinite element gives the norm infinity and the coefficient 0 (so
 * the infinite element becomes NaN, the others 0); a NaN makes norm, coefficient and every result NaN: a training
 * loop tests the norm before it takes the step.
 *
 * gc_tensor is a HOST array that the call reads before it returns (pointers travel to the
 * device as kernel arguments: no copy, no allocation, usable in a captured graph).  Tensors are
 * dense; any alignment of at least their element.  dst may be src (clipping in place), or NULL for every tensor (the
 * norm alone is wanted); other overlaps are not allowed.  Other conventions as in sc.h.
 */
#ifndef GC_MI355X_H
#define GC_MI355X_H

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GC_MAX_TENSORS 65536

typedef struct {
  const void* src; /* dev                                           */
  void* dst;       /* dev; src itself, another buffer, or NULL      */
  int64_t numel;   /* 0 is valid                                    */
  int32_t dtype;   /* sc_dtype: SC_F32, SC_F64 or SC_BF16           */
  int32_t reserved;
} gc_tensor;

typedef struct {
  int32_t struct_size; /* = sizeof(gc_config), ABI guard                 */
  int32_t dtype;       /* SC_F32 or SC_F64: type of norm_and_coefficient */
  int32_t device;      /* HIP device ordinal                             */
  int32_t reserved;    /* 0                                              */
  double max_norm;     /* > 0 (infinity: never clips)                    */
  double eps;          /* >= 0                                           */
} gc_config;

/* Bytes of device workspace that gc_clip needs for this list. */
sc_status gc_workspace_bytes(const gc_config* cfg, int64_t n_tensors, const gc_tensor* tensors, size_t* bytes);

/* norm_and_coefficient: dev, two values of cfg->dtype (overwritten).  workspace: device memory, 256-byte aligned, at
 * least gc_workspace_bytes().  An empty list has the norm 0 and the coefficient min(1, max_norm / eps). */
sc_status gc_clip(const gc_config* cfg, int64_t n_tensors, const gc_tensor* tensors, void* norm_and_coefficient,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GC_MI355X_H */
