// The activations of the dense layer with their first two derivatives, in the arithmetic type.
//
// SiLU and the GELU are z s(u(z)) with the logistic s and u = z, or u = 2 a (z + c z^3).  With p = s(u), q = 1 - p
// (each from exp(-|u|), so neither is a difference of two numbers near 1):
//   value   z p
//   first   p + z p q u'
//   second  2 p q u' + z (p q (q - p) u'^2 + p q u'')
// The polynomial of the GELU is evaluated at z cut to +-kCut, where p and q are 0 and 1 to the last bit already: its cube
// would overflow for large z and 0 * infinity follow.
#pragma once
#include "sc_internal.h"
#include "../../include/dl.h"

namespace dl {

__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

template <typename T>
struct Gate {
  struct Point {
    T p, q, u1, u2;
  };

  static __device__ __forceinline__ Point at(int act, T z) {
    constexpr T kTwoA = T(1.5957691216057307117597842397375), kC = T(0.044715), kCut = T(50);
    T u = z, u1 = T(1), u2 = T(0);
    if (act == DL_GELU) {
      const T w = z > kCut ? kCut : z < -kCut ? -kCut : z;   // a NaN stays one
      u = kTwoA * w * (T(1) + kC * w * w);
      u1 = kTwoA * (T(1) + T(3) * kC * w * w);
      u2 = T(6) * kTwoA * kC * w;
    }
    const T e = exp_of(u > T(0) ? -u : u);   // in (0, 1]
    const T small = e / (T(1) + e), large = T(1) / (T(1) + e);
    return {u > T(0) ? large : small, u > T(0) ? small : large, u1, u2};
  }

  static __device__ __forceinline__ T value(int act, T z) {
    if (act == DL_NONE) return z;
    if (act == DL_RELU) return z > T(0) ? z : z * T(0);   // a NaN stays one
    return z * at(act, z).p;
  }

  static __device__ __forceinline__ T first(int act, T z) {
    if (act == DL_NONE) return T(1);
    if (act == DL_RELU) return z > T(0) ? T(1) : T(0);
    const Point g = at(act, z);
    return g.p + z * (g.p * g.q) * g.u1;
  }

  // *second is set for the curved activations only
  static __device__ __forceinline__ void both(int act, T z, T* first_out, T* second) {
    *second = T(0);
    if (act == DL_NONE || act == DL_RELU) {
      *first_out = first(act, z);
      return;
    }
    const Point g = at(act, z);
    const T pq = g.p * g.q;
    *first_out = g.p + z * pq * g.u1;
    *second = T(2) * pq * g.u1 + z * pq * ((g.q - g.p) * g.u1 * g.u1 + g.u2);
  }
};

}  // namespace dl
