// The activations of the dense layer with their first two derivatives, in the arithmetic type.
//
// SiLU and the GELU are z s(u(z)) with the logistic s and u = c1 z + c3 z^3 (SiLU: c1 = 1, c3 = 0).  With e = exp(-u), p = s(u) = 1 / (1 + e) and
// q = 1 - p = e p (not the difference of two numbers near 1):
//   value   z p
//   first   p + z p q u'
//   second  2 p q u' + z (p q (q - p) u'^2 + p q u'')
// ReLU is the same with p = (z > 0) and p q = 0, so one straight line of code serves all three.  The polynomial is evaluated at z cut to +-kCut
// (its cube would overflow for large z and 0 * infinity follow), and u from kLow on, where p would be the smallest number of the type and is taken
// as 0: e stays finite, and a large z finds a true zero; exp(-kCut) is below every number of the type, and a large positive z finds one too.
#pragma once
#include "sc_internal.h"
#include "../../include/dl.h"

namespace dl {

// exp(x) and 1 / x for x from 1 to 1e38.  fp32: the hardware's 2^x and reciprocal, each good to a unit or two of the last place.  x log2(e) is rounded to
// |x| units of the exponential; what the rounding left, and the rest of log2(e) beyond its first 24 bits, is the small t below, and 2^t is 1 + t ln 2 to within
// t^2.  24 instructions less than the library's pair.
__device__ __forceinline__ float exp_of(float x) {
  constexpr double kLog2e = 1.4426950408889634073599246810019;
  constexpr float kFirst = static_cast<float>(kLog2e), kRest = static_cast<float>(kLog2e - static_cast<double>(kFirst));
  const float y = x * kFirst;
  const float t = fmaf(x, kRest, fmaf(x, kFirst, -y));
  const float e = __builtin_amdgcn_exp2f(y);
  return fmaf(e, t * 0.693147180559945309417f, e);
}
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
__device__ __forceinline__ float inverse_of(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ double inverse_of(double x) { return 1.0 / x; }

template <typename T>
struct Gate {
  T c1, c3;
  int on, relu;

  static __host__ __device__ Gate of(int act) {
    constexpr double kTwoA = 1.5957691216057307117597842397375;   // 2 sqrt(2 / pi)
    return {static_cast<T>(act == DL_GELU ? kTwoA : 1.0), static_cast<T>(act == DL_GELU ? kTwoA * 0.044715 : 0.0), act != DL_NONE, act == DL_RELU};
  }

  struct Point {
    T z, p, pq, diff, u1, u2;   // diff = q - p
  };

  __device__ __forceinline__ Point at(T z) const {
    constexpr T kCut = T(800), kLow = sizeof(T) == 8 ? T(-700) : T(-87);
    const T w = z > kCut ? kCut : z < -kCut ? -kCut : z;
    const T square = w * w;
    T u = w * (c1 + c3 * square);
    u = u < kLow ? kLow : u;   // a NaN stays one, and z carries it in any case
    const T e = exp_of(-u);
    Point g;
    g.z = relu ? w : z;   // (0 times minus infinity is no value of max(z, 0))
    g.p = u > kLow ? inverse_of(T(1) + e) : T(0);
    const T q = e * g.p;
    g.pq = g.p * q;
    g.diff = q - g.p;
    g.u1 = c1 + T(3) * c3 * square;
    g.u2 = T(6) * c3 * w;
    if (relu) {
      g.p = z > T(0) ? T(1) : T(0);
      g.pq = T(0);
    }
    return g;
  }

  __device__ __forceinline__ T value(T z) const {
    const Point g = at(z);
    return (z > T(0) ? z : g.z) * g.p;
  }

  __device__ __forceinline__ T first(T z) const {
    const Point g = at(z);
    return g.p + g.z * g.pq * g.u1;
  }

  __device__ __forceinline__ void both(T z, T* first_out, T* second) const {
    const Point g = at(z);
    *first_out = g.p + g.z * g.pq * g.u1;
    *second = T(2) * g.pq * g.u1 + (g.z * g.pq) * (g.diff * g.u1 * g.u1 + g.u2);   // z * p q first: 0 for large z
  }
};

}  // namespace dl
