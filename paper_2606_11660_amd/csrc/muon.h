// What the kernels of the Muon step share: the polynomial, the momentum's arithmetic, and which
// matrix of a launch a workgroup belongs to.
#pragma once

#include "common.h"
#include "kernels.h"
#include "rows.h"

#pragma clang fp contract(off)

namespace attr {

// p(x) = a x + b x^3 + c x^5, the coefficients published with the method (K. Jordan and others, 2024)
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

// The group of a launch that holds this workgroup: the last whose first workgroup is not past it.
template <typename First>
__device__ inline const MuonGroup& group_of(const MuonArgs& a, uint32_t block, First first) {
  int k = 0;
  while (k + 1 < a.n_groups && first(a.g[k + 1]) <= block) ++k;
  return a.g[k];
}

__device__ inline float momentum_of(const MuonArgs& a, float m, float g) {
  return m * a.momentum + g * a.one_momentum;
}
__device__ inline float update_of(const MuonArgs& a, float m, float g) {  // m after its step
  return a.nesterov ? m * a.momentum + g * a.one_momentum : m;
}

// Four elements at any element's address, n of them there (the others are 0).
template <typename T>
__device__ inline void load4(const T* p, int n, float (&x)[4]) {
  if (n >= 4) {
    Raw<T, 4> r;
    r.load(p);
    r.get(x);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = e < n ? (float)p[e] : 0.f;
  }
}
template <typename T>
__device__ inline void store4(T* p, int n, const float (&x)[4]) {
  if (n >= 4) {
    Raw<T, 4> r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.set(e, (T)x[e]);
    *reinterpret_cast<typename Raw<T, 4>::vec*>(p) = r.v[0];
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = (T)x[e];
  }
}

// What u is multiplied by to have the norm 1, from |u|^2: 0 for zeros, NaN past all numbers.
__device__ inline double inverse_norm(double square) {
  return square > 0 ? (square < INFINITY ? 1.0 / sqrt(square) : NAN) : square == 0 ? 0.0 : NAN;
}

// The weight's step.
__device__ inline float stepped(float w, float x, float lr, float lr_wd) { return w - w * lr_wd - x * lr; }

}  // namespace attr
