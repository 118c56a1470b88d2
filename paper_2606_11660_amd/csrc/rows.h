// Token rows of the embedding and layer norm kernels: where a slot's row is, loads and
// stores of a few elements at any element's address, and sums over a row's threads.
#pragma once

#include "common.h"
#include "kernels.h"

namespace attr {

// Token slot (the same for a wave's lanes) of a batch: example slot / T, token slot % T.
struct RowSlot {
  int64_t row;
  bool written;  // the slot's row belongs to the call
  bool inside;   // it is a token's; else a padding slot, whose outputs are zeros
};
template <typename I>
__device__ inline I wave_uniform(I x) {
  if constexpr (sizeof(I) == 8)
    return (I)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)x >> 32)) << 32) |
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint64_t)x));
  else
    return (I)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ inline RowSlot row_slot(const RowsArgs& a, uint32_t slot) {
  uint32_t i = 0, t = slot;
  if (a.row_offset || a.length) {
    i = slot / a.T;
    t = slot - i * a.T;
  }
  RowSlot r;
  r.inside = !a.length || (int32_t)t < a.length[i];
  r.row = a.row_offset ? (int64_t)((uint64_t)a.row_offset[i] + t) : (int64_t)slot;
  const bool there = (uint64_t)r.row < (uint64_t)a.n_rows;
  r.written = there && (r.inside || !a.row_offset);
  r.inside = r.inside && there;
  return r;
}

// N elements of type T at any element's address, in accesses of up to 16 bytes.
template <typename T, int N>
struct Vec {
  typedef T plain __attribute__((ext_vector_type(N)));
  typedef plain loose __attribute__((aligned(sizeof(T))));
};
template <typename T>
struct Vec<T, 1> {
  typedef T loose;
};
template <typename T, int N>
__device__ inline void load_n(const T* p, int n, float (&x)[N]) {  // n of them are there; the others are 0
  if (n >= N) {
    if constexpr (N == 1) {
      x[0] = (float)p[0];
    } else if constexpr (N * sizeof(T) > 16) {
      constexpr int H = 16 / sizeof(T);
#pragma unroll
      for (int h = 0; h < N / H; ++h) {
        const auto v = *reinterpret_cast<const typename Vec<T, H>::loose*>(p + h * H);
#pragma unroll
        for (int e = 0; e < H; ++e) x[h * H + e] = (float)v[e];
      }
    } else {
      const auto v = *reinterpret_cast<const typename Vec<T, N>::loose*>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (float)v[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = e < n ? (float)p[e] : 0.f;
  }
}
template <typename T, int N>
__device__ inline void store_n(T* p, int n, const float (&x)[N]) {
  if (n >= N) {
    if constexpr (N == 1) {
      p[0] = (T)x[0];
    } else if constexpr (N * sizeof(T) > 16) {
      constexpr int H = 16 / sizeof(T);
#pragma unroll
      for (int h = 0; h < N / H; ++h) {
        typename Vec<T, H>::loose v;
#pragma unroll
        for (int e = 0; e < H; ++e) v[e] = (T)x[h * H + e];
        *reinterpret_cast<typename Vec<T, H>::loose*>(p + h * H) = v;
      }
    } else {
      typename Vec<T, N>::loose v;
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = (T)x[e];
      *reinterpret_cast<typename Vec<T, N>::loose*>(p) = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = (T)x[e];
  }
}

// Workgroups of a launch; kernels stride over the work that is left.
inline uint32_t grid_of(uint64_t blocks) { return (uint32_t)(blocks < (1u << 21) ? blocks : 1u << 21); }

// Calls f(T{}) with the type that a dtype code names.
template <typename F>
inline hipError_t with_type(int dtype, F f) {
  if (dtype == 0) return f(float{});
  if (dtype == 1) return f(__bf16{});
  return f(_Float16{});
}

}  // namespace attr
