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

// N elements of type T at any element's address, as they come from memory: accesses of up to 16
// bytes, converted where they are used, so that the loads of several vectors are in flight together.
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
struct Raw {
  static constexpr int W = N * sizeof(T) > 16 ? 16 / sizeof(T) : N;  // elements of an access
  typedef typename Vec<T, W>::loose vec;
  vec v[N / W];
  __device__ inline T at(int e) const {
    if constexpr (W == 1) return v[e];
    else return v[e / W][e % W];
  }
  __device__ inline void set(int e, T x) {
    if constexpr (W == 1) v[e] = x;
    else v[e / W][e % W] = x;
  }
  __device__ inline void load(const T* p) {
#pragma unroll
    for (int k = 0; k < N / W; ++k) v[k] = *reinterpret_cast<const vec*>(p + k * W);
  }
  __device__ inline void store(T* p) const {
#pragma unroll
    for (int k = 0; k < N / W; ++k) *reinterpret_cast<vec*>(p + k * W) = v[k];
  }
  __device__ inline void get(float (&x)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)at(e);
  }
};
// A lane's N columns of rows of d >= N: from c on, or, where fewer are left, the row's last N, of
// which the first `skip` belong to the lane before (skip >= N: none is the lane's own).  So every
// lane loads whole vectors inside the row, without a branch.
template <int N>
struct Cols {
  int at, skip;
  __device__ inline Cols(int c, int d) {
    at = c < d - N ? c : d - N;
    skip = c - at;
  }
  __device__ inline bool own(int e) const { return e >= skip; }
};
template <typename T, int N>
__device__ inline void load_n(const T* row, Cols<N> c, float (&x)[N]) {
  Raw<T, N> r;
  r.load(row + c.at);
  r.get(x);
}
template <typename T, int N>
__device__ inline void store_n(T* row, Cols<N> c, const float (&x)[N]) {
  Raw<T, N> r;
#pragma unroll
  for (int e = 0; e < N; ++e) r.set(e, (T)x[e]);
  if (c.skip == 0) {
    r.store(row + c.at);
  } else if (c.skip < N) {
#pragma unroll
    for (int e = 1; e < N; ++e)
      if (c.own(e)) row[c.at + e] = r.at(e);
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
