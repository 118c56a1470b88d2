// Layer norm of token rows (attr_layer_norm) and its gradient (attr_layer_norm_backward).
//
//     y  = (x - mean) rstd w + b,   rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = rstd (e - mean(e) - u mean(e u)),  e = dy w,  u = (x - mean) rstd
//     dw = sum of dy u,  db = sum of dy  over the rows
//
// HBM-bound: a row is read once (forward: x; backward: x and dy) into the registers of its
// threads, so that the variance is taken about the mean itself, and written once.  All sums are
// in fp32 over a row's threads and over a chunk of rows; the chunks are joined in fp64.
#include "rows.h"

namespace attr {
namespace {

constexpr int kVec = 8;  // neighbouring elements of a thread

// Weights of w_dtype at column c, n of them there.
__device__ inline void load_w(const void* w, int dtype, int c, int n, float (&x)[kVec], float none) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) x[e] = none;
  } else if (dtype == 0) {
    load_n<float, kVec>((const float*)w + c, n, x);
  } else if (dtype == 1) {
    load_n<__bf16, kVec>((const __bf16*)w + c, n, x);
  } else {
    load_n<_Float16, kVec>((const _Float16*)w + c, n, x);
  }
}

// Sum over a row's NT threads; every thread has it.  `sm` has a float for each wave, and is
// used again only after another barrier.
template <int NT>
__device__ inline float row_sum(float v, float* sm) {
  v = wave_sum(v);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) v += sm[w];
  }
  return v;
}

template <int NT>
constexpr int block_of() { return NT < 256 ? 256 : NT; }

template <typename X, typename Y, int NT, int NV>
__device__ inline void layer_norm_row(const RowsArgs& r, const NormArgs& a, uint32_t slot, int t, float (&sm)[2][16]) {
  const RowSlot s = row_slot(r, slot);
  if (!s.written) return;
  const int d = a.d;
  Y* const y = (Y*)a.y + s.row * a.ldy;
  float x[NV][kVec];
  float mean = 0.f, rstd = 0.f;
  if (s.inside) {
    const X* const xr = (const X*)a.x + s.row * a.ldx;
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * NT + t) * kVec;
      load_n<X, kVec>(xr + c, d - c, x[v]);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum += x[v][e];
    mean = row_sum<NT>(sum, sm[0]) / (float)d;
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * NT + t) * kVec;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        x[v][e] = c + e < d ? x[v][e] - mean : 0.f;
        sq += x[v][e] * x[v][e];
      }
    }
    rstd = 1.f / sqrtf(row_sum<NT>(sq, sm[1]) / (float)d + a.eps);
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[v][e] = 0.f;
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * NT + t) * kVec;
    if (s.inside && c < d) {
      float w[kVec], b[kVec];
      load_w(a.weight, a.w_dtype, c, d - c, w, 1.f);
      load_w(a.bias, a.w_dtype, c, d - c, b, 0.f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[v][e] = x[v][e] * rstd * w[e] + b[e];
    }
    store_n<Y, kVec>(y + c, d - c, x[v]);
  }
  if (t == 0) {
    if (a.mean) a.mean[s.row] = mean;
    if (a.rstd) a.rstd[s.row] = rstd;
  }
}
template <typename X, typename Y, int NT, int NV>
__global__ __launch_bounds__(block_of<NT>()) void layer_norm_kernel(RowsArgs r, NormArgs a) {
  constexpr int ROWS = block_of<NT>() / NT;
  __shared__ float sm[2][16];
  const int t = ROWS == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT;
  for (uint64_t slot = (uint64_t)blockIdx.x * ROWS + (ROWS == 1 ? 0u : wave_uniform(threadIdx.x / NT)); slot < r.n_slots;
       slot += (uint64_t)gridDim.x * ROWS)
    layer_norm_row<X, Y, NT, NV>(r, a, (uint32_t)slot, t, sm);
}

// A chunk of a unit's slots: dx of its rows, and its share of the weights' gradients, each
// thread its own columns over the chunk's rows.  RELOAD: a row's registers do not fit beside
// those sums, and it is read twice.
template <typename X, typename Y, int NT, int NV, bool RELOAD>
__global__ __launch_bounds__(block_of<NT>()) void layer_norm_grad_kernel(RowsArgs r, NormGradArgs a) {
  constexpr int ROWS = block_of<NT>() / NT;
  __shared__ float sm[2][2][16];
  __shared__ float join[ROWS == 1 ? 1 : (ROWS - 1) * NV * NT * kVec];
  const int t = ROWS == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT;
  const int which = ROWS == 1 ? 0 : (int)wave_uniform(threadIdx.x / NT);
  const int d = a.d;
  int turn = 0;
  for (uint64_t block = blockIdx.x; block < (uint64_t)a.units * a.chunks; block += gridDim.x) {
  const uint32_t unit = (uint32_t)(block / a.chunks), chunk = (uint32_t)(block - (uint64_t)unit * a.chunks);
  const uint32_t base = unit * a.unit, from = chunk * a.chunk,
                 to = a.unit - from < a.chunk ? a.unit : from + a.chunk;
  float dw[NV][kVec], db[NV][kVec];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < kVec; ++e) dw[v][e] = db[v][e] = 0.f;
  for (uint32_t i = from + which; i < to; i += ROWS) {
    const RowSlot s = row_slot(r, base + i);
    if (!s.written) continue;
    X* const dx = (X*)a.dx + s.row * a.lddx;
    if (!s.inside) {
      if (a.dx) {
        const float zero[kVec] = {};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int c = (v * NT + t) * kVec;
          store_n<X, kVec>(dx + c, d - c, zero);
        }
      }
      continue;
    }
    const X* const xr = (const X*)a.x + s.row * a.ldx;
    const Y* const dyr = (const Y*)a.dy + s.row * a.lddy;
    const float mean = a.mean[s.row], rstd = a.rstd[s.row];
    constexpr int KEPT = RELOAD ? 1 : NV;
    float u[KEPT][kVec], e1[KEPT][kVec];
    float s1 = 0.f, s2 = 0.f;
    if constexpr (!RELOAD) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + t) * kVec;
        load_n<X, kVec>(xr + c, d - c, u[v]);
        load_n<Y, kVec>(dyr + c, d - c, e1[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * NT + t) * kVec, k = RELOAD ? 0 : v;
      if (RELOAD) {
        load_n<X, kVec>(xr + c, d - c, u[k]);
        load_n<Y, kVec>(dyr + c, d - c, e1[k]);
      }
      float w[kVec];
      load_w(a.weight, a.w_dtype, c, d - c, w, 1.f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        u[k][e] = c + e < d ? (u[k][e] - mean) * rstd : 0.f;
        dw[v][e] += e1[k][e] * u[k][e];
        db[v][e] += e1[k][e];
        e1[k][e] = c + e < d ? e1[k][e] * w[e] : 0.f;
        s1 += e1[k][e];
        s2 += e1[k][e] * u[k][e];
      }
    }
    if (!a.dx) continue;
    s1 = row_sum<NT>(s1, sm[turn][0]) / (float)d;
    s2 = row_sum<NT>(s2, sm[turn][1]) / (float)d;
    turn ^= 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * NT + t) * kVec, k = RELOAD ? 0 : v;
      if (RELOAD) {
        float w[kVec];
        load_n<X, kVec>(xr + c, d - c, u[k]);
        load_n<Y, kVec>(dyr + c, d - c, e1[k]);
        load_w(a.weight, a.w_dtype, c, d - c, w, 1.f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          u[k][e] = (u[k][e] - mean) * rstd;
          e1[k][e] *= w[e];
        }
      }
      float o[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) o[e] = (e1[k][e] - s1 - u[k][e] * s2) * rstd;
      store_n<X, kVec>(dx + c, d - c, o);
    }
  }
  // the sums of a workgroup's rows, those of its first threads last
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float(&own)[NV][kVec] = k ? db : dw;
    float* const to_out = k ? a.dbias : a.dweight;
    if (!to_out) continue;
    if constexpr (ROWS > 1) {
      __syncthreads();
      if (which > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int e = 0; e < kVec; ++e) join[((which - 1) * NV + v) * NT * kVec + e * NT + t] = own[v][e];
      }
      __syncthreads();
      if (which > 0) continue;
#pragma unroll
      for (int w = 0; w < ROWS - 1; ++w)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int e = 0; e < kVec; ++e) own[v][e] += join[(w * NV + v) * NT * kVec + e * NT + t];
    }
    float* const out = a.part ? a.part + ((int64_t)block * 2 + k) * d
                              : to_out + (int64_t)unit * (k ? a.ldb : a.ldw);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * NT + t) * kVec;
      if (!a.part && a.accumulate) {
        float was[kVec];
        load_n<float, kVec>(out + c, d - c, was);
#pragma unroll
        for (int e = 0; e < kVec; ++e) own[v][e] += was[e];
      }
      store_n<float, kVec>(out + c, d - c, own[v]);
    }
  }
  }
}

// Joins a unit's chunks: 64 columns a workgroup, its 16 waves every 16th chunk.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(NormGradArgs a) {
  __shared__ double sm[2][16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t cuts = (uint32_t)(a.d + 63) / 64;
  for (uint64_t block = blockIdx.x; block < (uint64_t)a.units * cuts; block += gridDim.x) {
  const uint32_t unit = (uint32_t)(block / cuts);
  const int c = (int)(block - (uint64_t)unit * cuts) * 64 + lane;
  double w = 0, b = 0;
  if (c < a.d) {
    const float* p = a.part + (int64_t)unit * a.chunks * 2 * a.d + c;
#pragma unroll 4
    for (uint32_t j = wave; j < a.chunks; j += 16) {
      if (a.dweight) w += p[(int64_t)j * 2 * a.d];
      if (a.dbias) b += p[((int64_t)j * 2 + 1) * a.d];
    }
  }
  __syncthreads();
  sm[0][wave][lane] = w;
  sm[1][wave][lane] = b;
  __syncthreads();
  float* const out = wave ? a.dbias : a.dweight;
  if (wave >= 2 || c >= a.d || !out) continue;
  double sum = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) sum += sm[wave][k][lane];
  float* const o = out + (int64_t)unit * (wave ? a.ldb : a.ldw) + c;
  *o = (float)(a.accumulate ? sum + *o : sum);
  }
}

template <typename X, typename Y, int NT, int NV>
hipError_t norm_rows(const RowsArgs& r, const NormArgs& a, hipStream_t s) {
  constexpr int ROWS = block_of<NT>() / NT;
  hipLaunchKernelGGL((layer_norm_kernel<X, Y, NT, NV>), dim3(grid_of((r.n_slots + (uint64_t)ROWS - 1) / ROWS)), dim3(block_of<NT>()), 0, s,
                     r, a);
  return hipGetLastError();
}
template <typename X, typename Y, int NT, int NV, bool RELOAD = false>
hipError_t norm_grad_rows(const RowsArgs& r, const NormGradArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((layer_norm_grad_kernel<X, Y, NT, NV, RELOAD>), dim3(grid_of((uint64_t)a.units * a.chunks)), dim3(block_of<NT>()), 0, s,
                     r, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(int x_dtype, int y_dtype, const RowsArgs& r, const NormArgs& a, hipStream_t s) {
  return with_type(x_dtype, [&](auto x) {
    return with_type(y_dtype, [&](auto y) {
      typedef decltype(x) X;
      typedef decltype(y) Y;
      if (a.d <= 512) return norm_rows<X, Y, 64, 1>(r, a, s);
      if (a.d <= 1024) return norm_rows<X, Y, 64, 2>(r, a, s);
      if (a.d <= 2048) return norm_rows<X, Y, 64, 4>(r, a, s);
      if (a.d <= 4096) return norm_rows<X, Y, 256, 2>(r, a, s);
      if (a.d <= 8192) return norm_rows<X, Y, 256, 4>(r, a, s);
      if (a.d <= 16384) return norm_rows<X, Y, 1024, 2>(r, a, s);
      return norm_rows<X, Y, 1024, 4>(r, a, s);
    });
  });
}

uint32_t norm_chunk(uint32_t unit, uint32_t units, int32_t d) {
  const uint64_t slots = (uint64_t)unit * units;
  const uint64_t want = (slots + 767) / 768;
  const uint32_t least = d <= 2048 ? 16 : 4;
  const uint32_t chunk = want < least ? least : (uint32_t)want;
  return chunk < unit ? chunk : unit;
}

hipError_t launch_layer_norm_grad(int x_dtype, int dy_dtype, const RowsArgs& r, const NormGradArgs& a, hipStream_t s) {
  const hipError_t e = with_type(x_dtype, [&](auto x) {
    return with_type(dy_dtype, [&](auto y) {
      typedef decltype(x) X;
      typedef decltype(y) Y;
      if (a.d <= 512) return norm_grad_rows<X, Y, 64, 1>(r, a, s);
      if (a.d <= 1024) return norm_grad_rows<X, Y, 64, 2>(r, a, s);
      if (a.d <= 2048) return norm_grad_rows<X, Y, 64, 4>(r, a, s);
      if (a.d <= 4096) return norm_grad_rows<X, Y, 256, 2>(r, a, s);
      if (a.d <= 8192) return norm_grad_rows<X, Y, 256, 4>(r, a, s);
      if (a.d <= 16384) return norm_grad_rows<X, Y, 1024, 2>(r, a, s);
      return norm_grad_rows<X, Y, 1024, 4, true>(r, a, s);
    });
  });
  if (e != hipSuccess || !a.part || (!a.dweight && !a.dbias)) return e;
  hipLaunchKernelGGL(layer_norm_join_kernel, dim3(grid_of((uint64_t)((a.d + 63) / 64) * a.units)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace attr
