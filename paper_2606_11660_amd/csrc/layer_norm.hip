// Layer norm of token rows (attr_layer_norm) and its gradient (attr_layer_norm_backward).
//
//     y  = (x - mean) rstd w + b,   rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = rstd (e - mean(e) - u mean(e u)),  e = dy w,  u = (x - mean) rstd
//     dw = sum of dy u,  db = sum of dy  over the rows
//
// HBM-bound: a row is read once (forward: x; backward: x and dy) into the registers of its
// threads, so that the variance is taken about the mean itself, and written once.  All sums are
// in fp32 over a row's threads and over a share of rows; the shares are joined in fp64.  The
// threads of a row are chosen by its width, for 8 to 32 values a thread: one wave up to 1024 columns
// needs no barrier, more waves keep enough of the registers free for several rows on a CU.
#include "rows.h"

namespace attr {
namespace {

// Weights of w_dtype, or `none`.
template <int N>
__device__ inline void load_w(const void* w, int dtype, Cols<N> c, float (&x)[N], float none) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = none;
  } else if (dtype == 0) {
    load_n<float, N>((const float*)w, c, x);
  } else if (dtype == 1) {
    load_n<__bf16, N>((const __bf16*)w, c, x);
  } else {
    load_n<_Float16, N>((const _Float16*)w, c, x);
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

// A thread holds NV vectors of N neighbouring columns, NT N columns from one to the next.
template <typename X, typename Y, int NT, int NV, int N>
__device__ inline void layer_norm_row(const RowsArgs& r, const NormArgs& a, uint32_t slot, int t, float (&sm)[2][16]) {
  const RowSlot s = row_slot(r, slot);
  if (!s.written) return;
  const int d = a.d;
  Y* const y = (Y*)a.y + s.row * a.ldy;
  float mean = 0.f, rstd = 0.f;
  if (!s.inside) {
    const float zero[N] = {};
#pragma unroll
    for (int v = 0; v < NV; ++v) store_n<Y, N>(y, Cols<N>((v * NT + t) * N, d), zero);
  } else {
    const X* const xr = (const X*)a.x + s.row * a.ldx;
    float sum = 0.f, x[NV][N];
    Raw<X, N> in[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) in[v].load(xr + Cols<N>((v * NT + t) * N, d).at);
    // one vector a thread: its weights come along; more would cost registers
    float w[N], b[N];
    if constexpr (NV == 1) {
      load_w<N>(a.weight, a.w_dtype, Cols<N>(t * N, d), w, 1.f);
      load_w<N>(a.bias, a.w_dtype, Cols<N>(t * N, d), b, 0.f);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<N> c((v * NT + t) * N, d);
      in[v].get(x[v]);
#pragma unroll
      for (int e = 0; e < N; ++e) sum += c.own(e) ? x[v][e] : 0.f;
    }
    mean = row_sum<NT>(sum, sm[0]) / (float)d;
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<N> c((v * NT + t) * N, d);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[v][e] -= mean;
        sq += c.own(e) ? x[v][e] * x[v][e] : 0.f;
      }
    }
    rstd = 1.f / sqrtf(row_sum<NT>(sq, sm[1]) / (float)d + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<N> c((v * NT + t) * N, d);
      if constexpr (NV > 1) {
        load_w<N>(a.weight, a.w_dtype, c, w, 1.f);
        load_w<N>(a.bias, a.w_dtype, c, b, 0.f);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) x[v][e] = x[v][e] * rstd * w[e] + b[e];
      store_n<Y, N>(y, c, x[v]);
    }
  }
  if (t == 0) {
    if (a.mean) a.mean[s.row] = mean;
    if (a.rstd) a.rstd[s.row] = rstd;
  }
}
template <typename X, typename Y, int NT, int NV, int N>
__global__ __launch_bounds__(block_of<NT>()) void layer_norm_kernel(RowsArgs r, NormArgs a) {
  constexpr int ROWS = block_of<NT>() / NT;
  __shared__ float sm[2][16];
  const int t = ROWS == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT;
  for (uint64_t slot = (uint64_t)blockIdx.x * ROWS + (ROWS == 1 ? 0u : wave_uniform(threadIdx.x / NT)); slot < r.n_slots;
       slot += (uint64_t)gridDim.x * ROWS)
    layer_norm_row<X, Y, NT, NV, N>(r, a, (uint32_t)slot, t, sm);
}

// Both sums over a row's NT threads.
template <int NT>
__device__ inline void row_sums(float& a, float& b, float (&sm)[2][16]) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) {
      sm[0][threadIdx.x >> 6] = a;
      sm[1][threadIdx.x >> 6] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      a += sm[0][w];
      b += sm[1][w];
    }
  }
}

// What is loaded of a row ahead of its turn.
template <typename X, typename Y, int NV, int N>
struct NormRow {
  Raw<X, N> x[NV];
  Raw<Y, N> dy[NV];
};
// Where 64 rows of a share are, and their statistics, one in each lane: a row's turn needs no
// memory for them.
struct NormRows {
  RowSlot s;
  float mean, rstd;
  __device__ inline NormRows(const RowsArgs& r, const NormGradArgs& a, uint32_t base, uint64_t i) {
    s.row = 0;
    s.written = s.inside = false;
    mean = rstd = 0.f;
    if (i < a.unit) s = row_slot(r, base + (uint32_t)i);
    if (s.inside) {
      mean = a.mean[s.row];
      rstd = a.rstd[s.row];
    }
  }
  __device__ inline RowSlot slot(int k) const {
    RowSlot o;
    o.row = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)s.row >> 32), k) << 32) |
                      (uint32_t)__builtin_amdgcn_readlane((int)(uint64_t)s.row, k));
    const int is = __builtin_amdgcn_readlane((int)s.written | (int)s.inside << 1, k);
    o.written = is & 1;
    o.inside = is & 2;
    return o;
  }
};
__device__ inline float lane_of(float x, int k) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), k));
}

// A share of a unit's slots (every chunks-th of them, so that padding is spread evenly): dx of
// its rows, and its part of the weights' gradients, each thread its own columns.  The next row
// is loaded while one is worked on.  RELOAD: a row's registers do not fit beside those sums;
// it is read twice.  Of 512 threads two workgroups a CU hide each other's waits where both types have
// 16 bits (8192 rows of 8192, bf16: 90.1 us, one workgroup 99.0); wider rows need the registers (fp32: 131 us,
// with two workgroups 254).
template <typename X, typename Y, int NT, int NV, int N, bool RELOAD>
__global__ __launch_bounds__(block_of<NT>(), NT == 512 ? (sizeof(X) + sizeof(Y) == 4 ? 4 : 2) : 1) void layer_norm_grad_kernel(RowsArgs r, NormGradArgs a) {
  constexpr int ROWS = block_of<NT>() / NT, KEPT = RELOAD ? 1 : NV;
  __shared__ float sm[2][2][16];
  __shared__ float join[ROWS == 1 ? 1 : (ROWS - 1) * NV * NT * N];
  const int t = ROWS == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT;
  const int which = ROWS == 1 ? 0 : (int)wave_uniform(threadIdx.x / NT);
  const int d = a.d;
  int turn = 0;
  for (uint64_t block = blockIdx.x; block < (uint64_t)a.units * a.chunks; block += gridDim.x) {
    const uint32_t unit = (uint32_t)(block / a.chunks), chunk = (uint32_t)(block - (uint64_t)unit * a.chunks);
    const uint32_t base = unit * a.unit;
    const uint64_t stride = (uint64_t)a.chunks * ROWS;
    float dw[NV][N], db[NV][N];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) dw[v][e] = db[v][e] = 0.f;
    NormRow<X, Y, KEPT, N> cur;
    const auto fetch = [&](const RowSlot& s) {
      if (RELOAD || !s.inside) return;
      const X* const xr = (const X*)a.x + s.row * a.ldx;
      const Y* const dyr = (const Y*)a.dy + s.row * a.lddy;
#pragma unroll
      for (int v = 0; v < KEPT; ++v) {
        const int c = Cols<N>((v * NT + t) * N, d).at;
        cur.x[v].load(xr + c);
        cur.dy[v].load(dyr + c);
      }
    };
    for (uint64_t i0 = (uint64_t)chunk * ROWS + which; i0 < a.unit; i0 += 64 * stride) {
      const NormRows ahead(r, a, base, i0 + (threadIdx.x & 63) * stride);
      RowSlot s = ahead.slot(0), next;
      fetch(s);
      for (int q = 0; q < 64 && i0 + q * stride < a.unit; ++q, s = next) {
        next = q < 63 ? ahead.slot(q + 1) : RowSlot{0, false, false};
        X* const dx = (X*)a.dx + s.row * a.lddx;
        if (!s.inside) {
          fetch(next);
          if (s.written && a.dx) {
            const float zero[N] = {};
#pragma unroll
            for (int v = 0; v < NV; ++v) store_n<X, N>(dx, Cols<N>((v * NT + t) * N, d), zero);
          }
          continue;
        }
        const float mean = lane_of(ahead.mean, q), rstd = lane_of(ahead.rstd, q);
        float u[KEPT][N], e1[KEPT][N];
        float s1 = 0.f, s2 = 0.f;
        const auto terms = [&](int v) {  // u and dy of vector v
          const Cols<N> c((v * NT + t) * N, d);
          const int k = RELOAD ? 0 : v;
          if constexpr (RELOAD) {
            cur.x[0].load((const X*)a.x + s.row * a.ldx + c.at);
            cur.dy[0].load((const Y*)a.dy + s.row * a.lddy + c.at);
          }
          cur.x[k].get(u[k]);
          cur.dy[k].get(e1[k]);
#pragma unroll
          for (int e = 0; e < N; ++e) u[k][e] = (u[k][e] - mean) * rstd;
        };
        if constexpr (!RELOAD) {
#pragma unroll
          for (int v = 0; v < NV; ++v) terms(v);
          fetch(next);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const Cols<N> c((v * NT + t) * N, d);
          const int k = RELOAD ? 0 : v;
          if constexpr (RELOAD) terms(v);
          float w[N];
          load_w<N>(a.weight, a.w_dtype, c, w, 1.f);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            dw[v][e] += e1[k][e] * u[k][e];
            db[v][e] += e1[k][e];
            e1[k][e] *= w[e];
            s1 += c.own(e) ? e1[k][e] : 0.f;
            s2 += c.own(e) ? e1[k][e] * u[k][e] : 0.f;
          }
          if (RELOAD) __builtin_amdgcn_sched_barrier(0);
        }
        if (a.dx) {
          row_sums<NT>(s1, s2, sm[turn]);
          s1 /= (float)d;
          s2 /= (float)d;
          turn ^= 1;
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            const int k = RELOAD ? 0 : v;
            if constexpr (RELOAD) {
              terms(v);
              float w[N];
              load_w<N>(a.weight, a.w_dtype, Cols<N>((v * NT + t) * N, d), w, 1.f);
#pragma unroll
              for (int e = 0; e < N; ++e) e1[0][e] *= w[e];
            }
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = (e1[k][e] - s1 - u[k][e] * s2) * rstd;
            store_n<X, N>(dx, Cols<N>((v * NT + t) * N, d), o);
            if (RELOAD) __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
    // the sums of a workgroup's rows, those of its first threads first
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float(&own)[NV][N] = k ? db : dw;
      float* const to_out = k ? a.dbias : a.dweight;
      if (!to_out) continue;
      if constexpr (ROWS > 1) {
        __syncthreads();
        if (which > 0) {
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) join[((which - 1) * NV + v) * NT * N + e * NT + t] = own[v][e];
        }
        __syncthreads();
        if (which > 0) continue;
#pragma unroll
        for (int w = 0; w < ROWS - 1; ++w)
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) own[v][e] += join[(w * NV + v) * NT * N + e * NT + t];
      }
      float* const out = a.part ? a.part + ((int64_t)block * 2 + k) * d : to_out + (int64_t)unit * (k ? a.ldb : a.ldw);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Cols<N> c((v * NT + t) * N, d);
        if (!a.part && a.accumulate) {
          float was[N];
          load_n<float, N>(out, c, was);
#pragma unroll
          for (int e = 0; e < N; ++e) own[v][e] += was[e];
        }
        store_n<float, N>(out, c, own[v]);
      }
    }
  }
}

// Joins a unit's shares: 64 columns of one of the two gradients a workgroup, its 16 waves
// every 16th share.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(NormGradArgs a) {
  __shared__ double sm[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t cuts = (uint32_t)(a.d + 63) / 64;
  for (uint64_t block = blockIdx.x; block < (uint64_t)a.units * cuts * 2; block += gridDim.x) {
    const int k = (int)(block & 1);
    const uint32_t unit = (uint32_t)((block >> 1) / cuts);
    const int c = (int)((block >> 1) - (uint64_t)unit * cuts) * 64 + lane;
    float* const out = k ? a.dbias : a.dweight;
    if (!out) continue;
    double sum = 0;
    if (c < a.d) {
      const float* p = a.part + ((int64_t)unit * a.chunks * 2 + k) * a.d + c;
#pragma unroll 8
      for (uint32_t j = wave; j < a.chunks; j += 16) sum += p[(int64_t)j * 2 * a.d];
    }
    __syncthreads();
    sm[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || c >= a.d) continue;
    sum = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += sm[w][lane];
    float* const o = out + (int64_t)unit * (k ? a.ldb : a.ldw) + c;
    *o = (float)(a.accumulate ? sum + *o : sum);
  }
}

template <typename X, typename Y, int NT, int NV, int N>
hipError_t norm_rows(const RowsArgs& r, const NormArgs& a, hipStream_t s) {
  constexpr int ROWS = block_of<NT>() / NT;
  hipLaunchKernelGGL((layer_norm_kernel<X, Y, NT, NV, N>), dim3(grid_of((r.n_slots + (uint64_t)ROWS - 1) / ROWS)), dim3(block_of<NT>()), 0, s,
                     r, a);
  return hipGetLastError();
}
template <typename X, typename Y, int NT, int NV, int N, bool RELOAD = false>
hipError_t norm_grad_rows(const RowsArgs& r, const NormGradArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((layer_norm_grad_kernel<X, Y, NT, NV, N, RELOAD>), dim3(grid_of((uint64_t)a.units * a.chunks)), dim3(block_of<NT>()), 0, s,
                     r, a);
  return hipGetLastError();
}

// Neighbouring elements of a thread: 16 bytes of the wider of two types, so that a wave's access is
// one run of memory.
template <typename X, typename Y>
constexpr int elements() { return sizeof(X) == 4 || sizeof(Y) == 4 ? 4 : 8; }

}  // namespace

hipError_t launch_layer_norm(int x_dtype, int y_dtype, const RowsArgs& r, const NormArgs& a, hipStream_t s) {
  // few rows: more threads for each, for the time of one row (1024 rows of 2048: 4.7 us, with a wave for
  // each 6.0; 64 of 8192: 4.6 with 1024 threads, 5.2 with 256, but 1024 of them 13.6 and 10.0)
  const bool few = r.n_slots <= (a.d <= 2048 ? 1024u : 256u);
  return with_type(x_dtype, [&](auto x) {
    return with_type(y_dtype, [&](auto y) {
      typedef decltype(x) X;
      typedef decltype(y) Y;
      if (a.d < 8) return norm_rows<X, Y, 64, 1, 1>(r, a, s);
      if (a.d <= 512) return norm_rows<X, Y, 64, 1, 8>(r, a, s);
      if (a.d <= 2048 && few) return norm_rows<X, Y, 256, 1, 8>(r, a, s);
      if (a.d <= 1024) return norm_rows<X, Y, 64, 2, 8>(r, a, s);
      if (a.d <= 2048) return norm_rows<X, Y, 64, 4, 8>(r, a, s);
      if (a.d <= 8192 && few) return norm_rows<X, Y, 1024, 1, 8>(r, a, s);
      if (a.d <= 4096) return norm_rows<X, Y, 256, 2, 8>(r, a, s);
      if (a.d <= 8192) return norm_rows<X, Y, 256, 4, 8>(r, a, s);
      if (a.d <= 16384) return norm_rows<X, Y, 1024, 2, 8>(r, a, s);
      return norm_rows<X, Y, 1024, 4, 8>(r, a, s);
    });
  });
}

// Shares of a unit: workgroups enough to fill the GPU, each with several rows, since its sums are written
// and read again; past 16384 columns, where a row takes 40 us, with one at least (64 rows of 32768: 55 us,
// with four 120).
// As many as the GPU holds at once: 1024 workgroups of a few registers a thread, 512 of many (32768 rows, us,
// with 512 / 1024: of 512 bf16 37.2 / 31.0, of 1024 fp32 81.4 / 86.5, of 2048 bf16 128 / 97.6; 16384 of 4096
// bf16 93.0 / 110).
uint32_t norm_chunks(uint32_t unit, uint32_t units, int32_t d) {
  const uint32_t rows = d <= 1024 ? 16 : d <= 16384 ? 4 : 1, most = d <= 512 || (d > 1024 && d <= 2048) ? 1024 : 512;
  const uint32_t by_rows = (unit + rows - 1) / rows, by_units = most / units;
  return by_rows < by_units ? by_rows : by_units > 1 ? by_units : 1;
}

hipError_t launch_layer_norm_grad(int x_dtype, int dy_dtype, const RowsArgs& r, const NormGradArgs& a, hipStream_t s) {
  const hipError_t e = with_type(x_dtype, [&](auto x) {
    return with_type(dy_dtype, [&](auto y) {
      typedef decltype(x) X;
      typedef decltype(y) Y;
      constexpr int N = elements<X, Y>(), M = 8 / N;
      if (a.d < 8) return norm_grad_rows<X, Y, 64, 1, 1>(r, a, s);
      if (a.d <= 512) return norm_grad_rows<X, Y, 64, 1 * M, N>(r, a, s);
      if (a.d <= 1024) return norm_grad_rows<X, Y, 64, 2 * M, N>(r, a, s);
      if (a.d <= 2048) return norm_grad_rows<X, Y, 256, 1 * M, N>(r, a, s);
      if (a.d <= 4096) return norm_grad_rows<X, Y, 256, 2 * M, N>(r, a, s);
      if (a.d <= 8192) return norm_grad_rows<X, Y, 512, 2 * M, N>(r, a, s);
      if (a.d <= 16384) return norm_grad_rows<X, Y, 1024, 2 * M, N>(r, a, s);
      return norm_grad_rows<X, Y, 1024, 4 * M, N, true>(r, a, s);
    });
  });
  if (e != hipSuccess || !a.part || (!a.dweight && !a.dbias)) return e;
  hipLaunchKernelGGL(layer_norm_join_kernel, dim3(grid_of((uint64_t)((a.d + 63) / 64) * a.units * 2)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace attr
