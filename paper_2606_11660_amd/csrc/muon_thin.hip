// The Muon step of thin matrices, whose shorter side s is at most 64 (adapters, small heads).
//
// X^T X has only s x s entries, so the iteration runs on them: with G = u^T u (u's longer side
// first, [t][s]), A = G / trace G and P = a I + b A + c A^2, a step X = X P turns A into P A P, and
// after all of them X = u Q / |u|_F with Q the product of the P's.  All symmetric, all
// polynomials of A.  A holds the squares of the singular values, so this needs twice the
// digits, and has them: G, the iteration and the last product are in fp64 on the matrix cores
// (16 x 16 x 4).  u is computed twice and nothing of its size is stored: bound by memory, the
// gradient and the momentum read twice, the momentum and the weights written once.  168 matrices of rank 16
// (59 MB): 14 us for G, 8.5 for the steps, whose 18 products, 14 of them one after another, are one
// workgroup's, 13 for X and 6.6 for the two launches that copy the matrices' table, of 38.7 in all; as
// 128 x 128 tiles with pairs 209 where this takes 27 (56 of 16 x 1024), and for 8 of 4096 x 64 473 where
// this takes 112.
//
// Lanes of the 16 x 16 x 4 product: A's row and B's column are lane % 16, the fourth of K is
// lane / 16, and D's column is lane % 16, its rows lane / 16 + 4 r.
#include "muon.h"

namespace attr {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));
__device__ inline f64x4 mma(double a, double b, f64x4 c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }

// Times 16 rows of a wave whose loads are in flight together.
template <int T>
constexpr int rounds_of() { return T == 1 ? 4 : T == 2 ? 2 : 1; }

// Element (l, s) of a matrix whose longer side is l: its place.
__device__ inline int64_t place_of(const MuonGroup& q, int l, int s) {
  return q.rows >= q.cols ? (int64_t)l * q.cols + s : (int64_t)s * q.cols + l;
}

// Momentum and gradient of four of the longer side from r on at s of the shorter one, below l1.
template <typename G>
__device__ inline void load_run(const MuonGroup& q, const MuonEntry& en, bool turned, int r, int s, int l1, const G* gt,
                                float (&m)[4], float (&g)[4]) {
  const int n = s < q.S ? l1 - r : 0;
  if (turned) {
    const int64_t p = n > 0 ? (int64_t)s * q.cols + r : 0;
    load4(en.m + p, n, m);
    load4(gt + p, n, g);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t p = e < n ? (int64_t)(r + e) * q.cols + s : 0;
      m[e] = e < n ? en.m[p] : 0.f;
      g[e] = e < n ? (float)gt[p] : 0.f;
    }
  }
}

// The momentum's step, and G's upper tiles over kThinRows of the longer side: a wave adds up every
// fourth 16 of them, the four waves' sums in the order of the waves.
template <typename G, int T>
__global__ __launch_bounds__(256) void muon_thin_gram_kernel(MuonArgs a) {
  constexpr int TILES = T * (T + 1) / 2;
  __shared__ double sm[3][TILES * 256];
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_flat; });
  const uint32_t at = blockIdx.x - q.tile_flat, mat = at / q.n_flat, part = at - mat * q.n_flat;
  const MuonEntry& en = a.table[q.entry + mat];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int lane = threadIdx.x & 63, wave = wave_uniform((int)(threadIdx.x >> 6));
  const int l0 = (int)part * kThinRows, l1 = q.L - l0 < kThinRows ? q.L : l0 + kThinRows;
  const bool turned = q.rows < q.cols;
  f64x4 acc[TILES];
#pragma unroll
  for (int k = 0; k < TILES; ++k) acc[k] = f64x4{0, 0, 0, 0};
  constexpr int R = rounds_of<T>();
  for (int l = l0 + wave * 16; l < l1; l += 64 * R) {
    // K in fours: step e takes the rows l + 4 (lane / 16) + e
    float m[R][T][4], g[R][T][4];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int t = 0; t < T; ++t)
        load_run(q, en, turned, l + 64 * i + 4 * (lane >> 4), 16 * t + (lane & 15), l1, (const G*)en.g, m[i][t], g[i][t]);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      double u[T][4];
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int r = l + 64 * i + 4 * (lane >> 4), s = 16 * t + (lane & 15), n = s < q.S ? l1 - r : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float gr = g[i][t][e] * gs;
          m[i][t][e] = momentum_of(a, m[i][t][e], gr);
          u[t][e] = e < n ? (double)update_of(a, m[i][t][e], gr) : 0.0;
        }
        if (turned) {
          if (n > 0) store4(en.m + (int64_t)s * q.cols + r, n, m[i][t]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n) en.m[(int64_t)(r + e) * q.cols + s] = m[i][t][e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int tj = 0, k = 0; tj < T; ++tj)
#pragma unroll
          for (int ti = 0; ti <= tj; ++ti, ++k) acc[k] = mma(u[ti][e], u[tj][e], acc[k]);
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) sm[wave - 1][k * 256 + e * 64 + lane] = acc[k][e];
  }
  __syncthreads();
  if (wave > 0) return;
  double* const out = reinterpret_cast<double*>(q.base + mat * q.stride + q.gram) + (int64_t)part * TILES * 256;
#pragma unroll
  for (int k = 0; k < TILES; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      double x = acc[k][e];
#pragma unroll
      for (int w = 0; w < 3; ++w) x += sm[w][k * 256 + e * 64 + lane];
      out[k * 256 + e * 64 + lane] = x;  // row 16 ti + lane / 16 + 4 e, column 16 tj + lane % 16
    }
}

// The sum of a long matrix's parts of G, in the first one's place: a workgroup for each tile, a quarter of
// it every fourth part.  (One CU reads some 80 GB/s: 512 parts of 64 x 64 took the next kernel 136 us.)
template <int T>
__global__ __launch_bounds__(1024) void muon_thin_sum_kernel(MuonArgs a) {
  constexpr int TILES = T * (T + 1) / 2;
  __shared__ double sm[3][256];
  const uint32_t mat = blockIdx.x / TILES, tile = blockIdx.x % TILES;
  int k = 0;
  while (k + 1 < a.n_groups && a.g[k + 1].entry <= mat) ++k;
  const MuonGroup& q = a.g[k];
  if (q.n_flat <= kThinParts) return;
  double* const first = reinterpret_cast<double*>(q.base + (int64_t)(mat - q.entry) * q.stride + q.gram) + tile * 256 + threadIdx.x % 256;
  const uint32_t w = threadIdx.x / 256;
  double x = 0;
#pragma unroll 8
  for (uint32_t p = w; p < q.n_flat; p += 4) x += first[(int64_t)p * TILES * 256];
  if (w > 0) sm[w - 1][threadIdx.x % 256] = x;
  __syncthreads();
  if (w == 0) *first = x + sm[0][threadIdx.x] + sm[1][threadIdx.x] + sm[2][threadIdx.x];
}

// Q / |u| of one matrix from its parts of G: a wave for each 16 x 16 tile.
template <int T>
__global__ __launch_bounds__(64 * T * T) void muon_thin_poly_kernel(MuonArgs a, int steps) {
  constexpr int W = 16 * T, TILES = T * (T + 1) / 2;
  __shared__ double A[W][W], P[W][W], Q[W][W];
  __shared__ double trace;
  int k = 0;
  while (k + 1 < a.n_groups && a.g[k + 1].entry <= blockIdx.x) ++k;
  const MuonGroup& q = a.g[k];
  char* const base = q.base + (int64_t)(blockIdx.x - q.entry) * q.stride;
  const int lane = threadIdx.x & 63, wave = wave_uniform((int)(threadIdx.x >> 6));
  const int ti = wave / T, tj = wave - ti * T;
  const uint32_t n_parts = q.n_flat > kThinParts ? 1 : q.n_flat;
  const int c = 16 * tj + (lane & 15), r0 = 16 * ti + (lane >> 4);  // this lane's column, first of its rows
  const double* const parts = reinterpret_cast<const double*>(base + q.gram);
  if (ti <= tj) {
    const int tile = tj * (tj + 1) / 2 + ti;
    double x[4] = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t p = 0; p < n_parts; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += parts[(int64_t)p * TILES * 256 + tile * 256 + e * 64 + lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      A[r0 + 4 * e][c] = x[e];
      if (ti != tj) A[c][r0 + 4 * e] = x[e];
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    double x = (int)threadIdx.x < W ? A[threadIdx.x][threadIdx.x] : 0.0;
    x = wave_sum(x);
    if (threadIdx.x == 0) trace = x;
  }
  __syncthreads();
  const double inv = inverse_norm(trace);
  double own[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    own[e] = A[r0 + 4 * e][c] * inv * inv;
    Q[r0 + 4 * e][c] = r0 + 4 * e == c ? inv : 0.0;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 4; ++e) A[r0 + 4 * e][c] = own[e];
  __syncthreads();
  // this wave's tile of x y, both symmetric
  const auto product = [&](const double(&x)[W][W], const double(&y)[W][W]) {
    f64x4 d = {0, 0, 0, 0};
#pragma unroll
    for (int n = 0; n < W / 4; ++n) {
      const int kk = 4 * n + (lane >> 4);
      d = mma(x[kk][16 * ti + (lane & 15)], y[kk][c], d);
    }
    return d;
  };
  for (int step = 0; step < steps; ++step) {
    const f64x4 sq = product(A, A);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = r0 + 4 * e;
      P[r][c] = (r == c ? (double)kNsA : 0.0) + (double)kNsB * A[r][c] + (double)kNsC * sq[e];
    }
    __syncthreads();
    const f64x4 nq = product(P, Q);
    if (step + 1 == steps) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) Q[r0 + 4 * e][c] = nq[e];
      break;  // what is written below is this lane's own
    }
    const f64x4 pa = product(P, A);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      Q[r0 + 4 * e][c] = nq[e];
      A[r0 + 4 * e][c] = pa[e];
    }
    __syncthreads();
    const f64x4 pap = product(P, A);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) A[r0 + 4 * e][c] = pap[e];
    __syncthreads();
  }
  double* const out = reinterpret_cast<double*>(base + q.poly);
#pragma unroll
  for (int e = 0; e < 4; ++e) out[(r0 + 4 * e) * W + c] = Q[r0 + 4 * e][c];
}

// X = u Q and the weights' step: a wave takes 16 of the longer side at a time.
template <typename P, typename G, bool MASTER, int T>
__global__ __launch_bounds__(256) void muon_thin_apply_kernel(MuonArgs a) {
  constexpr int W = 16 * T;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_flat; });
  const uint32_t at = blockIdx.x - q.tile_flat, mat = at / q.n_flat, part = at - mat * q.n_flat;
  const MuonEntry& en = a.table[q.entry + mat];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int lane = threadIdx.x & 63, wave = wave_uniform((int)(threadIdx.x >> 6));
  const int low = lane & 15, high = lane >> 4;
  const int l0 = (int)part * kThinRows, l1 = q.L - l0 < kThinRows ? q.L : l0 + kThinRows;
  const double* const Q = reinterpret_cast<const double*>(q.base + mat * q.stride + q.poly);
  const bool turned = q.rows < q.cols;
  typedef typename std::conditional<MASTER, float, P>::type W_;
  P* const pt = (P*)en.p;
  const W_* const weights = MASTER ? (const W_*)en.master : (const W_*)en.p;
  constexpr int R = rounds_of<T>();
  for (int l = l0 + wave * 16; l < l1; l += 64 * R) {
    // K step (t, e) takes the columns 16 t + 4 (lane / 16) + e
    float m[R][T][4], g[R][T][4];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int r = l + 64 * i + low, s = 16 * t + 4 * high, n = r < l1 ? q.S - s : 0;
        if (turned) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int64_t p = e < n ? (int64_t)(s + e) * q.cols + r : 0;
            m[i][t][e] = e < n ? en.m[p] : 0.f;
            g[i][t][e] = e < n ? (float)((const G*)en.g)[p] : 0.f;
          }
        } else {
          const int64_t p = n > 0 ? (int64_t)r * q.cols + s : 0;
          load4(en.m + p, n, m[i][t]);
          load4((const G*)en.g + p, n, g[i][t]);
        }
      }
    f64x4 acc[R][T];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int t = 0; t < T; ++t) acc[i][t] = f64x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int o = 0; o < T; ++o) {
          const double x = Q[(16 * t + 4 * high + e) * W + 16 * o + low];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const double u = (double)update_of(a, m[i][t][e], g[i][t][e] * gs);
            acc[i][o] = turned ? mma(x, u, acc[i][o]) : mma(u, x, acc[i][o]);  // D's column, its lanes' neighbours, is the weights'
          }
        }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int o = 0; o < T; ++o) {
        W_ w[4];
        int64_t p[4];
        bool there[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = l + 64 * i + (turned ? low : high + 4 * e), s = 16 * o + (turned ? high + 4 * e : low);
          there[e] = r < l1 && s < q.S;
          p[e] = there[e] ? place_of(q, r, s) : 0;
          w[e] = weights[p[e]];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!there[e]) continue;
          const float nw = stepped((float)w[e], (float)acc[i][o][e], en.lr, en.lr_wd);
          if (MASTER) en.master[p[e]] = nw;
          pt[p[e]] = (P)nw;
        }
      }
  }
}

// Calls f with T, the 16s of a shorter side.
template <typename F>
hipError_t with_sixteens(int t, F f) {
  if (t == 1) f(std::integral_constant<int, 1>{});
  else if (t == 2) f(std::integral_constant<int, 2>{});
  else if (t == 3) f(std::integral_constant<int, 3>{});
  else f(std::integral_constant<int, 4>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_muon_thin_gram(int g_dtype, int t, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_type(g_dtype, [&](auto g) {
    return with_sixteens(t, [&](auto n) {
      hipLaunchKernelGGL((muon_thin_gram_kernel<decltype(g), decltype(n)::value>), dim3(blocks), dim3(256), 0, s, a);
    });
  });
}
hipError_t launch_muon_thin_sum(int t, const MuonArgs& a, uint32_t matrices, hipStream_t s) {
  return with_sixteens(t, [&](auto n) {
    constexpr int T = decltype(n)::value;
    hipLaunchKernelGGL((muon_thin_sum_kernel<T>), dim3(matrices * (T * (T + 1) / 2)), dim3(1024), 0, s, a);
  });
}
hipError_t launch_muon_thin_poly(int t, int steps, const MuonArgs& a, uint32_t matrices, hipStream_t s) {
  return with_sixteens(t, [&](auto n) {
    constexpr int T = decltype(n)::value;
    hipLaunchKernelGGL((muon_thin_poly_kernel<T>), dim3(matrices), dim3(64 * T * T), 0, s, a, steps);
  });
}
hipError_t launch_muon_thin_apply(int p_dtype, int g_dtype, bool master, int t, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_type(p_dtype, [&](auto p) {
    return with_type(g_dtype, [&](auto g) {
      return with_sixteens(t, [&](auto n) {
        typedef decltype(p) P;
        typedef decltype(g) G;
        constexpr int T = decltype(n)::value;
        if (master) hipLaunchKernelGGL((muon_thin_apply_kernel<P, G, true, T>), dim3(blocks), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((muon_thin_apply_kernel<P, G, false, T>), dim3(blocks), dim3(256), 0, s, a);
      });
    });
  });
}

}  // namespace attr
