// One Muon step over many matrices (attr_muon_step).
//
//     m = mu m + (1 - mu) g',   u = mu m + (1 - mu) g' (nesterov) or m
//     X = u / |u|_F;  five times:  A = X X^T,  B = b A + c A^2,  X = a X + B X
//     w = w - lr wd w - lr X
//
// Bound by the matrix cores: with s and t a matrix's shorter and longer side, s^2 t + s^3 +
// 2 s^2 t flops a step of the iteration, since A and B are symmetric and only their upper
// triangles of tiles are computed.  The iteration holds Y, the update with its longer side
// first ([t][s]; A = Y^T Y, Y = a Y + Y B), so that Y is stored once and in one order: A reads
// it along its columns (transposing LDS reads), Y B along its rows.
//
// Operands are fp16 with powers of two before them: no entry of X passes 1.21, of A 1.45 or of
// B 2.9 (|p(x)| <= 1.2025 on [0, 1.2025] for p = a x + b x^3 + c x^5), so 2^15 X, 2^15 A and
// 2^14 B fit, and what is below 2^-24 of the largest entry is still held.  fp16 keeps 11 bits where
// bf16 keeps 8, at the same rate.  With pairs every operand is two fp16 values (22 bits) and a
// product three: hi hi + hi lo + lo hi.  Sums are fp32, the norm's fp64.
#include "muon.h"

namespace attr {
namespace {

constexpr float kScale = 32768.f, kScalePoly = 16384.f;  // of X and A; of B

__global__ __launch_bounds__(64) void muon_table_kernel(MuonTable t) {
  for (int j = threadIdx.x; j < t.n; j += 64) t.to[j] = t.e[j];
}

// Sum over a workgroup of 256 threads, for every thread.
__device__ inline double block_sum(double v, double* sm) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
  __syncthreads();
  return sm[0] + sm[1] + sm[2] + sm[3];
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

// The momentum's step, and a workgroup's share of |u|^2.
template <typename G>
__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonArgs a) {
  __shared__ double sm[4];
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_flat; });
  const uint32_t at = blockIdx.x - q.tile_flat, i = at / q.n_flat, part = at - i * q.n_flat;
  const MuonEntry& en = a.table[q.entry + i];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int64_t n = (int64_t)q.rows * q.cols;
  const int64_t share = ((n + q.n_flat - 1) / q.n_flat + 1023) / 1024 * 1024;
  const int64_t from = part * share, to = from + share < n ? from + share : n;
  float* const mt = en.m;
  const G* const gt = (const G*)en.g;
  double sq = 0;
  for (int64_t k = from + threadIdx.x * 4; k < to; k += 1024) {
    float m[4], g[4];
    const int c = to - k < 4 ? (int)(to - k) : 4;
    load4(mt + k, c, m);
    load4(gt + k, c, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      g[e] *= gs;
      m[e] = momentum_of(a, m[e], g[e]);
      const float u = update_of(a, m[e], g[e]);
      if (e < c) sq += (double)u * (double)u;
    }
    store4(mt + k, c, m);
  }
  sq = block_sum(sq, sm);
  if (threadIdx.x == 0) reinterpret_cast<double*>(q.base + i * q.stride + q.norm)[part] = sq;
}

template <bool PAIRS>
__device__ inline void put_halves(_Float16* hi, int64_t lo, float x) {  // lo: bytes
  const _Float16 h = (_Float16)x;
  *hi = h;
  if (PAIRS) *reinterpret_cast<_Float16*>(reinterpret_cast<char*>(hi) + lo) = (_Float16)(x - (float)h);
}
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
template <bool PAIRS>
__device__ inline void put_halves4(_Float16* hi, int64_t lo, const float (&x)[4]) {
  half4 h, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = (_Float16)x[e];
    l[e] = (_Float16)(x[e] - (float)h[e]);
  }
  *reinterpret_cast<half4*>(hi) = h;
  if (PAIRS) *reinterpret_cast<half4*>(reinterpret_cast<char*>(hi) + lo) = l;
}
template <bool PAIRS>
__device__ inline void get_halves4(const _Float16* hi, int64_t lo, float (&x)[4]) {
  const half4 h = *reinterpret_cast<const half4*>(hi);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = (float)h[e];
  if (PAIRS) {
    const half4 l = *reinterpret_cast<const half4*>(reinterpret_cast<const char*>(hi) + lo);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += (float)l[e];
  }
}

// u / |u| as halves, its longer side first: 64 x 64 elements of the matrix a workgroup, turned
// in LDS where the columns are the longer side.  Columns from S to ld are zeros.
template <typename G, bool PAIRS>
__global__ __launch_bounds__(256) void muon_split_kernel(MuonArgs a) {
  __shared__ double sm[4];
  __shared__ float tile[64][65];
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_turn; });
  const uint32_t at = blockIdx.x - q.tile_turn, i = at / q.n_turn, t = at - i * q.n_turn;
  const MuonEntry& en = a.table[q.entry + i];
  char* const base = q.base + i * q.stride;
  const double* const norm = reinterpret_cast<const double*>(base + q.norm);
  const double total = block_sum(threadIdx.x < q.n_flat ? norm[threadIdx.x] : 0.0, sm);
  const double inv = (double)kScale * inverse_norm(total);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const uint32_t across = (uint32_t)q.ld / 64;  // Y's tiles in a row
  const int l0 = (int)(t / across) * 64, s0 = (int)(t - t / across * across) * 64;
  const bool turned = q.rows < q.cols;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  _Float16* const y = reinterpret_cast<_Float16*>(base + q.y[0]);
#pragma unroll 4
  for (int k = wave; k < 64; k += 4) {
    const int r = turned ? s0 + k : l0 + k, c = turned ? l0 + lane : s0 + lane;
    float x = 0.f;
    if (r < q.rows && c < q.cols) {
      const int64_t e = (int64_t)r * q.cols + c;
      const float g = (float)((const G*)en.g)[e] * gs;
      x = (float)((double)update_of(a, en.m[e], g) * inv);
    }
    if (turned) tile[lane][k] = x;
    else tile[k][lane] = x;
  }
  __syncthreads();
#pragma unroll 4
  for (int k = wave * 4 + lane / 16; k < 64; k += 16) {
    if (l0 + k >= q.L) continue;
    const int s = (lane & 15) * 4;
    const float x[4] = {tile[k][s], tile[k][s + 1], tile[k][s + 2], tile[k][s + 3]};
    put_halves4<PAIRS>(y + (int64_t)(l0 + k) * q.ld + s0 + s, q.lo_y, x);
  }
}

// ----------------------------------------------------------------------------
// 128 x 128 tiles of a product, K in stages of 64
// ----------------------------------------------------------------------------
constexpr int MT = kMuonTile;
constexpr uint32_t M_SLOT = MT * 128;  // bytes of an operand's stage
struct MuonSmem {
  i32x4 a[2][MT * 8];
  i32x4 b[2][MT * 8];
};

template <int N>
__device__ inline void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Four waves (2 x 2) hold 64 x 64 each, as 4 x 4 accumulators.  C[m][n] += sum_k A[m][k] B[n][k];
// KMAJOR: of operands stored [k][m] and [k][n].  Stages go straight to LDS, one ahead.
template <bool KMAJOR>
struct MuonCore {
  f32x4 acc[4][4];

  __device__ inline void zero() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // n_st stages; da and db start at the tile's first row (KMAJOR: column), ld is both
  // operands' row stride.  What is past a descriptor's range reads as zeros.
  __device__ inline void run(MuonSmem& sm, const i32x4& da_, const i32x4& db_, int32_t ld, int n_st) {
    const i32x4 da = uniform_desc(da_), db = uniform_desc(db_);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63;
    const int wm = wave >> 1, wn = wave & 1;
    // loads: instruction h (0..3) of a wave fills 1 KB of the operand's stage: eight rows of 64
    // values, or (KMAJOR) four K-rows of 128
    uint32_t off[4];
    if constexpr (KMAJOR) {
      const int lr = lane >> 4, s = lane & 15;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int row = 16 * wave + 4 * h + lr;
        const int c = (((s >> 1) ^ swz(row)) << 1) | (s & 1);
        off[h] = (uint32_t)(row * ld * 2 + c * 16) - 1024u * (uint32_t)h;
      }
    } else {
      const int lr = lane >> 3, c = (lane & 7) ^ lr;
#pragma unroll
      for (int h = 0; h < 4; ++h)
        off[h] = (uint32_t)((32 * wave + 8 * h + lr) * ld * 2 + c * 16) - 1024u * (uint32_t)h;
    }
    const uint32_t step = KMAJOR ? (uint32_t)(64 * ld * 2) : 128u;
    const uint32_t sa = (uint32_t)(uintptr_t)&sm.a[0][0], sb = (uint32_t)(uintptr_t)&sm.b[0][0];
    const uint32_t lds_a = sa + (uint32_t)wave * 4096u, lds_b = sb + (uint32_t)wave * 4096u;
    auto issue = [&](int st) {
      const bool live = st < n_st;
      const uint32_t slot = (uint32_t)(st & 1) * M_SLOT;
      const i32x4 xa = desc_at(da, (uint32_t)st * step, live), xb = desc_at(db, (uint32_t)st * step, live);
      set_m0(lds_a + slot);
      lds_dma16_m0<0>(xa, off[0]);
      lds_dma16_m0<1024>(xa, off[1]);
      lds_dma16_m0<2048>(xa, off[2]);
      lds_dma16_m0<3072>(xa, off[3]);
      set_m0(lds_b + slot);
      lds_dma16_m0<0>(xb, off[0]);
      lds_dma16_m0<1024>(xb, off[1]);
      lds_dma16_m0<2048>(xb, off[2]);
      lds_dma16_m0<3072>(xb, off[3]);
    };
    const int ri = lane & 15, rg = lane >> 4;
    auto frag = [&](uint32_t base, int half, int t, int hk) -> i32x4 {  // block t of the operand's half, K-half hk
      if constexpr (KMAJOR) {
        const int gl = (ri >> 2) | ((rg & 1) << 2);
        const uint32_t at = base + (uint32_t)(32 * hk + 8 * rg + (ri >> 2)) * 256u + 32u * (uint32_t)((4 * half + t) ^ gl) +
                            8u * (uint32_t)(ri & 3);
        const i32x2 lo = read_tr(at), hi = read_tr(at + 4u * 256u);
        return i32x4{lo.x, lo.y, hi.x, hi.y};
      } else {
        const uint32_t at = base + (uint32_t)(64 * half + 16 * t + ri) * 128u + 16u * (uint32_t)((4 * hk + rg) ^ (ri & 7));
        return *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>((uintptr_t)at);
      }
    };
    issue(0);
    for (int st = 0; st < n_st; ++st) {
      wait_vm<0>();   // stage st has landed
      wait_lgkm0();   // this wave has read stage st - 1
      __builtin_amdgcn_s_barrier();
      issue(st + 1);  // past the end nothing is fetched
      const uint32_t slot = (uint32_t)(st & 1) * M_SLOT;
#pragma unroll
      for (int hk = 0; hk < 2; ++hk) {
        i32x4 fa[4], fb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) fb[t] = frag(sb + slot, wn, t, hk);
#pragma unroll
        for (int t = 0; t < 4; ++t) fa[t] = frag(sa + slot, wm, t, hk);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = mma16(F16Tag{}, fa[i], fb[j], acc[i][j]);
      }
    }
    wait_vm<0>();
    wait_lgkm0();
    __builtin_amdgcn_s_barrier();
  }

  __device__ static inline int swz(int r) { return (r & 3) | (((r >> 3) & 1) << 2); }
  __device__ static inline i32x2 read_tr(uint32_t at) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at);
    return __builtin_bit_cast(i32x2, v);
  }
  // First row (of four) and column of accumulator (i, j).
  __device__ static inline int row_of(int i) {
    return 64 * (int)(threadIdx.x >> 7) + 16 * i + 4 * (int)((threadIdx.x & 63) >> 4);
  }
  __device__ static inline int col_of(int j) { return 64 * (int)((threadIdx.x >> 6) & 1) + 16 * j + (int)(threadIdx.x & 15); }
};

// Descriptor of rows [r0, rows) of a matrix with row stride ld halves.
__device__ inline i32x4 rows_desc(const char* p, int32_t ld, int32_t r0, int32_t rows) {
  const int32_t n = rows - r0 < MT ? rows - r0 : MT;
  return make_desc(p + (int64_t)r0 * ld * 2, (uint32_t)n * (uint32_t)ld * 2u);
}
// Descriptor of a matrix of `rows` K-rows from column c0.
__device__ inline i32x4 cols_desc(const char* p, int32_t ld, int32_t c0, int32_t rows) {
  return make_desc(p + c0 * 2, ((uint32_t)rows * (uint32_t)ld - (uint32_t)c0) * 2u);
}

// Tile t of the upper triangle of an n x n grid of tiles, by columns: (0,0) (0,1) (1,1) (0,2) ...
__device__ inline void upper_tile(uint32_t t, int& ti, int& tj) {
  int j = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
  while ((uint32_t)(j + 1) * (uint32_t)(j + 2) / 2 <= t) ++j;
  while ((uint32_t)j * (uint32_t)(j + 1) / 2 > t) --j;
  tj = wave_uniform(j);
  ti = wave_uniform((int)(t - (uint32_t)j * (uint32_t)(j + 1) / 2));
}

// Writes a symmetric matrix's tile and its mirror image; columns from S to ld are zeros.
// value(row, col, sum): what is stored.
template <bool PAIRS, typename F>
__device__ inline void put_symmetric(const MuonGroup& q, char* to, int ti, int tj, const f32x4 (&acc)[4][4], F value) {
  _Float16* const o = reinterpret_cast<_Float16*>(to);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = ti * MT + MuonCore<false>::row_of(i), c = tj * MT + MuonCore<false>::col_of(j);
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = r + e < q.S && c < q.S ? value(r + e, c, acc[i][j][e]) : 0.f;
      if (c < q.S && r < q.ld) put_halves4<PAIRS>(o + (int64_t)c * q.ld + r, q.lo_s, x);
      if (ti == tj) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (r + e < q.S && c < q.ld) put_halves<PAIRS>(o + (int64_t)(r + e) * q.ld + c, q.lo_s, x[e]);
    }
}

template <bool PAIRS, bool KMAJOR, typename Desc>
__device__ inline void products(MuonCore<KMAJOR>& core, MuonSmem& sm, int32_t ld, int n_st, int64_t lo_a, int64_t lo_b, Desc desc) {
  core.zero();
  core.run(sm, desc(0, (int64_t)0), desc(1, (int64_t)0), ld, n_st);
  if (PAIRS) {
    core.run(sm, desc(0, (int64_t)0), desc(1, lo_b), ld, n_st);
    core.run(sm, desc(0, lo_a), desc(1, (int64_t)0), ld, n_st);
  }
}

// A = Y^T Y
template <bool PAIRS>
__global__ __launch_bounds__(256, 2) void muon_gram_kernel(MuonArgs a, int from) {
  __shared__ MuonSmem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_sym; });
  const uint32_t at = blockIdx.x - q.tile_sym, i = wave_uniform(at / q.n_sym);
  char* const base = q.base + i * q.stride;
  int ti, tj;
  upper_tile(at - i * q.n_sym, ti, tj);
  MuonCore<true> core;
  products<PAIRS>(core, sm, q.ld, (q.L + 63) / 64, q.lo_y, q.lo_y, [&](int b, int64_t lo) {
    return cols_desc(base + q.y[from] + lo, q.ld, (b ? tj : ti) * MT, q.L);
  });
  put_symmetric<PAIRS>(q, base + q.gram, ti, tj, core.acc,
                       [](int, int, float v) { return v * (1.f / kScale); });
}

// B = b A + c A A
template <bool PAIRS>
__global__ __launch_bounds__(256, 2) void muon_poly_kernel(MuonArgs a) {
  __shared__ MuonSmem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_sym; });
  const uint32_t at = blockIdx.x - q.tile_sym, i = wave_uniform(at / q.n_sym);
  char* const base = q.base + i * q.stride;
  int ti, tj;
  upper_tile(at - i * q.n_sym, ti, tj);
  MuonCore<false> core;
  products<PAIRS>(core, sm, q.ld, q.ld / 64, q.lo_s, q.lo_s, [&](int b, int64_t lo) {
    return rows_desc(base + q.gram + lo, q.ld, (b ? tj : ti) * MT, q.S);
  });
  const _Float16* const g = reinterpret_cast<const _Float16*>(base + q.gram);
  put_symmetric<PAIRS>(q, base + q.poly, ti, tj, core.acc, [&](int r, int c, float v) {
    const _Float16* const p = g + (int64_t)c * q.ld + r;  // A is symmetric
    float x = (float)*p;
    if (PAIRS) x += (float)*reinterpret_cast<const _Float16*>(reinterpret_cast<const char*>(p) + q.lo_s);
    return x * (kNsB * kScalePoly / kScale) + v * (kNsC * kScalePoly / (kScale * kScale));
  });
}

// Sums of B Y^T's tile (rows: Y's columns, columns: Y's rows), and Y's new values from them.
template <bool PAIRS>
__device__ inline void apply_tile(const MuonGroup& q, char* base, int from, int ts, int tl, MuonCore<false>& core, MuonSmem& sm) {
  products<PAIRS>(core, sm, q.ld, q.ld / 64, q.lo_s, q.lo_y, [&](int b, int64_t lo) {
    return b ? rows_desc(base + q.y[from] + lo, q.ld, tl * MT, q.L)
             : rows_desc(base + q.poly + lo, q.ld, ts * MT, q.S);
  });
}
template <bool PAIRS>
__device__ inline void new_y(const MuonGroup& q, const _Float16* y, const f32x4& sum, float (&x)[4]) {
  get_halves4<PAIRS>(y, q.lo_y, x);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = kNsA * x[e] + sum[e] * (1.f / kScalePoly);
}
__device__ inline void full_tile(const MuonGroup& q, uint32_t at, uint32_t& i, int& ts, int& tl) {
  i = wave_uniform(at / q.n_full);
  const uint32_t t = at - i * q.n_full, across = (uint32_t)(q.S + MT - 1) / MT;
  tl = wave_uniform((int)(t / across));
  ts = (int)(t - (uint32_t)tl * across);
}

// Y = a Y + Y B, into the other buffer
template <bool PAIRS>
__global__ __launch_bounds__(256, 2) void muon_apply_kernel(MuonArgs a, int from) {
  __shared__ MuonSmem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_full; });
  uint32_t i;
  int ts, tl;
  full_tile(q, blockIdx.x - q.tile_full, i, ts, tl);
  char* const base = q.base + i * q.stride;
  MuonCore<false> core;
  apply_tile<PAIRS>(q, base, from, ts, tl, core, sm);
  const _Float16* const y = reinterpret_cast<const _Float16*>(base + q.y[from]);
  _Float16* const o = reinterpret_cast<_Float16*>(base + q.y[1 - from]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int l = tl * MT + core.col_of(j);
    if (l >= q.L) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = ts * MT + core.row_of(k);
      if (s >= q.ld) continue;
      float x[4];
      new_y<PAIRS>(q, y + (int64_t)l * q.ld + s, core.acc[k][j], x);
      put_halves4<PAIRS>(o + (int64_t)l * q.ld + s, q.lo_y, x);
    }
  }
}

// The last product and the weights' step.
template <bool PAIRS, typename P, bool MASTER>
__global__ __launch_bounds__(256, 2) void muon_last_kernel(MuonArgs a, int from) {
  __shared__ MuonSmem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_full; });
  uint32_t i;
  int ts, tl;
  full_tile(q, blockIdx.x - q.tile_full, i, ts, tl);
  char* const base = q.base + i * q.stride;
  MuonCore<false> core;
  apply_tile<PAIRS>(q, base, from, ts, tl, core, sm);
  const _Float16* const y = reinterpret_cast<const _Float16*>(base + q.y[from]);
  const MuonEntry& en = a.table[q.entry + i];
  P* const p = (P*)en.p;
  const float lr = en.lr, lr_wd = en.lr_wd;
  const bool turned = q.rows < q.cols;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int l = tl * MT + core.col_of(j);
    if (l >= q.L) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = ts * MT + core.row_of(k);
      if (s >= q.S) continue;
      float x[4];
      new_y<PAIRS>(q, y + (int64_t)l * q.ld + s, core.acc[k][j], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (s + e >= q.S) continue;
        const int64_t at = turned ? (int64_t)(s + e) * q.cols + l : (int64_t)l * q.cols + s + e;
        const float w = MASTER ? en.master[at] : (float)p[at];
        const float nw = stepped(w, x[e] * (1.f / kScale), lr, lr_wd);
        if (MASTER) en.master[at] = nw;
        p[at] = (P)nw;
      }
    }
  }
}

template <typename F>
hipError_t with_pairs(bool pairs, F f) {
  if (pairs) f(std::true_type{});
  else f(std::false_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_muon_table(const MuonTable& t, hipStream_t s) {
  hipLaunchKernelGGL(muon_table_kernel, dim3(1), dim3(64), 0, s, t);
  return hipGetLastError();
}
hipError_t launch_muon_momentum(int g_dtype, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_type(g_dtype, [&](auto g) {
    hipLaunchKernelGGL((muon_momentum_kernel<decltype(g)>), dim3(blocks), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}
hipError_t launch_muon_split(int g_dtype, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_type(g_dtype, [&](auto g) {
    return with_pairs(pairs, [&](auto pr) {
      hipLaunchKernelGGL((muon_split_kernel<decltype(g), decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a);
    });
  });
}
hipError_t launch_muon_gram(bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_pairs(pairs, [&](auto pr) {
    hipLaunchKernelGGL((muon_gram_kernel<decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a, from);
  });
}
hipError_t launch_muon_poly(bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_pairs(pairs, [&](auto pr) {
    hipLaunchKernelGGL((muon_poly_kernel<decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a);
  });
}
hipError_t launch_muon_apply(bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_pairs(pairs, [&](auto pr) {
    hipLaunchKernelGGL((muon_apply_kernel<decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a, from);
  });
}
hipError_t launch_muon_last(bool pairs, int p_dtype, bool master, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_type(p_dtype, [&](auto p) {
    typedef decltype(p) T;
    return with_pairs(pairs, [&](auto pr) {
      if (master) hipLaunchKernelGGL((muon_last_kernel<decltype(pr)::value, T, true>), dim3(blocks), dim3(256), 0, s, a, from);
      else hipLaunchKernelGGL((muon_last_kernel<decltype(pr)::value, T, false>), dim3(blocks), dim3(256), 0, s, a, from);
    });
  });
}

}  // namespace attr
