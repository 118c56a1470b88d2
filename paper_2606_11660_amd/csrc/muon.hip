// One Muon step over many matrices (attr_muon_step).
//
//     m = mu m + (1 - mu) g',   u = mu m + (1 - mu) g' (nesterov) or m
//     X = u / |u|_F;  five times:  A = X X^T,  B = a I + b A + c A^2,  X = B X
//     w = w - lr wd w - lr X
//
// Bound by the matrix cores: with s and t a matrix's shorter and longer side, s^2 t + s^3 +
// 2 s^2 t flops a step of the iteration, since A and B are symmetric and only their upper
// triangles of tiles are computed.  The iteration holds Y, the update with its longer side
// first ([t][s]; A = Y^T Y, Y = Y B), so that Y is stored once and in one order: A reads
// it along its columns (transposing LDS reads), Y B along its rows.
//
// Operands are fp16 with powers of two before them: no entry of X passes 1.21, of A 1.45 or of
// B 3.45 (|p(x)| <= 1.2025 on [0, 1.2025] for p = a x + b x^3 + c x^5), so 2^15 X, 2^15 A and
// 2^14 B fit, and what is below 2^-24 of the largest entry is still held.  fp16 keeps 11 bits where
// bf16 keeps 8, at the same rate.  With pairs every operand is two fp16 values (22 bits) and a
// product three: hi hi + hi lo + lo hi.  Sums are fp32, the norm's fp64.
#include "gemm.h"
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

// The momentum's step, and a workgroup's share of |u|^2: 10 bytes an element with 16-bit gradients, bound
// by HBM (14 matrices of 134M elements in all: 258 us, 5.2 TB/s).
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
// u is computed a second time from what the first pass left (6 bytes an element read and 2 written, where
// keeping it would write and read 4 more; the same matrices: 247 us, 4.3 TB/s).
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
  // four neighbouring elements of the matrix a lane
  const int r0 = turned ? s0 : l0, c = (turned ? l0 : s0) + lane % 16 * 4;
  const int n = q.cols - c;
#pragma unroll
  for (int k = wave * 4 + lane / 16; k < 64; k += 16) {
    const int r = r0 + k;
    float m[4] = {0.f, 0.f, 0.f, 0.f}, g[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < q.rows && n > 0) {
      const int64_t e = (int64_t)r * q.cols + c;
      load4(en.m + e, n, m);
      load4((const G*)en.g + e, n, g);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = (float)((double)update_of(a, m[e], g[e] * gs) * inv);
      const float there = r < q.rows && e < n ? x : 0.f;
      if (turned) tile[lane % 16 * 4 + e][k] = there;
      else tile[k][lane % 16 * 4 + e] = there;
    }
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
// 128 x 128 tiles of a product
// ----------------------------------------------------------------------------
constexpr int MT = kMuonTile;
constexpr uint32_t M_SLOT = MT * 128;  // bytes of an operand's stage
struct MuonSmem {
  i32x4 a[2][MT * 8];
  i32x4 b[2][MT * 8];
};

// Four waves (2 x 2) hold 64 x 64 each, as 4 x 4 accumulators.  C[m][n] += sum_k A[m][k] B[n][k];
// KMAJOR: of operands stored [k][m] and [k][n].  Stages (K = 64, or with PAIRS 32 of both halves)
// go straight to LDS, one ahead of the one whose fragments are read, which is one ahead of the
// products; two workgroups a CU fill each other's waits (four slots and one workgroup: the products
// A of 14 matrices in 75 us, so in 66).  A wave whose rows or columns are past the matrix (rows,
// cols: what is left of it from the tile on) only loads.  With PAIRS the three products of a stage
// share their fragments: 16 reads for 48 products, where three passes took 24.
template <bool KMAJOR, bool PAIRS>
struct MuonCore {
  static constexpr int F = 4;  // 16 x 16 accumulators of a wave each way
  typedef MuonSmem Smem;
  f32x4 acc[F][F];

  // K in n_k rows (KMAJOR) or values; ao and bo: the operands' first halves from the tile's first
  // row (KMAJOR: column), ld both operands' row stride, a_lo and b_lo the second halves'
  // descriptors.  What is past a descriptor's range reads as zeros.
  __device__ inline void product(Smem& sm, const i32x4& a_hi_, const i32x4& a_lo_, const i32x4& b_hi_, const i32x4& b_lo_,
                                 int32_t ld, int n_k, int rows, int cols) {
    const i32x4 a_hi = uniform_desc(a_hi_), a_lo = uniform_desc(a_lo_), b_hi = uniform_desc(b_hi_), b_lo = uniform_desc(b_lo_);
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int KS = PAIRS ? 32 : 64;
    const int n_st = (n_k + KS - 1) / KS;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63;
    const int wm = wave >> 1, wn = wave & 1;
    // loads: an instruction fills 1 KB of a stage, four of them an operand's share of a wave:
    //   rows of K            eight rows of 64 values; PAIRS: 16 rows of 32, of each half
    //   KMAJOR               four K-rows of 128 values
    // The 16-byte pieces of a row (KMAJOR: 32-byte pieces) change places by row, so that the
    // fragment reads of 16 lanes meet distinct banks.
    uint32_t off[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int part = PAIRS ? h & 1 : h, first = PAIRS ? 2 * wave + part : 4 * wave + part;  // of the KBs of a half
      if constexpr (KMAJOR) {
        const int row = 4 * first + (lane >> 4), s = lane & 15;
        off[h] = (uint32_t)(row * ld * 2 + (((((s >> 1) ^ swz(row)) << 1) | (s & 1)) * 16));
      } else if constexpr (PAIRS) {
        const int row = 16 * first + (lane >> 2);
        off[h] = (uint32_t)(row * ld * 2 + (((lane & 3) ^ ((row >> 1) & 3)) * 16));
      } else {
        const int row = 8 * first + (lane >> 3);
        off[h] = (uint32_t)(row * ld * 2 + (((lane & 7) ^ (row & 7)) * 16));
      }
      off[h] -= 1024u * (uint32_t)(h & 1);
    }
    const uint32_t step = KMAJOR ? (uint32_t)(KS * ld * 2) : 2u * KS;
    const uint32_t sa = (uint32_t)(uintptr_t)&sm.a[0][0], sb = (uint32_t)(uintptr_t)&sm.b[0][0];
    // group g (0..3) of stage st's loads: A's and B's, two KB of the wave's four at a time
    const auto issue = [&](int st, int g) {
      const bool live = st < n_st;  // past the end nothing is fetched
      const uint32_t lds = (g < 2 ? sa : sb) + (uint32_t)(st & 1) * M_SLOT, ko = (uint32_t)st * step;
      const int h = g & 1;
      const i32x4 d = desc_at(PAIRS && h ? (g < 2 ? a_lo : b_lo) : (g < 2 ? a_hi : b_hi), ko, live);
      if constexpr (PAIRS) {
        set_m0(lds + (uint32_t)h * (M_SLOT / 2) + (uint32_t)wave * 2048u);
        lds_dma16_m0<0>(d, off[2 * h]);
        lds_dma16_m0<1024>(d, off[2 * h + 1]);
      } else {
        set_m0(lds + (uint32_t)wave * 4096u + (uint32_t)h * 2048u);
        lds_dma16_m0<0>(d, off[2 * h]);
        lds_dma16_m0<1024>(d, off[2 * h + 1]);
      }
    };
    const int ri = lane & 15, rg = lane >> 4;
    const auto frag = [&](uint32_t base, int half, int t, int hk) -> i32x4 {  // block t of the operand's half, K-half hk
      if constexpr (KMAJOR) {
        const int gl = (ri >> 2) | ((rg & 1) << 2);
        const uint32_t at = base + (uint32_t)(32 * hk + 8 * rg + (ri >> 2)) * 256u + 32u * (uint32_t)((4 * half + t) ^ gl) +
                            8u * (uint32_t)(ri & 3);
        const i32x2 lo = lds_read_tr16(at), hi = lds_read_tr16(at + 4u * 256u);
        return i32x4{lo.x, lo.y, hi.x, hi.y};
      } else {
        const uint32_t row = (uint32_t)(64 * half + 16 * t + ri);
        const uint32_t at = PAIRS ? base + row * 64u + 16u * (uint32_t)(rg ^ ((ri >> 1) & 3))
                                  : base + row * 128u + 16u * (uint32_t)((4 * hk + rg) ^ (ri & 7));
        return *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>((uintptr_t)at);
      }
    };
    // A stage's fragments: the two K-halves, or with PAIRS the two halves of the values.  While one
    // stage's are multiplied the next one's are read.
    struct Frags {
      i32x4 a[2][F], b[2][F];
    } even, odd;
    const auto read = [&](int st, int n, Frags& f) {  // n (0..7): two fragments, B's before A's
      const uint32_t base = (n & 2 ? sa : sb) + (uint32_t)(st & 1) * M_SLOT + (PAIRS ? (uint32_t)(n >> 2) * (M_SLOT / 2) : 0u);
      const int h = n >> 2, t = 2 * (n & 1);
      i32x4(&to)[F] = n & 2 ? f.a[h] : f.b[h];
#pragma unroll
      for (int k = 0; k < 2; ++k) to[t + k] = frag(base, n & 2 ? wm : wn, t + k, PAIRS ? 0 : h);
    };
    const bool there = rows > 64 * wm && cols > 64 * wn;  // something of the wave's
    constexpr int PRODUCTS = PAIRS ? 3 : 2;
    const auto stage = [&](int st, const Frags& cur, Frags& next) {
      gemm_wait_vm<0>();  // stage st + 1 has landed
      wait_lgkm0();       // this wave has read stage st, whose slot is free behind the barrier
      __builtin_amdgcn_s_barrier();
      if (there) {
#pragma unroll
        for (int r = 0; r < PRODUCTS * F; ++r) {  // a row of four products, two reads and two loads at a time
          const int p = r / F, i = r % F;
          if (r < 8) read(st + 1, r, next);
          if (r < 4) issue(st + 2, r);
          __builtin_amdgcn_sched_barrier(0);
          const i32x4(&x)[F] = cur.a[PAIRS ? p == 2 : p];
          const i32x4(&y)[F] = cur.b[PAIRS ? p == 1 : p];
#pragma unroll
          for (int j = 0; j < F; ++j) acc[i][j] = mma16(F16Tag{}, x[i], y[j], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) issue(st + 2, g);
      }
    };
#pragma unroll
    for (int k = 0; k < 8; ++k) issue(k / 4, k % 4);
    gemm_wait_vm<8>();
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int n = 0; n < 8; ++n) read(0, n, even);
    for (int st = 0; st < n_st; st += 2) {
      stage(st, even, odd);
      if (st + 1 < n_st) stage(st + 1, odd, even);
    }
    gemm_wait_vm<0>();
    wait_lgkm0();
    __builtin_amdgcn_s_barrier();
  }
  __device__ static inline int swz(int r) { return (r & 3) | (((r >> 3) & 1) << 2); }
};

// The same of 256 x 256 tiles, through the block-tile cores: one workgroup a CU, 128 x 128 a wave,
// which halves the LDS reads of a product.  PAIRS: the three products one after another.
template <bool KMAJOR, bool PAIRS>
struct MuonCoreBig : std::conditional<KMAJOR, GemmCoreT<F16Tag>, GemmCore<F16Tag>>::type {
  static constexpr int F = 8;
  typedef GemmSmem Smem;

  __device__ inline void product(GemmSmem& sm, const i32x4& a_hi, const i32x4& a_lo, const i32x4& b_hi, const i32x4& b_lo,
                                 int32_t ld, int n_k, int, int) {
    const int n_st = (n_k + 63) / 64;
    this->zero();
    i32x4 da = uniform_desc(a_hi), db = uniform_desc(b_hi);
#pragma unroll 1
    for (int k = 0;; ++k) {
      if constexpr (KMAJOR) this->run(sm, da, db, ld, n_st);
      else this->run(sm, da, ld, db, ld, n_st);
      if (!PAIRS || k == 2) break;
      da = uniform_desc(k == 1 ? a_lo : a_hi);
      db = uniform_desc(k == 0 ? b_lo : b_hi);
    }
  }
};

template <bool BIG, bool KMAJOR, bool PAIRS>
struct CoreOf {
  typedef typename std::conditional<BIG, MuonCoreBig<KMAJOR, PAIRS>, MuonCore<KMAJOR, PAIRS>>::type type;
  static constexpr int tile = BIG ? 256 : 128;
};

// Descriptor of rows [r0, rows) of a matrix with row stride ld halves, of a tile.
template <int TILE>
__device__ inline i32x4 rows_desc(const char* p, int32_t ld, int32_t r0, int32_t rows) {
  const int32_t n = rows - r0 < TILE ? rows - r0 : TILE;
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

// A workgroup's tile of a group of n: workgroups go to the eight dies in turn, and each die takes
// an eighth of the tiles, one after another, so that the operands' panels that neighbouring tiles
// share are in its own L2.  False: the group has no such tile (its workgroups are rounded up).
__device__ inline bool tile_of(uint32_t block, uint32_t n, uint32_t& tile) {
  tile = (block & 7) * ((n + 7) / 8) + block / 8;
  return block / 8 < (n + 7) / 8 && tile < n;
}

// ----------------------------------------------------------------------------
// a tile's way out
// ----------------------------------------------------------------------------
// A wave's 16F x 16F sums go through its own part of LDS, 32 of C's columns at a time, so that
// memory is read and written in runs of rows: eight neighbouring rows m of one column n in a
// lane, or eight columns n of one row m.
template <int F>
struct Stage {
  static constexpr int W = 16 * F, PITCH = W + 4, LANES = W / 8, PER = 64 / LANES;
  float* st;
  int lane;
  static constexpr int FLOATS = 32 * PITCH;  // of a wave
  __device__ inline Stage(void* smem) {
    st = reinterpret_cast<float*>(smem) + wave_uniform((int)(threadIdx.x >> 6)) * FLOATS;
    lane = threadIdx.x & 63;
  }
  // Columns 32 jp .. 32 jp + 31 of the wave's sums.
  __device__ inline void put(const f32x4 (&acc)[F][F], int jp) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int i = 0; i < F; ++i)
        *reinterpret_cast<f32x4*>(st + (16 * jj + (lane & 15)) * PITCH + 16 * i + 4 * (lane >> 4)) = acc[i][2 * jp + jj];
  }
  // Eight rows from m() of column n(k), k below 32 / PER.
  __device__ inline int n(int k) const { return k * PER + lane / LANES; }
  __device__ inline int m() const { return lane % LANES * 8; }
  __device__ inline void get(int k, float (&x)[8]) const {
    const f32x4* p = reinterpret_cast<const f32x4*>(st + n(k) * PITCH + m());
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = p[h][e];
  }
  __device__ inline void keep(int k, const float (&x)[8]) {
    f32x4* p = reinterpret_cast<f32x4*>(st + n(k) * PITCH + m());
#pragma unroll
    for (int h = 0; h < 2; ++h) p[h] = f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
  }
  // Eight columns from tn() of row tm(k), k below F.
  __device__ inline int tn() const { return lane % 4 * 8; }
  __device__ inline int tm(int k) const { return k * 16 + lane / 4; }
  __device__ inline void turned(int k, float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = st[(tn() + e) * PITCH + tm(k)];
  }
};
// First row and column of a wave's sums within its tile.
__device__ inline int this_wave() { return (int)wave_uniform(threadIdx.x >> 6); }
template <int F>
__device__ inline int wave_row(int wave = this_wave()) { return 16 * F * (wave >> 1); }
template <int F>
__device__ inline int wave_col(int wave = this_wave()) { return 16 * F * (wave & 1); }

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
template <bool PAIRS>
__device__ inline void put_halves8(_Float16* hi, int64_t lo, const float (&x)[8]) {
  half8 h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = (_Float16)x[e];
    l[e] = (_Float16)(x[e] - (float)h[e]);
  }
  *reinterpret_cast<half8*>(hi) = h;
  if (PAIRS) *reinterpret_cast<half8*>(reinterpret_cast<char*>(hi) + lo) = l;
}
template <bool PAIRS>
__device__ inline void get_halves8(const _Float16* hi, int64_t lo, float (&x)[8]) {
  const half8 h = *reinterpret_cast<const half8*>(hi);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  if (PAIRS) {
    const half8 l = *reinterpret_cast<const half8*>(reinterpret_cast<const char*>(hi) + lo);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += (float)l[e];
  }
}

// A symmetric matrix's tile and its mirror image; columns from S to ld are zeros.  value(r, c, x)
// turns the sums of eight rows from r of column c into what is stored.
template <bool PAIRS, int F, typename V>
__device__ inline void put_symmetric(const MuonGroup& q, char* to, void* smem, int ti, int tj, const f32x4 (&acc)[F][F], V value,
                                     int wave = this_wave()) {
  _Float16* const o = reinterpret_cast<_Float16*>(to);
  Stage<F> st(smem);
  const int r0 = ti * 32 * F + wave_row<F>(wave), c0 = tj * 32 * F + wave_col<F>(wave);
#pragma unroll
  for (int jp = 0; jp < F / 2; ++jp) {
    st.put(acc, jp);
#pragma unroll 2
    for (int k = 0; k < 32 / Stage<F>::PER; ++k) {
      const int r = r0 + st.m(), c = c0 + 32 * jp + st.n(k);
      float x[8];
      st.get(k, x);
      if (c < q.S && r < q.ld) value(r, c, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c < q.S && r + e < q.S ? x[e] : 0.f;
      if (c < q.S && r < q.ld) put_halves8<PAIRS>(o + (int64_t)c * q.ld + r, q.lo_s, x);
      if (ti != tj) st.keep(k, x);
    }
    if (ti != tj) {
#pragma unroll 2
      for (int k = 0; k < F; ++k) {
        const int r = r0 + st.tm(k), c = c0 + 32 * jp + st.tn();
        float x[8];
        st.turned(k, x);
        if (r < q.S && c < q.ld) put_halves8<PAIRS>(o + (int64_t)r * q.ld + c, q.lo_s, x);
      }
    }
  }
}

struct AsA {  // a product of X's halves to A's
  __device__ inline void operator()(int, int, float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= 1.f / kScale;
  }
};

// A = Y^T Y, or the sums of a part of Y's rows.  Bound by the matrix cores: 14 matrices of
// 2048 x 2048 and 8192 take 274 us, 1000 TFLOP/s.  Of sizes like 769 and 2310, with pairs, 66 us: whole tiles
// are a third more work than the matrices, and the longest ones end last.
template <bool BIG, bool PAIRS>
__global__ __launch_bounds__(256, BIG ? 1 : 2) void muon_gram_kernel(MuonArgs a, int from) {
  typedef CoreOf<BIG, true, PAIRS> C;
  constexpr int F = C::type::F;
  __shared__ typename C::type::Smem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_gram; });
  const uint32_t each = q.n_sym * q.splits;
  uint32_t at;
  if (!tile_of(blockIdx.x - q.tile_gram, each * q.count, at)) return;
  const uint32_t i = wave_uniform(at / each), part = wave_uniform((at - i * each) / q.n_sym);
  char* const base = q.base + i * q.stride;
  int ti, tj;
  upper_tile(at - i * each - part * q.n_sym, ti, tj);
  const int k0 = (int)part * q.split_rows, n = q.L - k0 < q.split_rows ? q.L - k0 : q.split_rows;
  const char* const y = base + q.y[from] + (int64_t)k0 * q.ld * 2;
  typename C::type core;
  core.product(sm, cols_desc(y, q.ld, ti * C::tile, n), cols_desc(y + q.lo_y, q.ld, ti * C::tile, n),
               cols_desc(y, q.ld, tj * C::tile, n), cols_desc(y + q.lo_y, q.ld, tj * C::tile, n), q.ld, n,
               q.S - ti * C::tile, q.S - tj * C::tile);
  if (q.splits > 1) {
    f32x4* const out = reinterpret_cast<f32x4*>(q.part) + (int64_t)at * (F * F * 256) + threadIdx.x;
#pragma unroll
    for (int k = 0; k < F * F; ++k) out[k * 256] = core.acc[k / F][k % F];
  } else {
    put_symmetric<PAIRS>(q, base + q.gram, &sm, ti, tj, core.acc, AsA());
  }
}

// A from the parts' sums: a workgroup for each wave's quarter of a tile, whose four waves add up every
// fourth part, and then those sums in turn (one wave: 60 us for 32 parts of one tile).
template <bool BIG, bool PAIRS>
__global__ __launch_bounds__(256) void muon_join_kernel(MuonArgs a) {
  constexpr int F = BIG ? 8 : 4;
  __shared__ f32x4 sums[F * F][64];
  __shared__ float sm[Stage<F>::FLOATS];
  const uint32_t block = blockIdx.x / 4, quarter = blockIdx.x % 4;
  const MuonGroup& q = group_of(a, block, [](const MuonGroup& x) { return x.tile_sym; });
  const uint32_t at = block - q.tile_sym;
  if (q.splits < 2 || at >= q.n_sym * q.count) return;
  const uint32_t i = at / q.n_sym, t = at - i * q.n_sym;
  int ti, tj;
  upper_tile(t, ti, tj);
  const int wave = this_wave(), lane = threadIdx.x & 63;
  const f32x4* const from = reinterpret_cast<const f32x4*>(q.part) + ((int64_t)i * q.splits * q.n_sym + t) * (F * F * 256) +
                            quarter * 64 + lane;
  f32x4 acc[F][F];
#pragma unroll
  for (int k = 0; k < F * F; ++k) acc[k / F][k % F] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (uint32_t part = (uint32_t)wave; part < q.splits; part += 4) {
    const f32x4* const p = from + (int64_t)part * q.n_sym * (F * F * 256);
#pragma unroll
    for (int k = 0; k < F * F; ++k) acc[k / F][k % F] += p[k * 256];
  }
  for (int w = 3; w >= 0; --w) {
    if (wave == w) {
#pragma unroll
      for (int k = 0; k < F * F; ++k) {
        if (w < 3) acc[k / F][k % F] += sums[k][lane];
        if (w > 0) sums[k][lane] = acc[k / F][k % F];
      }
    }
    __syncthreads();
  }
  if (wave == 0) put_symmetric<PAIRS>(q, q.base + i * q.stride + q.gram, sm, ti, tj, acc, AsA(), (int)quarter);
}

// B = a I + b A + c A A: 146 us and 816 TFLOP/s there, the shortest of the products
template <bool BIG, bool PAIRS>
__global__ __launch_bounds__(256, BIG ? 1 : 2) void muon_poly_kernel(MuonArgs a) {
  typedef CoreOf<BIG, false, PAIRS> C;
  __shared__ typename C::type::Smem sm;
  const MuonGroup& q = group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_sym; });
  uint32_t at;
  if (!tile_of(blockIdx.x - q.tile_sym, q.n_sym * q.count, at)) return;
  const uint32_t i = wave_uniform(at / q.n_sym);
  char* const base = q.base + i * q.stride;
  int ti, tj;
  upper_tile(at - i * q.n_sym, ti, tj);
  const char* const g = base + q.gram;
  typename C::type core;
  core.product(sm, rows_desc<C::tile>(g, q.ld, ti * C::tile, q.S), rows_desc<C::tile>(g + q.lo_s, q.ld, ti * C::tile, q.S),
           rows_desc<C::tile>(g, q.ld, tj * C::tile, q.S), rows_desc<C::tile>(g + q.lo_s, q.ld, tj * C::tile, q.S), q.ld, q.ld,
               q.S - ti * C::tile, q.S - tj * C::tile);
  put_symmetric<PAIRS>(q, base + q.poly, &sm, ti, tj, core.acc, [&](int r, int c, float(&x)[8]) {
    float v[8];
    get_halves8<PAIRS>(reinterpret_cast<const _Float16*>(g) + (int64_t)c * q.ld + r, q.lo_s, v);  // A is symmetric
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = v[e] * (kNsB * kScalePoly / kScale) + x[e] * (kNsC * kScalePoly / (kScale * kScale));
      if (r + e == c) x[e] += kNsA * kScalePoly;
    }
  });
}

// Sums of B Y^T's tile: rows are Y's columns (s), columns its rows (l).
template <bool BIG, bool PAIRS>
struct ApplyTile {
  typedef CoreOf<BIG, false, PAIRS> C;
  const MuonGroup& q;
  uint32_t i;
  int ts, tl;
  char* base;
  bool there;
  __device__ inline ApplyTile(const MuonArgs& a) : q(group_of(a, blockIdx.x, [](const MuonGroup& x) { return x.tile_full; })) {
    uint32_t at;
    there = tile_of(blockIdx.x - q.tile_full, q.n_full * q.count, at);
    i = wave_uniform(at / q.n_full);
    const uint32_t t = at - i * q.n_full, across = (uint32_t)(q.S + C::tile - 1) / C::tile;
    tl = wave_uniform((int)(t / across));
    ts = wave_uniform((int)(t - (uint32_t)tl * across));
    base = q.base + i * q.stride;
  }
  __device__ inline void run(typename C::type& core, typename C::type::Smem& sm, int from) const {
    const char *y = base + q.y[from], *b = base + q.poly;
    core.product(sm, rows_desc<C::tile>(b, q.ld, ts * C::tile, q.S), rows_desc<C::tile>(b + q.lo_s, q.ld, ts * C::tile, q.S),
             rows_desc<C::tile>(y, q.ld, tl * C::tile, q.L), rows_desc<C::tile>(y + q.lo_y, q.ld, tl * C::tile, q.L), q.ld, q.ld,
             q.S - ts * C::tile, q.L - tl * C::tile);
  }
};

// Y = Y B, into the other buffer: the same matrices take 461 us, 1190 TFLOP/s, where a library product
// of 8192 x 2048 x 2048 reaches 1217.
template <bool BIG, bool PAIRS>
__global__ __launch_bounds__(256, BIG ? 1 : 2) void muon_apply_kernel(MuonArgs a, int from) {
  typedef CoreOf<BIG, false, PAIRS> C;
  constexpr int F = C::type::F;
  __shared__ typename C::type::Smem sm;
  const ApplyTile<BIG, PAIRS> t(a);
  if (!t.there) return;
  const MuonGroup& q = t.q;
  typename C::type core;
  t.run(core, sm, from);
  _Float16* const o = reinterpret_cast<_Float16*>(t.base + q.y[1 - from]);
  Stage<F> st(&sm);
  const int s = t.ts * C::tile + wave_row<F>() + st.m(), l0 = t.tl * C::tile + wave_col<F>();
#pragma unroll
  for (int jp = 0; jp < F / 2; ++jp) {
    st.put(core.acc, jp);
#pragma unroll 2
    for (int k = 0; k < 32 / Stage<F>::PER; ++k) {
      const int l = l0 + 32 * jp + st.n(k);
      if (l >= q.L || s >= q.ld) continue;
      float x[8];
      st.get(k, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= 1.f / kScalePoly;
      put_halves8<PAIRS>(o + (int64_t)l * q.ld + s, q.lo_y, x);
    }
  }
}

// The step of n of eight neighbouring weights from p on.
template <typename P, bool MASTER>
__device__ inline void step8(P* p, float* master, const float (&x)[8], int n, float lr, float lr_wd) {
  if (n >= 8) {
    float w[8];
    if constexpr (MASTER) {
      Raw<float, 8> in;
      in.load(master);
      in.get(w);
    } else {
      Raw<P, 8> in;
      in.load(p);
      in.get(w);
    }
    Raw<P, 8> out;
    Raw<float, 8> wide;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = stepped(w[e], x[e] * (1.f / (kScale * kScalePoly)), lr, lr_wd);
      out.set(e, (P)w[e]);
      if (MASTER) wide.set(e, w[e]);
    }
    if constexpr (MASTER) wide.store(master);
    out.store(p);
  } else {
    for (int e = 0; e < n; ++e) {
      const float w = stepped(MASTER ? master[e] : (float)p[e], x[e] * (1.f / (kScale * kScalePoly)), lr, lr_wd);
      if (MASTER) master[e] = w;
      p[e] = (P)w;
    }
  }
}

// The last product and the weights' step.
template <bool BIG, bool PAIRS, typename P, bool MASTER>
__global__ __launch_bounds__(256, BIG ? 1 : 2) void muon_last_kernel(MuonArgs a, int from) {
  typedef CoreOf<BIG, false, PAIRS> C;
  constexpr int F = C::type::F;
  __shared__ typename C::type::Smem sm;
  const ApplyTile<BIG, PAIRS> t(a);
  if (!t.there) return;
  const MuonGroup& q = t.q;
  typename C::type core;
  t.run(core, sm, from);
  const MuonEntry& en = a.table[q.entry + t.i];
  P* const p = (P*)en.p;
  const float lr = en.lr, lr_wd = en.lr_wd;
  const bool turned = q.rows < q.cols;
  Stage<F> st(&sm);
  const int s0 = t.ts * C::tile + wave_row<F>(), l0 = t.tl * C::tile + wave_col<F>(), s = s0 + st.m();
#pragma unroll
  for (int jp = 0; jp < F / 2; ++jp) {
    st.put(core.acc, jp);
#pragma unroll 2
    for (int k = 0; k < 32 / Stage<F>::PER; ++k) {
      const int l = l0 + 32 * jp + st.n(k);
      if (turned || l >= q.L || s >= q.S) continue;
      float x[8];
      st.get(k, x);
      const int64_t at = (int64_t)l * q.cols + s;
      step8<P, MASTER>(p + at, MASTER ? en.master + at : nullptr, x, q.S - s, lr, lr_wd);
    }
    if (turned) {
#pragma unroll 2
      for (int k = 0; k < F; ++k) {
        const int r = s0 + st.tm(k), l = l0 + 32 * jp + st.tn();
        if (r >= q.S || l >= q.L) continue;
        float x[8];
        st.turned(k, x);
        const int64_t at = (int64_t)r * q.cols + l;
        step8<P, MASTER>(p + at, MASTER ? en.master + at : nullptr, x, q.L - l, lr, lr_wd);
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

// Calls f with big and pairs as types.
template <typename F>
hipError_t with_both(bool big, bool pairs, F f) {
  return with_pairs(pairs, [&](auto pr) {
    if (big) f(std::true_type{}, pr);
    else f(std::false_type{}, pr);
  });
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
hipError_t launch_muon_gram(bool big, bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_both(big, pairs, [&](auto b, auto pr) {
    hipLaunchKernelGGL((muon_gram_kernel<decltype(b)::value, decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a, from);
  });
}
hipError_t launch_muon_join(bool big, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_both(big, pairs, [&](auto b, auto pr) {
    hipLaunchKernelGGL((muon_join_kernel<decltype(b)::value, decltype(pr)::value>), dim3(4 * blocks), dim3(256), 0, s, a);
  });
}
hipError_t launch_muon_poly(bool big, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_both(big, pairs, [&](auto b, auto pr) {
    hipLaunchKernelGGL((muon_poly_kernel<decltype(b)::value, decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a);
  });
}
hipError_t launch_muon_apply(bool big, bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s) {
  return with_both(big, pairs, [&](auto b, auto pr) {
    hipLaunchKernelGGL((muon_apply_kernel<decltype(b)::value, decltype(pr)::value>), dim3(blocks), dim3(256), 0, s, a, from);
  });
}
hipError_t launch_muon_last(bool big, bool pairs, int p_dtype, bool master, int from, const MuonArgs& a, uint32_t blocks,
                            hipStream_t s) {
  return with_type(p_dtype, [&](auto p) {
    typedef decltype(p) T;
    return with_both(big, pairs, [&](auto b, auto pr) {
      constexpr bool B = decltype(b)::value, R = decltype(pr)::value;
      if (master) hipLaunchKernelGGL((muon_last_kernel<B, R, T, true>), dim3(blocks), dim3(256), 0, s, a, from);
      else hipLaunchKernelGGL((muon_last_kernel<B, R, T, false>), dim3(blocks), dim3(256), 0, s, a, from);
    });
  });
}

}  // namespace attr
