// One AdamW step over many tensors (attr_adamw_step).
//
// Every element is read once and written once: HBM-bound (with 32-bit
// states 26 or 28 bytes an element of fp32 weights, 22 or 24 of 16-bit ones, 28 or 30 with
// masters; with 8-bit states 12 fewer and 1/16 for the scales).  The descriptors travel in
// kernel arguments; a workgroup finds its tensor by its first chunk and takes one
// chunk of it, a wave U runs of 256 elements, four elements a lane, all loads in
// flight before the first is used.  A run is a block of the 8-bit states: its
// largest magnitude is one reduction over the wave's lanes, without LDS or barriers.
// Loads and stores need no alignment beyond the element's; with 32-bit states the runs
// start at the 128-byte lines of the first moment, the first run with what is before
// one (40M fp32 elements that start between lines: 204 us with runs from there, 182 so).
//
// Arithmetic is fp32 and never contracted into fused multiply-adds: every
// element's result is the same however the tensors are split over workgroups.
//
// Measured on one MI355X (large copies: 5.2 TB/s): 268M elements with bf16 weights,
// fp32 masters and 32-bit states 1.26 to 1.29 ms (5.9 TB/s); 134M fp32 weights with 8-bit
// states 310 us (6.1 TB/s, 69 vector instructions an element: 82 to 93% of what the
// rate allows, by the clock); 168 adapter tensors side by side, 2.9M elements, 15 us.
#include "common.h"
#include "kernels.h"

#include <type_traits>

#pragma clang fp contract(off)

namespace attr {
namespace {

constexpr int kQuantBlock = kAdamwRun;  // elements that share a scale of the 8-bit states: a wave's run
constexpr int kAdamwRuns = 4, kAdamwRunsEight = 2;  // runs of a wave
constexpr float kE4M3Max = 448.f;
constexpr float kE4M3Least = 0.001953125f;  // 2^-9, the smallest positive value
constexpr float kAmaxLeast = 0x1p-100f;     // below it 448 / amax nears fp32's range

// four elements at any element's address
template <typename T>
struct Four;
template <>
struct Four<float> { typedef f32x4 vec __attribute__((aligned(4))); };
template <>
struct Four<__bf16> {
  typedef __bf16 plain __attribute__((ext_vector_type(4)));
  typedef plain vec __attribute__((aligned(2)));
};
template <>
struct Four<_Float16> { typedef f16x4 vec __attribute__((aligned(2))); };

// Which of four elements there are: those from `lo` on, below `hi`.
struct Part {
  int lo, hi;
  __device__ inline bool has(int e) const { return e >= lo && e < hi; }
};
__device__ inline Part part_of(int64_t i, int64_t n) {
  return {i < 0 ? (i > -4 ? (int)-i : 4) : 0, n - i >= 4 ? 4 : (int)(n - i)};
}

// Four elements in one access, or (not WHOLE) those that there are and 0 for the others.
template <bool WHOLE, typename T>
__device__ inline void load4(const T* p, Part in, T (&x)[4]) {
  if constexpr (WHOLE) {
    const auto v = __builtin_nontemporal_load(reinterpret_cast<const typename Four<T>::vec*>(p));
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = in.has(e) ? p[e] : (T)0;
  }
}
template <bool WHOLE, typename T>
__device__ inline void store4(T* p, Part in, const T (&x)[4]) {
  if constexpr (WHOLE) {
    typename Four<T>::vec v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
    __builtin_nontemporal_store(v, reinterpret_cast<typename Four<T>::vec*>(p));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (in.has(e)) p[e] = x[e];
  }
}

// The same of the 8-bit states: four codes in a word, at any address.
typedef uint32_t loose_u32 __attribute__((aligned(1)));
template <bool WHOLE>
__device__ inline uint32_t load_codes(const uint8_t* p, Part in) {
  if constexpr (WHOLE) return __builtin_nontemporal_load(reinterpret_cast<const loose_u32*>(p));
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) w |= in.has(e) ? (uint32_t)p[e] << (8 * e) : 0u;
  return w;
}
template <bool WHOLE>
__device__ inline void store_codes(uint8_t* p, Part in, uint32_t w) {
  if constexpr (WHOLE) {
    __builtin_nontemporal_store(w, reinterpret_cast<loose_u32*>(p));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (in.has(e)) p[e] = (uint8_t)(w >> (8 * e));
  }
}
__device__ inline void decode(uint32_t w, float scale, float (&x)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0] * scale;
  x[1] = lo[1] * scale;
  x[2] = hi[0] * scale;
  x[3] = hi[1] * scale;
}
__device__ inline uint32_t encode(const float (&x)[4]) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
}

// Square root within an ulp, for the step itself (the states' roots are rounded
// correctly: one bit of them would move codes).  The instruction takes normal inputs.
__device__ inline float near_sqrt(float x) {
  const bool tiny = x < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(tiny ? x * 0x1p96f : x);
  return tiny ? r * 0x1p-48f : r;
}

// largest of a wave's values: magnitudes as their bits, whose order keeps
// infinities and NaN above every finite value
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_max(uint32_t x) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
  return o > x ? o : x;
}
__device__ inline float wave_amax(const float (&x)[4]) {
  uint32_t b = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t o = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu;
    b = o > b ? o : b;
  }
  b = dpp_max<0x111, 0xf>(b);
  b = dpp_max<0x112, 0xf>(b);
  b = dpp_max<0x114, 0xf>(b);
  b = dpp_max<0x118, 0xf>(b);
  b = dpp_max<0x142, 0xa>(b);
  b = dpp_max<0x143, 0xc>(b);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)b, 63));
}

// RUNS runs of a wave from run0 on, of `lead` elements fewer in the first; all of their
// elements are there (WHOLE), or some are not.
template <typename P, typename G, bool EIGHT, bool MASTER, bool WHOLE, int RUNS>
__device__ inline void adamw_runs(const AdamwStep& a, const AdamwEntry& t, const AdamwExtra& ex, float gs, int64_t run0,
                                  int lead) {
  typedef typename std::conditional<EIGHT, uint8_t, float>::type S;
  typedef typename std::conditional<MASTER, float, P>::type W;
  const int lane = threadIdx.x & 63;
  const int64_t i0 = run0 * kQuantBlock - lead + lane * 4;
  W* const wt = (MASTER ? (W*)ex.master : (W*)t.p) + i0;
  P* const pt = (P*)t.p + i0;
  const G* const gt = (const G*)t.g + i0;
  S* const mt = (S*)t.m + i0;
  S* const vt = (S*)t.v + i0;
  W x[RUNS][4];
  G g[RUNS][4];
  float m[RUNS][4], v[RUNS][4], ms[RUNS], vs[RUNS];
  uint32_t mw[RUNS], vw[RUNS];
#pragma unroll
  for (int u = 0; u < RUNS; ++u) {
    const int k = u * kQuantBlock;
    const Part in = part_of(i0 + k, t.n);
    load4<WHOLE>(wt + k, in, x[u]);
    load4<WHOLE>(gt + k, in, g[u]);
    if constexpr (EIGHT) {
      mw[u] = load_codes<WHOLE>(mt + k, in);
      vw[u] = load_codes<WHOLE>(vt + k, in);
      ms[u] = ex.m_scale[run0 + u];
      vs[u] = ex.v_scale[run0 + u];
    } else {
      load4<WHOLE>(mt + k, in, m[u]);
      load4<WHOLE>(vt + k, in, v[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < RUNS; ++u) {
    const int k = u * kQuantBlock;
    const Part in = part_of(i0 + k, t.n);
    if constexpr (EIGHT) {
      decode(mw[u], ms[u], m[u]);
      decode(vw[u], vs[u], v[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = v[u][e] * v[u][e];
    }
    float nm[4], nv[4];
    W nx[4];
    P np[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gr = (float)g[u][e] * gs, w = (float)x[u][e];
      nm[e] = m[u][e] * a.beta1 + gr * a.one_beta1;
      nv[e] = v[u][e] * a.beta2 + (gr * gr) * a.one_beta2;
      const float root = near_sqrt(nv[e] * a.corr2 + a.eps_root) + a.eps;
      const float r = w - w * t.lr_wd - nm[e] * t.lr * __builtin_amdgcn_rcpf(root);
      nx[e] = (W)r;
      np[e] = (P)r;
    }
    store4<WHOLE>(wt + k, in, nx);
    if (MASTER) store4<WHOLE>(pt + k, in, np);
    if constexpr (EIGHT) {
      float root[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        root[e] = sqrtf(nv[e]);
        if (!WHOLE && !in.has(e)) root[e] = nm[e] = 0.f;
      }
      float am = wave_amax(nm), av = wave_amax(root);
      am = am < kAmaxLeast ? kAmaxLeast : am;
      av = av < kAmaxLeast ? kAmaxLeast : av;
      const float fm = 1.f / am * kE4M3Max, fv = 1.f / av * kE4M3Max;
      float qm[4], qv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        qm[e] = nm[e] * fm;
        const float q = root[e] * fv;
        qv[e] = q > 0.f && q < kE4M3Least ? kE4M3Least : q;
      }
      store_codes<WHOLE>(mt + k, in, encode(qm));
      store_codes<WHOLE>(vt + k, in, encode(qv));
      if (lane == 0) {
        ex.m_scale[run0 + u] = am < INFINITY ? am * (1.f / kE4M3Max) : NAN;
        ex.v_scale[run0 + u] = av < INFINITY ? av * (1.f / kE4M3Max) : NAN;
      }
    } else {
      store4<WHOLE>(mt + k, in, nm);
      store4<WHOLE>(vt + k, in, nv);
    }
  }
}

template <typename P, typename G, bool EIGHT, bool MASTER, int RUNS, typename Args>
__global__ __launch_bounds__(256) void adamw_kernel(Args a) {
  int lo = 0, hi = a.step.n - 1;  // the last tensor whose first chunk is not past this workgroup
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.e[mid].chunk0 <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwEntry& t = a.e[lo];
  AdamwExtra ex{};
  if constexpr (EIGHT || MASTER) ex = a.x[lo];
  const float gs = a.step.grad_scale ? *a.step.grad_scale : 1.f;
  const int64_t run0 = ((int64_t)(blockIdx.x - t.chunk0) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * RUNS;
  const int lead = EIGHT ? 0 : adamw_lead(t.m);
  if (run0 * kQuantBlock >= lead && (run0 + RUNS) * kQuantBlock - lead <= t.n) {
    adamw_runs<P, G, EIGHT, MASTER, true, RUNS>(a.step, t, ex, gs, run0, lead);
  } else {
#pragma unroll 1
    for (int64_t r = run0; r < run0 + RUNS && r * kQuantBlock - lead < t.n; ++r)
      adamw_runs<P, G, EIGHT, MASTER, false, 1>(a.step, t, ex, gs, r, lead);
  }
}

template <typename P, typename G, bool EIGHT, bool MASTER, typename Args>
void launch_runs(int runs, uint32_t blocks, const Args& a, hipStream_t s) {
  constexpr int kMany = EIGHT ? kAdamwRunsEight : kAdamwRuns;
  if (runs == 1) hipLaunchKernelGGL((adamw_kernel<P, G, EIGHT, MASTER, 1, Args>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adamw_kernel<P, G, EIGHT, MASTER, kMany, Args>), dim3(blocks), dim3(256), 0, s, a);
}
template <typename P, typename G>
void launch(bool, bool, int runs, uint32_t blocks, const AdamwPlain& a, hipStream_t s) {
  launch_runs<P, G, false, false>(runs, blocks, a, s);
}
template <typename P, typename G>
void launch(bool eight, bool master, int runs, uint32_t blocks, const AdamwFull& a, hipStream_t s) {
  if (eight && master) launch_runs<P, G, true, true>(runs, blocks, a, s);
  else if (eight) launch_runs<P, G, true, false>(runs, blocks, a, s);
  else launch_runs<P, G, false, true>(runs, blocks, a, s);
}
template <typename P, typename Args>
void launch_g(int g_dtype, bool eight, bool master, int runs, uint32_t blocks, const Args& a, hipStream_t s) {
  if (g_dtype == 0) launch<P, float>(eight, master, runs, blocks, a, s);
  else if (g_dtype == 1) launch<P, __bf16>(eight, master, runs, blocks, a, s);
  else launch<P, _Float16>(eight, master, runs, blocks, a, s);
}
template <typename Args>
hipError_t launch_p(int p_dtype, int g_dtype, bool eight, bool master, int runs, uint32_t blocks, const Args& a,
                    hipStream_t s) {
  if (p_dtype == 0) launch_g<float>(g_dtype, eight, master, runs, blocks, a, s);
  else if (p_dtype == 1) launch_g<__bf16>(g_dtype, eight, master, runs, blocks, a, s);
  else launch_g<_Float16>(g_dtype, eight, master, runs, blocks, a, s);
  return hipGetLastError();
}

}  // namespace

// Loads in flight against waves: with 32-bit states four runs a wave (1294 us for 268M
// elements with masters; two 1341, eight 1335), with 8-bit ones two (134M: 314; four 319,
// eight 330), and one in small models, for more waves.
int adamw_runs_per_wave(int64_t elements, bool eight) {
  return elements < (8 << 20) ? 1 : eight ? kAdamwRunsEight : kAdamwRuns;
}

hipError_t launch_adamw(int p_dtype, int g_dtype, int runs, uint32_t blocks, const AdamwPlain& a, hipStream_t s) {
  return launch_p(p_dtype, g_dtype, false, false, runs, blocks, a, s);
}
hipError_t launch_adamw(int p_dtype, int g_dtype, bool eight, bool master, int runs, uint32_t blocks,
                        const AdamwFull& a, hipStream_t s) {
  return launch_p(p_dtype, g_dtype, eight, master, runs, blocks, a, s);
}

}  // namespace attr
