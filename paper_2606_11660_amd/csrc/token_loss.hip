// Log-probabilities of given tokens, the clipped policy loss with a KL term and
// the paired log-ratio preference loss, with their gradients with respect to
// the logits.
//
// With c = s log2 e, an offset m and e_j = exp2(c z_j - c m), S = sum e_j:
//     logp = (c z_y - c m - log2 S) ln 2,   p_j = e_j / S,
// and the gradient of a loss with derivative g by logp is s g ([j = y] - p_j).  m is
// the row's largest element, or the largest of its first ones.  c z_j - c m is one fused
// multiply-add with the rounded c m: its rounding is the same factor in every e_j and
// cancels (up to |c m| = 2^20, see kMostMc; other rows, those of infinities and of
// nothing but a mask's lowest value among them, form the differences z_j - m first).
// Sums are fp32 chains per thread, then trees; the losses' sums over tokens are fp64.
//
// All of it is bound by HBM: rows are read with 16-byte loads.  An odd vocabulary's
// rows start anywhere; the elements before a row's first line or 16-byte boundary and
// those after its last whole vector go one a thread (vectors across the boundaries cost
// a fifth of the rate).  Stores follow the loads' cut, wherever that falls in dlogits.
// An element takes one exponential for the sum and one for the gradient (a quarter of
// the other instructions' rate): at 16-bit types half of the time that its bytes take.
//
// Measured on one MI355X (large copies: 5.2 TB/s; one read stream: 7.1):
//   log-probabilities of 3984 bf16 rows of 65536: 81 us, 6.5 TB/s
//   policy loss and gradient of 11008 bf16 rows of 131072, an eighth of them masked:
//     994 us, 5.4 TB/s; 8192 rows of 65536: 355 us, 6.0 TB/s
//   preference loss and gradient of 5312 fp16 rows of 50257, a quarter of them masked:
//     212 us (rows read twice: 1.33 GB, 6.3 TB/s)
#include "common.h"
#include "kernels.h"

namespace attr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;
constexpr float kMostMc = 1048576.f;  // 2^20: the residual of the fused form stays below 2^-4

// What a workgroup does with one token's slot.
struct Slot {
  int64_t row;
  int32_t target;   // in [0, V) where counts
  float weight;
  bool write;       // the row's outputs are written
  bool counts;      // its logits are read
};

// A value that is the same in a wave's lanes, into a scalar register: a slot's row, its
// addresses and its loss's inputs then take none of the registers that hold the row.
__device__ inline float uniform(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}
__device__ inline int64_t uniform(int64_t x) {
  return ((int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// Token slot (the same for a wave's lanes) of a batch: example slot / T, token slot % T
// (attr_token_rows).  Loads that do not depend on each other are issued together: their
// latency is what a call of few rows consists of.
__device__ inline Slot slot_of(const TokenArgs& a, uint32_t slot) {
  const uint32_t i = slot / a.T, t = slot - i * a.T;
  Slot r;
  const int32_t len = a.length ? a.length[i] : (int32_t)a.T;
  r.row = a.row_offset ? uniform(a.row_offset[i]) + t : (int64_t)slot;
  const bool inside = r.row >= 0 && r.row < a.n_rows, in = (int32_t)t < __builtin_amdgcn_readfirstlane(len);
  const int64_t y = uniform(inside ? a.target[r.row] : -1);
  r.weight = uniform(inside && a.weight ? a.weight[r.row] : 1.f);
  r.write = inside && (in || !a.row_offset);
  r.counts = inside && in && y >= 0 && y < a.V && r.weight != 0.f;
  r.target = (int32_t)y;
  return r;
}

// ---------------------------------------------------------------------------
// 16-byte vectors of elements
// ---------------------------------------------------------------------------
template <typename T>
constexpr int kE = 16 / (int)sizeof(T);  // elements of a vector

// vectors at any element's address
template <typename T>
struct Loose;
template <>
struct Loose<float> { typedef i32x4 vec __attribute__((aligned(4))); };
template <>
struct Loose<__bf16> { typedef i32x4 vec __attribute__((aligned(2))); };
template <>
struct Loose<_Float16> { typedef i32x4 vec __attribute__((aligned(2))); };

// a vector of -inf: it adds nothing to a maximum or a sum
__device__ inline i32x4 no_vec(float) { return i32x4{(int)0xff800000, (int)0xff800000, (int)0xff800000, (int)0xff800000}; }
__device__ inline i32x4 no_vec(__bf16) { return i32x4{(int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80}; }
__device__ inline i32x4 no_vec(_Float16) { return i32x4{(int)0xfc00fc00, (int)0xfc00fc00, (int)0xfc00fc00, (int)0xfc00fc00}; }

// KEEP: the row is read again by a later launch; else it streams past the caches
// (bf16 rows of 65536: 6.5 TB/s against 5.8).
template <bool KEEP = false, typename T>
__device__ inline i32x4 load_vec(const T* p) {
  const auto* v = reinterpret_cast<const typename Loose<T>::vec*>(p);
  if constexpr (KEEP) return *v;
  else return __builtin_nontemporal_load(v);
}
template <typename T>
__device__ inline void store_vec(T* p, i32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<typename Loose<T>::vec*>(p));
}

__device__ inline void unpack(i32x4 v, float, float (&x)[4]) {
  const f32x4 f = __builtin_bit_cast(f32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = f[e];
}
__device__ inline void unpack(i32x4 v, __bf16, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __builtin_bit_cast(float, v[e] << 16);
    x[2 * e + 1] = __builtin_bit_cast(float, v[e] & (int)0xffff0000);
  }
}
__device__ inline void unpack(i32x4 v, _Float16, float (&x)[8]) {
  const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
}

// Makes the compiler forget what it knows of a value: without it the unpacked
// elements of one stage are kept for the next (twice the registers for 16-bit
// types), and the lane masks of the loads for the stores.
__device__ inline void forget(i32x4& v) { asm volatile("" : "+v"(v)); }
__device__ inline void forget(int32_t& v) { asm volatile("" : "+v"(v)); }
template <int N>
__device__ inline void forget(i32x4 (&v)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) forget(v[k]);
}

__device__ inline i32x4 pack(const float (&x)[4], float) {
  return __builtin_bit_cast(i32x4, f32x4{x[0], x[1], x[2], x[3]});
}
__device__ inline i32x4 pack(const float (&x)[8], __bf16) {
  bf16x8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (__bf16)x[e];
  return __builtin_bit_cast(i32x4, h);
}
__device__ inline i32x4 pack(const float (&x)[8], _Float16) {
  f16x8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
  return __builtin_bit_cast(i32x4, h);
}

// ---------------------------------------------------------------------------
// reductions
// ---------------------------------------------------------------------------
// Lane shifts within rows of 16 and broadcasts across them, no LDS: the result
// is in lane 63 and returned to all.
template <int CTRL, int ROWS>
__device__ inline float dpp(float old, float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, x),
                                                               CTRL, ROWS, 0xf, false));
}
__device__ inline float lane63(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ inline float wave_max_dpp(float x) {
  x = fmaxf(x, dpp<0x111, 0xf>(-INFINITY, x));
  x = fmaxf(x, dpp<0x112, 0xf>(-INFINITY, x));
  x = fmaxf(x, dpp<0x114, 0xf>(-INFINITY, x));
  x = fmaxf(x, dpp<0x118, 0xf>(-INFINITY, x));
  x = fmaxf(x, dpp<0x142, 0xa>(-INFINITY, x));
  x = fmaxf(x, dpp<0x143, 0xc>(-INFINITY, x));
  return lane63(x);
}
__device__ inline float wave_sum_dpp(float x) {
  x += dpp<0x111, 0xf>(0.f, x);
  x += dpp<0x112, 0xf>(0.f, x);
  x += dpp<0x114, 0xf>(0.f, x);
  x += dpp<0x118, 0xf>(0.f, x);
  x += dpp<0x142, 0xa>(0.f, x);
  x += dpp<0x143, 0xc>(0.f, x);
  return lane63(x);
}
template <int NT>
__device__ inline float block_max(float x, float* sh) {
  x = wave_max_dpp(x);
  if (NT == 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  x = sh[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) x = fmaxf(x, sh[w]);
  return x;
}
template <int NT>
__device__ inline float block_add(float x, float* sh) {
  x = wave_sum_dpp(x);
  if (NT == 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  x = sh[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) x += sh[w];
  return x;
}

// A row is swept by NT threads: a whole workgroup, or (64) one of its four waves,
// since a workgroup a short row would be bound by their dispatch (16384 rows of
// 2 KB: 12.3 us).
template <int NT>
__device__ inline int32_t thread() { return NT == 64 ? threadIdx.x & 63 : threadIdx.x; }
template <int NT>
__device__ inline uint32_t first_slot() {
  return NT == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
}

// A row of V elements: `head` before the first boundary, `whole` in vectors from there
// on, fewer than a vector's after them; `at`: this thread's element of the first and
// last (V or more: none).  Boundaries are those of 128-byte lines where there are
// threads for the head, so that a wave's stores fill whole lines.
struct Cut {
  int32_t head, whole, at;
};
template <typename T, int NT>
__device__ inline Cut cut_row(const T* z, int32_t V) {
  constexpr int E = kE<T>, A = NT > 64 ? 128 / (int)sizeof(T) : E;
  const int32_t off = (int32_t)(-(reinterpret_cast<intptr_t>(z) / (int)sizeof(T)) & (A - 1));
  Cut k;
  k.head = off < V ? off : V;
  k.whole = (V - k.head) / E * E;
  k.at = thread<NT>() < k.head ? thread<NT>() : k.whole + thread<NT>();
  return k;
}

// Scratch of a workgroup: two sets, so that a reduction's reads need no barrier
// before the next one's writes.
struct Shared {
  float max[16], sum[16], slow[16], part[16], zy;
};

// A row's maximum and sum in either form: offset is c m and x_j = fma(z_j, c,
// -offset) in the fused form; in the other, x_j = (z_j - offset) c, offset = m.
struct RowSum {
  float offset, sum, top;  // top: m
  bool apart;
};
__device__ inline float exponent(float z, float c, const RowSum& r) {
  return r.apart ? (z - r.offset) * c : fmaf(z, c, -r.offset);
}
// logp / ln 2 = x - n - log2 f with the linear part x, and the sum's binary exponent n and
// mantissa f: the offset need not be the row's maximum, so x and n may be large and are
// joined in fp64; log2 f is in [-1, 0].
struct LogParts {
  double whole;
  float rest;
};
__device__ inline LogParts log_parts(float zy, float c, const RowSum& r) {
  const double x = r.apart ? ((double)zy - (double)r.offset) * (double)c : (double)zy * (double)c - (double)r.offset;
  return {x - (double)__builtin_amdgcn_frexp_expf(r.sum), log2f(__builtin_amdgcn_frexp_mantf(r.sum))};
}
__device__ inline double row_logp(float zy, float c, const RowSum& r) {
  const LogParts l = log_parts(zy, c, r);
  return (l.whole - (double)l.rest) * kLn2;
}

// c m as the fused form's offset: the rounded product itself, and never the exact one within
// a difference of two offsets (contracted, a sum would be rescaled to another offset than its
// next terms are relative to: at logits near 1e5 logp lost 1e-4).
__device__ inline float offset_at(float m, float c) {
#pragma clang fp contract(off)
  return m * c;
}

// Whether the fused form takes a row (part) with maximum m; not if it is NaN.
__device__ inline bool fused(float m, float c) { return fabsf(m * c) <= kMostMc; }

// The sum with the differences formed first, one element at a time: rows whose
// maximum m the fused form does not take, and rows in registers whose largest entries
// come late.  Two loads in flight: more, or whole vectors, take registers that the rows
// in registers need (2048 bf16 rows of 50257, all late: 280 us with one, 211 with two, 181
// with four, which spill; 74 for rows of the common kind).
template <typename T, int NT>
__device__ RowSum row_sum_apart(const T* z, int32_t V, float c, float m, float* sh) {
  float s = 0.f;
#pragma unroll 2
  for (int32_t j = thread<NT>(); j < V; j += NT) s += __builtin_amdgcn_exp2f(((float)z[j] - m) * c);
  return {m, block_add<NT>(s, sh), m, true};
}
template <typename T, int NT>
__device__ RowSum row_sum_apart(const T* z, int32_t V, float c, Shared& sh) {
  float m = -INFINITY;
#pragma unroll 2
  for (int32_t j = thread<NT>(); j < V; j += NT) m = fmaxf(m, (float)z[j]);
  return row_sum_apart<T, NT>(z, V, c, block_max<NT>(m, sh.max), sh.slow);
}
template <typename T, int NT>
__device__ void row_grad_apart(const T* z, T* out, int32_t V, int32_t y, float c, const RowSum& r, float cs,
                               float ce) {
#pragma unroll 1
  for (int32_t j = thread<NT>(); j < V; j += NT) {
    float d = ce * __builtin_amdgcn_exp2f(exponent((float)z[j], c, r));
    if (j == y) d += cs;
    out[j] = (T)d;
  }
}

template <typename T, int NT>
__device__ inline void row_zero(T* out, int32_t V) {
  constexpr int E = kE<T>;
  const Cut k = cut_row<T, NT>(out, V);
  for (int32_t j = thread<NT>() * E; j < k.whole; j += NT * E) store_vec(out + k.head + j, i32x4{0, 0, 0, 0});
  if (k.at < V) out[k.at] = (T)0.f;
}

// One vector's gradient, from its elements.
template <typename T>
__device__ inline i32x4 grad_vec(i32x4 v, float c, float offset, float cs, float ce, int32_t y_at) {
  float x[kE<T>];
  unpack(v, T{}, x);
#pragma unroll
  for (int e = 0; e < kE<T>; ++e) x[e] = ce * __builtin_amdgcn_exp2f(fmaf(x[e], c, -offset));
  if ((uint32_t)y_at < (uint32_t)kE<T>) {
#pragma unroll
    for (int e = 0; e < kE<T>; ++e) x[e] += e == y_at ? cs : 0.f;
  }
  return pack(x, T{});
}

template <typename T>
__device__ inline T grad_one(T z, float c, float offset, float cs, float ce, bool y) {
  const float d = ce * __builtin_amdgcn_exp2f(fmaf((float)z, c, -offset));
  return (T)(y ? d + cs : d);
}

// A row's maximum and sum in one sweep: per thread a running maximum (not below
// -2^20 / c, so that nothing but -inf needs no case of its own) and a sum that is
// rescaled when it grows, U vectors at a time.
template <typename T, int NT, int U, bool KEEP>
__device__ inline RowSum row_sum_stream(const T* z, int32_t V, float c, Shared& sh) {
  constexpr int E = kE<T>;
  const Cut k = cut_row<T, NT>(z, V);
  const T* zv = z + k.head;
  float top = k.at < V ? (float)z[k.at] : -INFINITY;
  float mc = fmaxf(offset_at(top, c), -kMostMc), s = __builtin_amdgcn_exp2f(fmaf(top, c, -mc));
  for (int32_t j0 = thread<NT>() * E; j0 < k.whole; j0 += NT * E * U) {
    i32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = j0 + u * NT * E < k.whole ? load_vec<KEEP>(zv + j0 + u * NT * E) : no_vec(T{});
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[E];
      unpack(v[u], T{}, x);
      float m = x[0];
#pragma unroll
      for (int e = 1; e < E; ++e) m = fmaxf(m, x[e]);
      top = fmaxf(top, m);
      const float up = offset_at(m, c);
      if (up > mc) {
        s *= __builtin_amdgcn_exp2f(mc - up);
        mc = up;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(x[e], c, -mc));
    }
  }
  const float m = block_max<NT>(top, sh.max);
  if (!fused(m, c)) return row_sum_apart<T, NT>(z, V, c, m, sh.slow);
  const float most = offset_at(m, c);
  s *= __builtin_amdgcn_exp2f(mc - most);
  return {most, block_add<NT>(s, sh.sum), m, false};
}

// The gradient of one row, read a second time.  A thread reads and writes its own
// elements only: the two may be one buffer.
template <typename T, int NT, int U>
__device__ inline void row_grad_stream(const T* z, T* out, int32_t V, int32_t y, float c, const RowSum& r, float cs,
                                       float ce) {
  constexpr int E = kE<T>;
  if (r.apart) return row_grad_apart<T, NT>(z, out, V, y, c, r, cs, ce);
  const Cut k = cut_row<T, NT>(z, V);
  if (k.at < V) out[k.at] = grad_one(z[k.at], c, r.offset, cs, ce, k.at == y);
  z += k.head;
  out += k.head;
  y -= k.head;
  for (int32_t j0 = thread<NT>() * E; j0 < k.whole; j0 += NT * E * U) {
    i32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * NT * E < k.whole) v[u] = load_vec(z + j0 + u * NT * E);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t j = j0 + u * NT * E;
      if (j < k.whole) store_vec(out + j, grad_vec<T>(v[u], c, r.offset, cs, ce, y - j));
    }
  }
}

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------
// A token's part of the policy loss, loaded before its row.
struct PolicyToken {
  float weight, advantage, old, ref;
};
__device__ inline PolicyToken policy_inputs(const PolicyArgs& p, const TokenArgs& a, uint32_t slot, const Slot& sl) {
  // what there is not is read elsewhere, without a branch (and its wait), and not used
  const float* advantage = p.advantage + (p.per_token ? sl.row : (int64_t)(slot / a.T));
  const float* old = p.logp_old ? p.logp_old + sl.row : advantage;
  const float* ref = p.beta != 0.f ? p.logp_ref + sl.row : advantage;
  return {sl.weight, *advantage, *old, *ref};
}

// Loss and derivative by logp of one token of the policy loss, weights included.
struct TokenLoss {
  float loss, c;
};
__device__ inline TokenLoss policy_token(const PolicyArgs& p, const PolicyToken& k, float logp) {
  const float ratio = p.logp_old ? expf(logp - k.old) : logp == logp ? 1.f : logp;
  const float taken = k.advantage == 0.f ? 1.f : ratio;  // an advantage of 0 takes 0 of a ratio past fp32 too
  const float free_ = -k.advantage * taken;
  const float held = -k.advantage * fminf(fmaxf(taken, p.lo), p.hi);
  float loss = free_ >= held ? free_ : held, c = free_ >= held ? free_ : 0.f;
  if (ratio != ratio) loss = c = ratio;  // a NaN stays
  if (p.beta != 0.f) {
    const float d = k.ref - logp, less = expm1f(d);
    loss += p.beta * (less == INFINITY ? less : less - d);  // a token of probability 0: d is infinite too
    c -= p.beta * less;
  }
  return {k.weight * loss, k.weight * c};
}

// Outputs of a slot that does not count.
template <typename T, int NT>
__device__ inline void skip_slot(const TokenArgs& a, const Slot& sl) {
  if (!sl.write) return;
  if (thread<NT>() == 0 && a.logp) a.logp[sl.row] = 0.f;
  if (a.dlogits) row_zero<T, NT>((T*)a.dlogits + sl.row * a.ldd, a.V);
}

// Threads of a workgroup whose rows are swept by NT threads each.
constexpr int group_of(int nt) { return nt == 64 ? 256 : nt; }

// A counting token's share of its log ratio; one thread writes its log-probability.  The
// ratios are small differences of sums: here the difference is in fp64.
__device__ inline double token_part(const TokenArgs& a, const Slot& sl, float zy, float c, const RowSum& r,
                                    const float* logp_ref) {
  const double logp = row_logp(zy, c, r);
  if (thread<64>() == 0 && a.logp) a.logp[sl.row] = (float)logp;
  return (double)sl.weight * (logp - (logp_ref ? (double)logp_ref[sl.row] : 0.0));
}

// A slot's log-probability, and (PREF) what the preference loss keeps of it: one thread.
template <bool PREF>
__device__ inline void write_logp(const TokenArgs& a, uint32_t slot, const Slot& sl, float zy, float c,
                                  const RowSum& r, const float* logp_ref) {
  if (!PREF) {
    a.logp[sl.row] = (float)row_logp(zy, c, r);
    return;
  }
  a.part[slot] = token_part(a, sl, zy, c, r, logp_ref);
  a.stats[slot] = float2{r.offset, r.apart ? -r.sum : r.sum};
}
template <bool PREF>
__device__ inline void skip_logp(const TokenArgs& a, uint32_t slot, const Slot& sl) {
  if (sl.write && (!PREF || a.logp)) a.logp[sl.row] = 0.f;
  if (PREF) a.part[slot] = 0.0;
}

// Log-probabilities (PREF: and what the gradient needs of each row), one sweep.  What
// the caches keep of PREF's rows saves the gradient a part of its reads (4000 fp16
// rows of 50257: both passes 221 us without, 204 with; no difference from 1.6 GB on).
template <typename T, int NT, int U, bool PREF>
__global__ __launch_bounds__(group_of(NT)) void token_logp_kernel(TokenArgs a, const float* logp_ref) {
  __shared__ Shared sh;
  const float c = a.scale * kLog2e;
  const uint32_t slot = a.slot0 + first_slot<NT>();
  if (slot >= a.n_slots) return;
  const Slot sl = slot_of(a, slot);
  if (!sl.counts) {
    if (thread<NT>() == 0) skip_logp<PREF>(a, slot, sl);
    return;
  }
  const T* z = (const T*)a.logits + sl.row * a.ldl;
  const float zy = (float)z[sl.target];
  const RowSum r = row_sum_stream<T, NT, U, PREF>(z, a.V, c, sh);
  if (thread<NT>() == 0) write_logp<PREF>(a, slot, sl, zy, c, r, logp_ref);
}

// A row in the registers of NT threads, NV vectors each: V <= NT NV kE.  16-bit rows of
// more than 128 KB, one to a CU, are read through the caches after all (8192 bf16 rows
// of 131072: 804 us, 829 past them; fp32 rows of 256 KB: 393 and 387).
template <typename T, int NT, int NV>
struct RowRegs {
  static constexpr int E = kE<T>;
  static constexpr bool KEEP = sizeof(T) == 2 && NT * NV > 8192;  // vectors
  const T* z;
  Cut cut;
  T rest;
  i32x4 v[NV];

  __device__ inline void load(const T* row, int32_t V) {
    z = row;
    cut = cut_row<T, NT>(z, V);
    rest = cut.at < V ? z[cut.at] : (T)-INFINITY;
    // range-checked, so that no branch is around them: the sums wait for each vector
    // alone.  Lanes past the row's end read nothing and hold zeros.
    const __amdgpu_buffer_rsrc_t r = make_rsrc(z + cut.head, (uint32_t)cut.whole * (uint32_t)sizeof(T));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t off = (uint32_t)(k * NT + thread<NT>()) * 16u;
      v[k] = KEEP ? load16_cached(r, off) : load16_stream(r, off);
    }
  }
  __device__ inline float vec_sum(int k, float mc, float c) {
    float x[E], s = 0.f;
    unpack(v[k], T{}, x);
#pragma unroll
    for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(x[e], c, -mc));
    return s;
  }
  // The row's sum relative to the largest of its first vectors, which is known while the
  // others are still on their way; `also`, an element of the row, is read before anything
  // is written.  Not ok: a sum past 2^60, from entries far above them (a gradient is
  // divided by it: 2^100 would leave one of 1e-15 to subnormal numbers), or a row that
  // the fused form does not take.
  __device__ inline RowSum sum(float also, float c, Shared& sh, bool& ok) {
    const int32_t at = thread<NT>() * E;
    float m = fmaxf(also, (float)rest);
    if (at < cut.whole) {
      float x[E];
      unpack(v[0], T{}, x);
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, x[e]);
    }
    m = block_max<NT>(m, sh.max);
    const float mc = offset_at(m, c);
    float s = __builtin_amdgcn_exp2f(fmaf((float)rest, c, -mc));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      forget(v[k]);
      if ((k + 1) * NT * E <= cut.whole) s += vec_sum(k, mc, c);
      else if (at + k * NT * E < cut.whole) s += vec_sum(k, mc, c);
    }
    s = block_add<NT>(s, sh.sum);
    ok = fused(m, c) && s < 0x1p60f;
    return {mc, s, m, false};
  }
  // g ([j = y] - p_j) into out
  __device__ inline void grad(T* out, int32_t V, int32_t y, float c, const RowSum& r, float g) {
    const float ce = -g / r.sum;
    if (cut.at < V) out[cut.at] = grad_one(rest, c, r.offset, g, ce, cut.at == y);
    out += cut.head;
    forget(v);
    int32_t j0 = thread<NT>() * E;
    forget(j0);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int32_t j = j0 + k * NT * E;
      if (j < cut.whole) store_vec(out + j, grad_vec<T>(v[k], c, r.offset, g, ce, y - cut.head - j));
    }
  }
};
// One slot of the policy loss, its row in registers.
template <typename T, int NT, int NV>
struct PolicySlot {
  Slot sl;
  PolicyToken in;
  float zy;
  RowRegs<T, NT, NV> row;

  // sl is set, and counts
  __device__ inline void load(const TokenArgs& a, const PolicyArgs& p, uint32_t slot) {
    in = policy_inputs(p, a, slot, sl);
    const T* z = (const T*)a.logits + sl.row * a.ldl;
    zy = (float)z[sl.target];
    row.load(z, a.V);
  }
  // Writes the row's outputs; returns the token's loss.
  __device__ inline float finish(const TokenArgs& a, const PolicyArgs& p, Shared& sh) {
    const float c = a.scale * kLog2e;
    T* out = (T*)a.dlogits + sl.row * a.ldd;
    bool ok;
    const RowSum r = row.sum(zy, c, sh, ok);
    if (!ok) {  // a path of its own, which needs no registers
      const RowSum r = row_sum_apart<T, NT>(row.z, a.V, c, sh);
      const float logp = (float)row_logp(zy, c, r);
      const TokenLoss l = policy_token(p, in, logp);
      if (thread<NT>() == 0 && a.logp) a.logp[sl.row] = logp;
      if (a.dlogits) row_grad_apart<T, NT>(row.z, out, a.V, sl.target, c, r, l.c * a.scale, -l.c * a.scale / r.sum);
      return l.loss;
    }
    const float logp = (float)row_logp(zy, c, r);
    const TokenLoss l = policy_token(p, in, logp);
    if (thread<NT>() == 0 && a.logp) a.logp[sl.row] = logp;
    if (a.dlogits) row.grad(out, a.V, sl.target, c, r, l.c * a.scale);
    return l.loss;
  }
};

template <typename T, int NT, int NV>
__global__ __launch_bounds__(group_of(NT), NV > 8 ? 4 : 8) void policy_kernel(TokenArgs a, PolicyArgs p) {
  __shared__ Shared sh;
  const uint32_t slot = a.slot0 + first_slot<NT>();
  if (slot >= a.n_slots) return;
  PolicySlot<T, NT, NV> k;
  k.sl = slot_of(a, slot);
  if (!k.sl.counts) {
    skip_slot<T, NT>(a, k.sl);
    if (thread<NT>() == 0) p.token_loss[slot] = 0.f;
    return;
  }
  k.load(a, p, slot);
  const float loss = k.finish(a, p, sh);
  if (thread<NT>() == 0) p.token_loss[slot] = loss;
}

// Examples of few short rows in one launch: a workgroup an example, K tokens a wave
// with all of their rows in flight; the first wave adds the losses up, in fp64 in the
// order of the tokens.
template <typename T, int NV, int K>
__global__ __launch_bounds__(1024) void policy_example_kernel(TokenArgs a, PolicyArgs p, float* loss) {
  __shared__ Shared sh;
  __shared__ float token[kPolicyExampleMost];
  const uint32_t t0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), step = blockDim.x >> 6;
  PolicySlot<T, 64, NV> k[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const uint32_t t = t0 + i * step;
    k[i].sl.counts = false;
    if (t >= a.T) continue;
    k[i].sl = slot_of(a, blockIdx.x * a.T + t);
    if (k[i].sl.counts) k[i].load(a, p, blockIdx.x * a.T + t);
    else skip_slot<T, 64>(a, k[i].sl);
  }
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const uint32_t t = t0 + i * step;
    if (t >= a.T) continue;
    const float l = k[i].sl.counts ? k[i].finish(a, p, sh) : 0.f;
    if ((threadIdx.x & 63) == 0) token[t] = l;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const double v = wave_sum(threadIdx.x < a.T ? (double)token[threadIdx.x] : 0.0);
  if (threadIdx.x == 0) loss[blockIdx.x] = (float)v;
}

// Policy loss of any row length, the row read twice.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void policy_stream_kernel(TokenArgs a, PolicyArgs p) {
  __shared__ Shared sh;
  const float c = a.scale * kLog2e;
  const uint32_t slot = a.slot0 + first_slot<NT>();
  const Slot sl = slot_of(a, slot);
  const bool first = thread<NT>() == 0;
  if (!sl.counts) {
    skip_slot<T, NT>(a, sl);
    if (first) p.token_loss[slot] = 0.f;
    return;
  }
  const PolicyToken in = policy_inputs(p, a, slot, sl);
  const T* z = (const T*)a.logits + sl.row * a.ldl;
  if (first) sh.zy = (float)z[sl.target];  // read before anything of the row is written
  const RowSum r = row_sum_stream<T, NT, 4, true>(z, a.V, c, sh);
  const float logp = (float)row_logp(sh.zy, c, r);
  const TokenLoss l = policy_token(p, in, logp);
  if (first) p.token_loss[slot] = l.loss;
  if (first && a.logp) a.logp[sl.row] = logp;
  const float g = l.c * a.scale;
  if (a.dlogits)
    row_grad_stream<T, NT, 4>(z, (T*)a.dlogits + sl.row * a.ldd, a.V, sl.target, c, r, g, -g / r.sum);
}

// ---------------------------------------------------------------------------
// few long rows: each in parts, joined
// ---------------------------------------------------------------------------
// One CU reads 50 GB/s: a row of 1 MB takes 20 us in one workgroup.  A part's result
// is its largest element m and the sum of exp2(c (z - m)), without the rounding of
// c m (0 where the part holds -inf only, so that it adds nothing).
template <typename T, int NT, int U>
__device__ inline float2 part_sum(const T* z, int32_t n, float c, Shared& sh) {
  const RowSum r = row_sum_stream<T, NT, U, true>(z, n, c, sh);
  if (!r.apart) return float2{r.top, r.sum * __builtin_amdgcn_exp2f(-fmaf(r.top, c, -r.offset))};
  if (r.top != -INFINITY) return float2{r.top, r.sum};
  float s = 0.f;
#pragma unroll 1
  for (int32_t j = thread<NT>(); j < n; j += NT) {
    const float x = (float)z[j];
    s += x == x ? 0.f : x;
  }
  return float2{r.top, block_add<NT>(s, sh.part)};
}

// A row's sum from its parts (at most 64), by every wave.
__device__ inline RowSum join_parts(const float2* part, int32_t n, float c) {
  const int lane = threadIdx.x & 63;
  const float2 k = lane < n ? part[lane] : float2{-INFINITY, 0.f};
  const float m = wave_max_dpp(k.x), mc = offset_at(m, c);
  const float s = wave_sum_dpp(k.y == 0.f ? 0.f : k.y * __builtin_amdgcn_exp2f((k.x - m) * c));
  if (fused(m, c)) return {mc, s * __builtin_amdgcn_exp2f(fmaf(m, c, -mc)), m, false};
  return {m, s, m, true};
}

// Part blockIdx.y of a row: elements [from, from + n).
struct Range {
  int32_t from, n;
};
__device__ inline Range part_of(const TokenArgs& a) {
  const int32_t from = (int32_t)blockIdx.y * a.part_len;
  return {from, a.V - from < a.part_len ? a.V - from : a.part_len};
}

template <typename T, int NT, int U>
__global__ __launch_bounds__(NT) void split_sum_kernel(TokenArgs a) {
  __shared__ Shared sh;
  const uint32_t slot = blockIdx.x;
  const Slot sl = slot_of(a, slot);
  if (!sl.counts) return;
  const T* z = (const T*)a.logits + sl.row * a.ldl;
  const Range g = part_of(a);
  const float zy = (float)z[sl.target];
  const float2 v = part_sum<T, NT, U>(z + g.from, g.n, a.scale * kLog2e, sh);
  if (threadIdx.x != 0) return;
  a.parts[slot * gridDim.y + blockIdx.y] = v;
  if (blockIdx.y == 0) a.zy[slot] = zy;
}

// The log-probabilities of rows summed in n_parts parts: a wave a slot.
template <bool PREF>
__global__ __launch_bounds__(256) void split_logp_kernel(TokenArgs a, int32_t n_parts, const float* logp_ref) {
  const uint32_t slot = first_slot<64>();
  if (slot >= a.n_slots) return;
  const Slot sl = slot_of(a, slot);
  const float c = a.scale * kLog2e;
  if (!sl.counts) {
    if (thread<64>() == 0) skip_logp<PREF>(a, slot, sl);
    return;
  }
  const RowSum r = join_parts(a.parts + (size_t)slot * n_parts, n_parts, c);
  if (thread<64>() == 0) write_logp<PREF>(a, slot, sl, a.zy[slot], c, r, logp_ref);
}

template <typename T, int NT, int U>
__global__ __launch_bounds__(NT) void split_policy_kernel(TokenArgs a, PolicyArgs p) {
  const uint32_t slot = blockIdx.x;
  const Slot sl = slot_of(a, slot);
  const Range g = part_of(a);
  const bool first = blockIdx.y == 0 && threadIdx.x == 0;
  T* out = a.dlogits ? (T*)a.dlogits + sl.row * a.ldd + g.from : nullptr;
  if (!sl.counts) {
    if (first) p.token_loss[slot] = 0.f;
    if (!sl.write) return;
    if (first && a.logp) a.logp[sl.row] = 0.f;
    if (out) row_zero<T, NT>(out, g.n);
    return;
  }
  const PolicyToken in = policy_inputs(p, a, slot, sl);
  const float c = a.scale * kLog2e;
  const RowSum r = join_parts(a.parts + (size_t)slot * gridDim.y, gridDim.y, c);
  const float logp = (float)row_logp(a.zy[slot], c, r);
  const TokenLoss l = policy_token(p, in, logp);
  if (first) {
    p.token_loss[slot] = l.loss;
    if (a.logp) a.logp[sl.row] = logp;
  }
  const float cs = l.c * a.scale;
  if (out)
    row_grad_stream<T, NT, U>((const T*)a.logits + sl.row * a.ldl + g.from, out, g.n, sl.target - g.from, c, r, cs,
                              -cs / r.sum);
}

__device__ inline double block_sum(double v, double* sh) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  __syncthreads();
  return v;
}

// loss[i] = sum of example i's token losses, in fp64 in a fixed order.
__global__ __launch_bounds__(256) void example_sum_kernel(const float* __restrict__ token_loss, uint32_t T,
                                                          uint32_t n, float* __restrict__ loss) {
  __shared__ double sh[4];
  for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
    double v = 0.0;
    for (uint32_t t = threadIdx.x; t < T; t += 256) v += (double)token_loss[(size_t)i * T + t];
    v = block_sum(v, sh);
    if (threadIdx.x == 0) loss[i] = (float)v;
  }
}

// Sum over NT threads, the result in all of them.
template <int NT>
__device__ inline double threads_sum(double v, double* sh) {
  v = wave_sum(v);
  if (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v += sh[w];
  __syncthreads();
  return v;
}

// A pair's loss from its log ratios (written where `outputs`); returns the derivative
// by the log-probability of a chosen token of weight 1.  A pair of weight 0 has 0 of both,
// whatever its log ratios.
__device__ inline float pair_loss(const PrefArgs& p, uint32_t pair, const double (&ratio)[2], bool outputs) {
  const double h = (double)p.beta * (ratio[0] - ratio[1]) - (double)p.margin;
  const float pw = p.pair_weight ? p.pair_weight[pair] : 1.f, e = p.smoothing;
  if (outputs) {
    // softplus(x) = max(x, 0) + log1p(exp(-|x|)); a share of nothing is not taken of an
    // infinite ratio's loss
    const double tail = log1p(exp(-fabs(h)));
    const double won = e < 1.f ? (1.0 - (double)e) * (fmax(-h, 0.0) + tail) : 0.0;
    const double lost = e > 0.f ? (double)e * (fmax(h, 0.0) + tail) : 0.0;
    p.loss[pair] = pw != 0.f ? (float)((double)pw * (won + lost)) : 0.f;
    if (p.log_ratio) {
      p.log_ratio[pair] = (float)ratio[0];
      p.log_ratio[pair + p.n_pairs] = (float)ratio[1];
    }
  }
  return pw != 0.f ? pw * p.beta * (e / (1.f + expf((float)-h)) - (1.f - e) / (1.f + expf((float)h))) : 0.f;
}

// The same from the parts of its tokens, summed by NT threads.
template <int NT>
__device__ inline float pair_coefficient(const TokenArgs& a, const PrefArgs& p, uint32_t pair, bool outputs, double* sh) {
  double ratio[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const double* part = a.part + (size_t)(pair + side * p.n_pairs) * a.T;
    double v = 0.0;
    for (uint32_t t = thread<NT>(); t < a.T; t += NT) v += part[t];
    ratio[side] = threads_sum<NT>(v, sh);
  }
  return pair_loss(p, pair, ratio, outputs && thread<NT>() == 0);
}

__global__ __launch_bounds__(256) void pair_kernel(TokenArgs a, PrefArgs p) {
  __shared__ double sh[4];
  for (uint32_t pair = blockIdx.x; pair < p.n_pairs; pair += gridDim.x) {
    const float g = pair_coefficient<256>(a, p, pair, true, sh);
    if (threadIdx.x == 0) p.coef[pair] = g;
  }
}

// Short pairs of short rows in one launch: a workgroup a pair, a wave a chosen token and
// the rejected one beside it, both rows in registers between the sums and the gradient.
template <typename T, int NV>
__global__ __launch_bounds__(1024) void pref_pair_kernel(TokenArgs a, PrefArgs p) {
  __shared__ Shared sh;
  __shared__ double parts[2][kPrefPairMost];
  const uint32_t t = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pair = blockIdx.x;
  const float c = a.scale * kLog2e;
  Slot sl[2];
  float zy[2];
  RowRegs<T, 64, NV> row[2];
  RowSum r[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    sl[side] = slot_of(a, (pair + side * p.n_pairs) * a.T + t);
    if (!sl[side].counts) continue;
    const T* z = (const T*)a.logits + sl[side].row * a.ldl;
    zy[side] = (float)z[sl[side].target];
    row[side].load(z, a.V);
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    double part = 0.0;
    if (sl[side].counts) {
      bool ok;
      r[side] = row[side].sum(zy[side], c, sh, ok);
      if (!ok) r[side] = row_sum_apart<T, 64>(row[side].z, a.V, c, sh);
      part = token_part(a, sl[side], zy[side], c, r[side], p.logp_ref);
    } else if (thread<64>() == 0 && sl[side].write && a.logp) {
      a.logp[sl[side].row] = 0.f;
    }
    if (thread<64>() == 0) parts[side][t] = part;
  }
  __syncthreads();
  double ratio[2];
#pragma unroll
  for (int side = 0; side < 2; ++side)
    ratio[side] = wave_sum((uint32_t)thread<64>() < a.T ? parts[side][thread<64>()] : 0.0);
  const float g = pair_loss(p, pair, ratio, threadIdx.x == 0);
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    if (!a.dlogits || !sl[side].write) continue;
    T* out = (T*)a.dlogits + sl[side].row * a.ldd;
    const float cs = (side == 0 ? g : -g) * sl[side].weight * a.scale;
    if (!sl[side].counts || cs == 0.f) row_zero<T, 64>(out, a.V);
    else if (r[side].apart) row_grad_apart<T, 64>(row[side].z, out, a.V, sl[side].target, c, r[side], cs, -cs / r[side].sum);
    else row[side].grad(out, a.V, sl[side].target, c, r[side], cs);
  }
}

// PAIR: every row forms its pair's sums itself, and the pair's first slot writes its
// outputs; else they are there.  The grid's second dimension is a row's parts.
template <typename T, int NT, int U, bool PAIR>
__global__ __launch_bounds__(group_of(NT)) void pref_grad_kernel(TokenArgs a, PrefArgs p) {
  __shared__ double sh[16];
  const float c = a.scale * kLog2e;
  const uint32_t slot = a.slot0 + first_slot<NT>();
  if (slot >= a.n_slots) return;
  const Slot sl = slot_of(a, slot);
  const uint32_t i = slot / a.T, pair = i < p.n_pairs ? i : i - p.n_pairs;
  const bool outputs = PAIR && slot == pair * a.T && blockIdx.y == 0;
  const Range part = part_of(a);
  T* const out = (T*)a.dlogits + sl.row * a.ldd + part.from;
  float g = 0.f;
  if (PAIR && (sl.counts || outputs)) g = pair_coefficient<NT>(a, p, pair, outputs, sh);
  if (!sl.counts) {
    if (sl.write) row_zero<T, NT>(out, part.n);
    return;
  }
  if (!PAIR) g = p.coef[pair];
  const float2 st = a.stats[slot];
  const RowSum r{st.x, fabsf(st.y), 0.f, st.y < 0.f};
  const float cs = (i < p.n_pairs ? g : -g) * sl.weight * a.scale, ce = -cs / r.sum;
  if (cs == 0.f) return row_zero<T, NT>(out, part.n);  // also of a row that holds NaN, in a pair of weight 0
  row_grad_stream<T, NT, U>((const T*)a.logits + sl.row * a.ldl + part.from, out, part.n, sl.target - part.from, c, r,
                            cs, ce);
}

uint32_t blocks_for(uint32_t n) { return n < (1u << 20) ? n : (1u << 20); }

// Every slot's row swept by NT threads, in launches of fewer than 2^32 threads.
template <int NT, typename... K, typename... Args>
void launch_slots(void (*kernel)(TokenArgs, K...), TokenArgs a, hipStream_t s, Args... args) {
  constexpr uint32_t kMost = 1u << 21, kRows = group_of(NT) / NT;
  for (a.slot0 = 0; a.slot0 < a.n_slots; a.slot0 += kMost) {
    const uint32_t n = a.n_slots - a.slot0 < kMost ? a.n_slots - a.slot0 : kMost;
    hipLaunchKernelGGL(kernel, dim3((n + kRows - 1) / kRows, a.n_parts), dim3(group_of(NT)), 0, s, a, args...);
  }
}

template <typename T>
void launch_split_sum(const TokenArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((split_sum_kernel<T, 512, 4>), dim3(a.n_slots, a.n_parts), dim3(512), 0, s, a);
}

template <typename T, bool PREF>
void launch_logp(TokenArgs a, const float* ref, hipStream_t s) {
  const int64_t bytes = (int64_t)a.V * (int64_t)sizeof(T);
  if (a.n_parts > 1) {
    launch_split_sum<T>(a, s);
    hipLaunchKernelGGL((split_logp_kernel<PREF>), dim3((a.n_slots + 3) / 4), dim3(256), 0, s, a, (int32_t)a.n_parts, ref);
    return;
  }
  // Up to a row a CU, more threads a row finish it sooner (64 bf16 rows of 50257: 6.6 us,
  // 7.8 with 512); with more rows they cost (512 rows: 12.4 and 11.4).
  if (bytes <= 4096) launch_slots<64>(token_logp_kernel<T, 64, 4, PREF>, a, s, ref);
  else if (bytes > 16384 && bytes <= 131072 && a.n_slots <= 256)
    launch_slots<1024>(token_logp_kernel<T, 1024, 2, PREF>, a, s, ref);
  else if (bytes <= 65536) launch_slots<256>(token_logp_kernel<T, 256, 4, PREF>, a, s, ref);
  else if (bytes <= 131072) launch_slots<512>(token_logp_kernel<T, 512, 2, PREF>, a, s, ref);
  else launch_slots<512>(token_logp_kernel<T, 512, 4, PREF>, a, s, ref);
}

template <typename T>
void launch_policy(const TokenArgs& a, const PolicyArgs& p, hipStream_t s) {
  const int64_t bytes = (int64_t)a.V * (int64_t)sizeof(T);
  if (a.n_parts > 1) {
    launch_split_sum<T>(a, s);
    hipLaunchKernelGGL((split_policy_kernel<T, 512, 4>), dim3(a.n_slots, a.n_parts), dim3(512), 0, s, a, p);
    return;
  }
  // Threads and vectors by the row's bytes; us of 32768, 16384, 8192 or 6400 rows at the
  // neighbouring choices: bf16 1000 wide 29 (256 x 2: 62), 4000 wide 50 (256 x 8: 57),
  // 10000 wide 58 (512 x 8: 61), 16000 wide 89 (256 x 8: 94), 24000 wide 104 (1024 x 8:
  // 112), 32003 wide 140 (1024 x 8: 140), 65536 wide 282 (512 x 16: 283).  50257 wide 232
  // (512 x 16: 219), but 226 against 237 with half of the rows masked.
  if (bytes <= 4096) launch_slots<64>(policy_kernel<T, 64, 4>, a, s, p);
  else if (bytes <= 8192) launch_slots<256>(policy_kernel<T, 256, 2>, a, s, p);
  else if (bytes <= 24576) launch_slots<256>(policy_kernel<T, 256, 8>, a, s, p);
  else if (bytes <= 65536) launch_slots<512>(policy_kernel<T, 512, 8>, a, s, p);
  else if (bytes <= 131072) launch_slots<1024>(policy_kernel<T, 1024, 8>, a, s, p);
  else if (bytes <= 262144) launch_slots<1024>(policy_kernel<T, 1024, 16>, a, s, p);
  else launch_slots<1024>(policy_stream_kernel<T, 1024>, a, s, p);
}

template <typename T>
void launch_examples(const TokenArgs& a, const PolicyArgs& p, uint32_t n, float* loss, hipStream_t s) {
  if ((int64_t)a.V * (int64_t)sizeof(T) > 4096)
    hipLaunchKernelGGL((policy_example_kernel<T, 8, 1>), dim3(n), dim3(64 * a.T), 0, s, a, p, loss);
  else if (a.T <= 16)
    hipLaunchKernelGGL((policy_example_kernel<T, 4, 1>), dim3(n), dim3(64 * a.T), 0, s, a, p, loss);
  else
    hipLaunchKernelGGL((policy_example_kernel<T, 4, 2>), dim3(n), dim3(64 * ((a.T + 1) / 2)), 0, s, a, p, loss);
}

template <typename T, bool PAIR>
void launch_grad(const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  const int64_t bytes = (int64_t)a.V * (int64_t)sizeof(T);
  if (bytes <= 4096) launch_slots<64>(pref_grad_kernel<T, 64, 4, PAIR>, a, s, p);
  else if (bytes <= 65536) launch_slots<256>(pref_grad_kernel<T, 256, 4, PAIR>, a, s, p);
  else if (a.n_parts > 1) launch_slots<512>(pref_grad_kernel<T, 512, 4, PAIR>, a, s, p);
  else launch_slots<1024>(pref_grad_kernel<T, 1024, 2, PAIR>, a, s, p);
}

}  // namespace

hipError_t launch_token_logp(int dtype, const TokenArgs& a, hipStream_t s) {
  if (dtype == 0) launch_logp<float, false>(a, nullptr, s);
  else if (dtype == 1) launch_logp<__bf16, false>(a, nullptr, s);
  else launch_logp<_Float16, false>(a, nullptr, s);
  return hipGetLastError();
}

hipError_t launch_pref_stats(int dtype, const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  if (dtype == 0) launch_logp<float, true>(a, p.logp_ref, s);
  else if (dtype == 1) launch_logp<__bf16, true>(a, p.logp_ref, s);
  else launch_logp<_Float16, true>(a, p.logp_ref, s);
  return hipGetLastError();
}

// Parts of a row where there are fewer rows than CUs: of 32 KB or more, a thousand in
// all, from rows of more than 128 KB on (below, the launch that joins them takes as
// long as it saves: log-probabilities of one row of 100 KB 6.1 us whole, 8.4 in parts; of
// 64 bf16 rows of 100000 9.2 and 7.8, of 200 fp32 rows of 131072 26 and 21).  Where the
// gradient is read again in parts though a whole row's would be in registers, up to half
// as many rows (one bf16 row of 131072: 14.7 us whole, 7.8 in parts; 64: 15.4 and 10.4;
// 128 fp32 rows of 80000: 21.4 and 21.2; 200: 28.3 and 30.7).
int token_parts(int mode, int64_t n_slots, int64_t row_bytes) {
  const int64_t most = mode == kTokenPolicy ? 128 : 256;
  if (n_slots < 1 || n_slots >= most || row_bytes <= 131072) return 1;
  const int64_t by_size = (row_bytes + 32767) / 32768, by_count = (1024 + n_slots - 1) / n_slots;
  return (int)(by_size < by_count ? (by_size < 64 ? by_size : 64) : (by_count < 64 ? by_count : 64));
}

// Threads of a launch stay below 2^32.
constexpr int64_t kGroupsMost = 1 << 20;

// A second launch costs the host 3 us, what a call this small waits for: 8 examples of
// 32 rows of 4 KB take 7.6 us in one launch, 8.5 in two; 512 of 16 rows of 8 KB 23.8 and
// 24.7; 16384 of 4 of 4 KB 86 and 97.  Many long ones fill the card either way: 2048 of
// 32 rows of 4 KB 95 and 89.  Longer rows take too long in one wave: 16 rows of 16 KB,
// 15.2 against 6.6.
bool policy_by_example(int64_t row_bytes, int64_t T, int64_t n) {
  if (T < 2 || n > kGroupsMost || (T > 8 && n * T > 16384)) return false;
  return row_bytes <= 4096 ? T <= kPolicyExampleMost : row_bytes <= 8192 && T <= 16;
}

hipError_t launch_policy_examples(int dtype, const TokenArgs& a, const PolicyArgs& p, uint32_t n, float* loss,
                                  hipStream_t s) {
  if (dtype == 0) launch_examples<float>(a, p, n, loss, s);
  else if (dtype == 1) launch_examples<__bf16>(a, p, n, loss, s);
  else launch_examples<_Float16>(a, p, n, loss, s);
  return hipGetLastError();
}

hipError_t launch_policy_rows(int dtype, const TokenArgs& a, const PolicyArgs& p, hipStream_t s) {
  if (dtype == 0) launch_policy<float>(a, p, s);
  else if (dtype == 1) launch_policy<__bf16>(a, p, s);
  else launch_policy<_Float16>(a, p, s);
  return hipGetLastError();
}

hipError_t launch_example_sum(const float* token_loss, uint32_t T, uint32_t n, float* loss, hipStream_t s) {
  hipLaunchKernelGGL(example_sum_kernel, dim3(blocks_for(n)), dim3(256), 0, s, token_loss, T, n, loss);
  return hipGetLastError();
}

// Pairs of short rows at once: 32 pairs of 16 tokens and rows of 4 KB 9.3 us, 13.1 in
// two launches; 2048 of 8 tokens 48 and 68 (4 of 16 tokens of 8 KB: 10.5 and 8.8).
bool pref_by_pair(int64_t row_bytes, int64_t T, int64_t n_pairs) {
  return row_bytes <= 8192 && T <= kPrefPairMost && n_pairs <= kGroupsMost;
}

// Every row adds up its pair's tokens itself instead of a launch between the two: 192
// tokens of 32 KB take 10.5 us, 13.7 with it; 2048 of 16 KB 16.2 and 17.9; 4096 of 4 KB in
// sequences of 512 16.4 and 14.8.  Of long rows, whose workgroups are large, fewer: 800 of
// 100 KB take 49.2 and 46.4.
bool pref_pairs_within(int64_t row_bytes, int64_t T, int64_t n_slots) {
  return T <= 1024 && n_slots <= (row_bytes <= 65536 ? 2048 : 512);
}

hipError_t launch_pref_pairs(int dtype, const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  const dim3 grid(p.n_pairs), block(64 * a.T);
  if (dtype == 0) hipLaunchKernelGGL((pref_pair_kernel<float, 8>), grid, block, 0, s, a, p);
  else if (dtype == 1) hipLaunchKernelGGL((pref_pair_kernel<__bf16, 8>), grid, block, 0, s, a, p);
  else hipLaunchKernelGGL((pref_pair_kernel<_Float16, 8>), grid, block, 0, s, a, p);
  return hipGetLastError();
}

hipError_t launch_pairs(const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  hipLaunchKernelGGL(pair_kernel, dim3(blocks_for(p.n_pairs)), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

hipError_t launch_pref_grad(int dtype, bool pair, const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  if (dtype == 0) pair ? launch_grad<float, true>(a, p, s) : launch_grad<float, false>(a, p, s);
  else if (dtype == 1) pair ? launch_grad<__bf16, true>(a, p, s) : launch_grad<__bf16, false>(a, p, s);
  else pair ? launch_grad<_Float16, true>(a, p, s) : launch_grad<_Float16, false>(a, p, s);
  return hipGetLastError();
}

}  // namespace attr
