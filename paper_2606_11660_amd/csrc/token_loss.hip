// Log-probabilities of given tokens, the clipped policy loss with a KL term and
// the paired log-ratio preference loss, with their gradients with respect to
// the logits.
//
// A row's log-probability is s (z_y - m) - log S with m = max_j z_j and
// S = sum_j exp(s (z_j - m)); the differences are formed first, so large or
// lowest-value logits neither overflow nor cancel.  The gradient of any loss
// with derivative c by that log-probability is s c ([j = y] - e_j / S), e_j the
// same exponentials.
#include "common.h"
#include "kernels.h"

namespace attr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// What a workgroup does with one token's slot.
struct Slot {
  int64_t row;
  int32_t target;   // in [0, V) where counts
  bool write;       // the row's outputs are written
  bool counts;      // its logits are read
};

// Token slot of a batch: example slot / T, token slot % T (attr_token_rows).
__device__ inline Slot slot_of(const TokenArgs& a, uint32_t slot) {
  const uint32_t i = slot / a.T, t = slot - i * a.T;
  Slot r;
  bool in = true;
  if (a.length) in = (int64_t)t < (int64_t)a.length[i];
  r.row = a.row_offset ? a.row_offset[i] + t : (int64_t)slot;
  const bool inside = r.row >= 0 && r.row < a.n_rows;
  r.write = inside && (in || !a.row_offset);
  r.counts = inside && in;
  r.target = 0;
  if (r.counts) {
    const int64_t y = a.target[r.row];
    r.counts = y >= 0 && y < a.V && !(a.weight && a.weight[r.row] == 0.f);
    r.target = (int32_t)y;
  }
  return r;
}

template <typename T>
__device__ inline float as_f32(T x) { return (float)x; }

// A running maximum of logits and the sum of exp2(c (z - max)), c = s log2 e.
struct MaxSum {
  float m, s;
};
__device__ inline MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  // a side that holds nothing (-inf) adds nothing; NaN stays NaN through its sum
  const float sa = a.m == m ? a.s : a.s * __builtin_amdgcn_exp2f((a.m - m) * c);
  const float sb = b.m == m ? b.s : b.s * __builtin_amdgcn_exp2f((b.m - m) * c);
  return {m, sa + sb};
}
__device__ inline MaxSum wave_join(MaxSum v, float c) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    v = join(v, MaxSum{__shfl_xor(v.m, off, kWave), __shfl_xor(v.s, off, kWave)}, c);
  return v;
}

// Loss and derivative by logp of one token of the policy loss, weights included.
struct TokenLoss {
  float loss, c;
};
__device__ inline TokenLoss policy_token(const PolicyArgs& p, const TokenArgs& a, uint32_t slot,
                                         int64_t row, float logp) {
  const float w = a.weight ? a.weight[row] : 1.f;
  const float adv = p.advantage[p.per_token ? row : (int64_t)(slot / a.T)];
  const float ratio = p.logp_old ? expf(logp - p.logp_old[row]) : logp == logp ? 1.f : logp;
  const float free_ = -adv * ratio;
  const float held = -adv * fminf(fmaxf(ratio, p.lo), p.hi);
  float loss = free_ >= held ? free_ : held, c = free_ >= held ? free_ : 0.f;
  if (ratio != ratio) loss = c = ratio;  // a NaN stays
  if (p.beta != 0.f) {
    const float d = p.logp_ref[row] - logp, less = expm1f(d);
    loss += p.beta * (less - d);
    c -= p.beta * less;
  }
  return {w * loss, w * c};
}

template <typename T, int MODE>
__global__ __launch_bounds__(256) void token_kernel(TokenArgs a, PolicyArgs p) {
  __shared__ MaxSum sh[4];
  const float c = a.scale * kLog2e;
  for (uint32_t slot = blockIdx.x; slot < a.n_slots; slot += gridDim.x) {
    const Slot sl = slot_of(a, slot);
    T* out = a.dlogits ? (T*)a.dlogits + sl.row * a.ldd : nullptr;
    if (!sl.counts) {
      if (threadIdx.x == 0) {
        if (sl.write && a.logp) a.logp[sl.row] = 0.f;
        if (MODE == kTokenPolicy) p.token_loss[slot] = 0.f;
      }
      if (sl.write && out)
        for (int32_t j = threadIdx.x; j < a.V; j += 256) out[j] = (T)0.f;
      continue;
    }
    const T* z = (const T*)a.logits + sl.row * a.ldl;
    const float zy = as_f32(z[sl.target]);
    MaxSum v{-INFINITY, 0.f};
    for (int32_t j = threadIdx.x; j < a.V; j += 256) {
      const float x = as_f32(z[j]);
      v = join(v, MaxSum{x, x == -INFINITY ? 0.f : 1.f}, c);
      if (x != x) v.s = x;
    }
    v = wave_join(v, c);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = join(join(sh[0], sh[1], c), join(sh[2], sh[3], c), c);
    __syncthreads();
    if (v.m == INFINITY) v.s = NAN;
    const float logp = (zy - v.m) * a.scale - logf(v.s);
    if (MODE == kTokenPref) {
      if (threadIdx.x == 0) {
        a.stats[slot] = float2{v.m, v.s};
        a.slot_logp[slot] = logp;
      }
    }
    if (threadIdx.x == 0 && a.logp) a.logp[sl.row] = logp;
    if (MODE != kTokenPolicy) continue;
    const TokenLoss l = policy_token(p, a, slot, sl.row, logp);
    if (threadIdx.x == 0) p.token_loss[slot] = l.loss;
    if (!out) continue;
    const float cs = l.c * a.scale, ce = -cs / v.s;
    for (int32_t j = threadIdx.x; j < a.V; j += 256) {
      float d = ce * __builtin_amdgcn_exp2f((as_f32(z[j]) - v.m) * c);
      if (j == sl.target) d += cs;
      out[j] = (T)d;
    }
  }
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

__device__ inline double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

// A pair's log ratios, its loss and the derivative by its log-probabilities.
__global__ __launch_bounds__(256) void pair_kernel(TokenArgs a, PrefArgs p) {
  __shared__ double sh[4];
  for (uint32_t pair = blockIdx.x; pair < p.n_pairs; pair += gridDim.x) {
    double ratio[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const uint32_t i = pair + side * p.n_pairs;
      double v = 0.0;
      for (uint32_t t = threadIdx.x; t < a.T; t += 256) {
        const uint32_t slot = i * a.T + t;
        const Slot sl = slot_of(a, slot);
        if (!sl.counts) continue;
        const double d = (double)a.slot_logp[slot] - (p.logp_ref ? (double)p.logp_ref[sl.row] : 0.0);
        v += (a.weight ? (double)a.weight[sl.row] : 1.0) * d;
      }
      ratio[side] = block_sum(v, sh);
    }
    if (threadIdx.x != 0) continue;
    const double h = (double)p.beta * (ratio[0] - ratio[1]) - (double)p.margin, e = (double)p.smoothing;
    const double pw = p.pair_weight ? (double)p.pair_weight[pair] : 1.0;
    p.loss[pair] = (float)(pw * ((1.0 - e) * softplus(-h) + e * softplus(h)));
    if (p.log_ratio) {
      p.log_ratio[pair] = (float)ratio[0];
      p.log_ratio[pair + p.n_pairs] = (float)ratio[1];
    }
    p.coef[pair] = (float)(pw * (double)p.beta * (e / (1.0 + exp(-h)) - (1.0 - e) / (1.0 + exp(h))));
  }
}

template <typename T>
__global__ __launch_bounds__(256) void pref_grad_kernel(TokenArgs a, PrefArgs p) {
  const float c = a.scale * kLog2e;
  for (uint32_t slot = blockIdx.x; slot < a.n_slots; slot += gridDim.x) {
    const Slot sl = slot_of(a, slot);
    if (!sl.write) continue;
    T* out = (T*)a.dlogits + sl.row * a.ldd;
    if (!sl.counts) {
      for (int32_t j = threadIdx.x; j < a.V; j += 256) out[j] = (T)0.f;
      continue;
    }
    const T* z = (const T*)a.logits + sl.row * a.ldl;
    const float2 st = a.stats[slot];
    const uint32_t i = slot / a.T;
    const float w = a.weight ? a.weight[sl.row] : 1.f;
    const float cs = (i < p.n_pairs ? p.coef[i] : -p.coef[i - p.n_pairs]) * w * a.scale, ce = -cs / st.y;
    for (int32_t j = threadIdx.x; j < a.V; j += 256) {
      float d = ce * __builtin_amdgcn_exp2f((as_f32(z[j]) - st.x) * c);
      if (j == sl.target) d += cs;
      out[j] = (T)d;
    }
  }
}

uint32_t blocks_for(uint32_t n) { return n < (1u << 20) ? n : (1u << 20); }

}  // namespace

hipError_t launch_token_rows(int mode, int dtype, const TokenArgs& a, const PolicyArgs& p, hipStream_t s) {
  const dim3 grid(blocks_for(a.n_slots)), block(256);
#define ATTR_TOKEN(T, M) hipLaunchKernelGGL((token_kernel<T, M>), grid, block, 0, s, a, p)
  if (dtype == 0) {
    if (mode == kTokenLogp) ATTR_TOKEN(float, kTokenLogp);
    else if (mode == kTokenPolicy) ATTR_TOKEN(float, kTokenPolicy);
    else ATTR_TOKEN(float, kTokenPref);
  } else if (dtype == 1) {
    if (mode == kTokenLogp) ATTR_TOKEN(__bf16, kTokenLogp);
    else if (mode == kTokenPolicy) ATTR_TOKEN(__bf16, kTokenPolicy);
    else ATTR_TOKEN(__bf16, kTokenPref);
  } else {
    if (mode == kTokenLogp) ATTR_TOKEN(_Float16, kTokenLogp);
    else if (mode == kTokenPolicy) ATTR_TOKEN(_Float16, kTokenPolicy);
    else ATTR_TOKEN(_Float16, kTokenPref);
  }
#undef ATTR_TOKEN
  return hipGetLastError();
}

hipError_t launch_example_sum(const float* token_loss, uint32_t T, uint32_t n, float* loss, hipStream_t s) {
  hipLaunchKernelGGL(example_sum_kernel, dim3(blocks_for(n)), dim3(256), 0, s, token_loss, T, n, loss);
  return hipGetLastError();
}

hipError_t launch_pairs(const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  hipLaunchKernelGGL(pair_kernel, dim3(blocks_for(p.n_pairs)), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

hipError_t launch_pref_grad(int dtype, const TokenArgs& a, const PrefArgs& p, hipStream_t s) {
  const dim3 grid(blocks_for(a.n_slots)), block(256);
  if (dtype == 0) hipLaunchKernelGGL(pref_grad_kernel<float>, grid, block, 0, s, a, p);
  else if (dtype == 1) hipLaunchKernelGGL(pref_grad_kernel<__bf16>, grid, block, 0, s, a, p);
  else hipLaunchKernelGGL(pref_grad_kernel<_Float16>, grid, block, 0, s, a, p);
  return hipGetLastError();
}

}  // namespace attr
