// One AdamW step over many tensors (attr_adamw_step).
//
// The descriptors travel in kernel arguments; a workgroup finds its tensor by
// its first chunk and takes one chunk of it.  Arithmetic is fp32 and never
// contracted into fused multiply-adds: every element's result is the same
// however the tensors are split over workgroups.
#include "common.h"
#include "kernels.h"

#pragma clang fp contract(off)

namespace attr {
namespace {

constexpr int kQuantBlock = 256;       // elements that share a scale of the 8-bit states
constexpr float kE4M3Max = 448.f;
constexpr float kE4M3Least = 0.001953125f;  // 2^-9, the smallest positive value
constexpr float kAmaxLeast = 0x1p-100f;     // below it 448 / amax nears fp32's range

__device__ inline float e4m3_value(uint8_t code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
__device__ inline uint8_t e4m3_code(float x) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
}

struct Step {
  float m, v, x;
};
__device__ inline Step adamw_element(const AdamwArgs& a, float lr, float lr_wd, float x, float g, float m,
                                     float v) {
  m = m * a.beta1 + g * a.one_beta1;
  v = v * a.beta2 + (g * g) * a.one_beta2;
  const float root = sqrtf(v * a.corr2 + a.eps_root) + a.eps;
  x = x - x * lr_wd - (m * a.corr1) / root * lr;
  return {m, v, x};
}

// largest magnitude of a 256-thread workgroup's values, as fp32 bits: integer
// order keeps infinities and NaN above every finite value
__device__ inline uint32_t block_amax(float x, uint32_t* sh) {
  uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)b, off, kWave);
    b = o > b ? o : b;
  }
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = b;
  __syncthreads();
  const uint32_t p = sh[0] > sh[1] ? sh[0] : sh[1], q = sh[2] > sh[3] ? sh[2] : sh[3];
  __syncthreads();
  return p > q ? p : q;
}

template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a) {
  __shared__ uint32_t sh[4];
  int lo = 0, hi = a.n - 1;  // the last tensor whose first chunk is not past this workgroup
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.e[mid].chunk0 <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwEntry& t = a.e[lo];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float lr = t.lr, lr_wd = t.lr_wd;
  const int64_t i0 = (int64_t)(blockIdx.x - t.chunk0) * kAdamwChunk;
  for (int64_t b = i0; b < t.n && b < i0 + kAdamwChunk; b += 256) {
    const int64_t i = b + threadIdx.x;
    const bool in = i < t.n;
    float x = 0.f, g = 0.f, m = 0.f, v = 0.f;
    if (in) {
      x = t.master ? t.master[i] : (float)((const P*)t.p)[i];
      g = (float)((const G*)t.g)[i] * gs;
      if (EIGHT) {
        m = e4m3_value(((const uint8_t*)t.m)[i]) * t.m_scale[b / kQuantBlock];
        v = e4m3_value(((const uint8_t*)t.v)[i]) * t.v_scale[b / kQuantBlock];
        v = v * v;
      } else {
        m = ((const float*)t.m)[i];
        v = ((const float*)t.v)[i];
      }
    }
    const Step r = adamw_element(a, lr, lr_wd, x, g, m, v);
    if (in) {
      if (t.master) t.master[i] = r.x;
      ((P*)t.p)[i] = (P)r.x;
    }
    if (EIGHT) {
      const float root = sqrtf(r.v);
      float am = __builtin_bit_cast(float, block_amax(in ? r.m : 0.f, sh));
      float av = __builtin_bit_cast(float, block_amax(in ? root : 0.f, sh));
      am = am < kAmaxLeast ? kAmaxLeast : am;
      av = av < kAmaxLeast ? kAmaxLeast : av;
      if (in) {
        ((uint8_t*)t.m)[i] = e4m3_code(r.m * (1.f / am * kE4M3Max));
        const float q = root * (1.f / av * kE4M3Max);
        ((uint8_t*)t.v)[i] = e4m3_code(q > 0.f && q < kE4M3Least ? kE4M3Least : q);
      }
      if (threadIdx.x == 0) {
        t.m_scale[b / kQuantBlock] = am < INFINITY ? am * (1.f / kE4M3Max) : NAN;
        t.v_scale[b / kQuantBlock] = av < INFINITY ? av * (1.f / kE4M3Max) : NAN;
      }
    } else if (in) {
      ((float*)t.m)[i] = r.m;
      ((float*)t.v)[i] = r.v;
    }
  }
}

template <typename P, typename G>
void launch(bool eight, uint32_t blocks, const AdamwArgs& a, hipStream_t s) {
  if (eight) hipLaunchKernelGGL((adamw_kernel<P, G, true>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adamw_kernel<P, G, false>), dim3(blocks), dim3(256), 0, s, a);
}
template <typename P>
void launch_g(int g_dtype, bool eight, uint32_t blocks, const AdamwArgs& a, hipStream_t s) {
  if (g_dtype == 0) launch<P, float>(eight, blocks, a, s);
  else if (g_dtype == 1) launch<P, __bf16>(eight, blocks, a, s);
  else launch<P, _Float16>(eight, blocks, a, s);
}

}  // namespace

hipError_t launch_adamw(int p_dtype, int g_dtype, bool eight, uint32_t blocks, const AdamwArgs& a,
                        hipStream_t s) {
  if (p_dtype == 0) launch_g<float>(g_dtype, eight, blocks, a, s);
  else if (p_dtype == 1) launch_g<__bf16>(g_dtype, eight, blocks, a, s);
  else launch_g<_Float16>(g_dtype, eight, blocks, a, s);
  return hipGetLastError();
}

}  // namespace attr
