// Attention of a band's queries over fresh K/V and the 8-bit cache: one thread a
// query, online softmax with the running max and sum.
#include "common.h"
#include "kernels.h"

namespace orch {

template <typename T, int D>
__global__ __launch_bounds__(64) void attn_quantized_kernel(AttnQParams p) {
  const int q = blockIdx.x * 64 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
  if (q >= p.n_q) return;
  const size_t H = (size_t)p.heads * D;
  const int N = p.c.tokens;
  const T* qv = reinterpret_cast<const T*>(p.q) + (((size_t)b * p.heads + h) * p.n_q + q) * D;
  const unsigned char* vals = p.c.values + b * p.c.values_bs;
  const unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  const T* kf = reinterpret_cast<const T*>(p.kv_fresh) + b * p.fresh_bs + (size_t)h * p.n_fresh * D;
  const T* vf = reinterpret_cast<const T*>(p.kv_fresh) + b * p.fresh_bs + p.n_fresh * H + (size_t)h * D * p.n_fresh;
  float qr[D], acc[D];
  const float scale = 1.4426950408889634f / sqrtf((float)D);
#pragma unroll
  for (int d = 0; d < D; ++d) {
    qr[d] = to_f<T>(qv[d]);
    acc[d] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int n = 0; n < N; ++n) {
    const int f = n - p.fresh_begin;
    const bool fresh = (unsigned)f < (unsigned)p.n_fresh;
    const size_t kr = (size_t)h * N + n, vr = (size_t)(p.heads + h) * N + n;
    const float ke = __uint_as_float((unsigned)exps[kr] << 23), ve = __uint_as_float((unsigned)exps[vr] << 23);
    float s = 0.0f;
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const float k = fresh ? to_f<T>(kf[(size_t)f * D + d]) : __builtin_amdgcn_cvt_scalef32_f32_fp8((unsigned)vals[kr * D + d], ke, 0);
      s = fmaf(qr[d], k, s);
    }
    s *= scale;
    const float mn = fmaxf(m, s);
    const float a = exp2f(m - mn), e = exp2f(s - mn);
    l = l * a + e;
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const float v = fresh ? to_f<T>(vf[(size_t)d * p.n_fresh + f]) : __builtin_amdgcn_cvt_scalef32_f32_fp8((unsigned)vals[vr * D + d], ve, 0);
      acc[d] = fmaf(acc[d], a, e * v);
    }
    m = mn;
  }
  T* o = reinterpret_cast<T*>(p.out) + ((size_t)b * p.n_q + q) * H + h * D;
  const float inv = 1.0f / l;
#pragma unroll
  for (int d = 0; d < D; ++d) o[d] = from_f<T>(acc[d] * inv);
}

size_t attention_quantized_workspace_bytes(int, int, int, int, int, int) { return 0; }

template <typename T>
static hipError_t launch_simple(const AttnQParams& p, hipStream_t s) {
  dim3 grid(ceil_div(p.n_q, 64), p.heads, p.B);
  switch (p.d) {
    case 32: hipLaunchKernelGGL((attn_quantized_kernel<T, 32>), grid, dim3(64), 0, s, p); break;
    case 64: hipLaunchKernelGGL((attn_quantized_kernel<T, 64>), grid, dim3(64), 0, s, p); break;
    case 72: hipLaunchKernelGGL((attn_quantized_kernel<T, 72>), grid, dim3(64), 0, s, p); break;
    case 80: hipLaunchKernelGGL((attn_quantized_kernel<T, 80>), grid, dim3(64), 0, s, p); break;
    case 96: hipLaunchKernelGGL((attn_quantized_kernel<T, 96>), grid, dim3(64), 0, s, p); break;
    case 128: hipLaunchKernelGGL((attn_quantized_kernel<T, 128>), grid, dim3(64), 0, s, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_attention_quantized(const AttnQParams& p, int dtype, hipStream_t s) {
  if (p.n_q <= 0) return hipSuccess;
  return dtype == kBF16 ? launch_simple<bf16>(p, s) : launch_simple<float>(p, s);
}

}  // namespace orch
