// The 8-bit K/V cache: a band's K/V quantised as they are written, and the cache
// read back into a K/V buffer of the operand type.
//
// A token's d channels of one head share the scale s, the smallest power of two
// with max |x| <= 448 s: x / s and value * s are exact, so rounding to e4m3 (4
// significant bits, relative 2^-4) is the only error, and it keeps its relative
// size over 2^15 below the largest.  A power of two loses nothing against max / 448
// there, takes one byte (E8M0), and is what the conversion instructions take as
// their scale.  K rows are contiguous in both layouts; V is transposed (V^T
// [d][tokens] in the buffer, token-major in the cache) through LDS in tiles of 64
// tokens.  One read and one write of every element: bound by memory.
#include "common.h"
#include "kernels.h"

namespace orch {

namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;       // tokens of a V tile

// |x| as an ordered integer, zero where x is not finite
__device__ __forceinline__ unsigned finite_bits(float x) {
  const unsigned u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}

// E8M0 byte of the smallest power of two s >= 2^-126 with amax <= 448 s (448 = 1.75 2^8)
__device__ __forceinline__ unsigned scale_byte(unsigned amax) {
  const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (unsigned)max(e, 1);
}
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Two values over the scale s as e4m3 bytes, in the low half of the result.  The
// instruction divides by s and rounds to nearest even; what it cannot hold (only
// infinities, the scale keeps the rest within 448) and NaN become NaN.  Past 15 / 8
// 2^127 the nearest e4m3 multiple of 2^120 would be 2^128, no number: those go down.
__device__ __forceinline__ unsigned to_e4m3(float a, float b, float s) {
  constexpr float kTop = 0x1.ep127f;
  auto clip = [](float x) __attribute__((always_inline)) {
    return fabsf(x) > kTop && fabsf(x) < __builtin_inff() ? copysignf(kTop, x) : x;
  };
  const s16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, clip(a), clip(b), s, false);
  return (unsigned short)r[0];
}

template <typename T>
__device__ __forceinline__ void load8(const T* src, bool vec, int count, float (&v)[8]) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  if (vec) {
    const vec8 x = *reinterpret_cast<const vec8*>(src);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f<T>(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? to_f<T>(src[e]) : 0.0f;
  }
}

// G lanes take a K row of d = 8 x chunks channels, a chunk each.
__host__ __device__ inline int row_lanes(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : 16; }

struct Launch {
  KvCacheParams p;
  int k_blocks;      // workgroups of one (branch, head) on K; the rest take V tiles
  int vec;           // V^T rows and offsets in whole 16-byte chunks
};

template <typename T>
__global__ __launch_bounds__(256) void kv_quantize_kernel(Launch L) {
  const KvCacheParams& p = L.p;
  const int b = blockIdx.y / p.heads, h = blockIdx.y - b * p.heads, tid = threadIdx.x;
  const size_t H = (size_t)p.heads * p.d;
  const T* kv = reinterpret_cast<const T*>(p.kv) + b * p.kv_bs;
  unsigned char* vals = p.c.values + b * p.c.values_bs;
  unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  if ((int)blockIdx.x < L.k_blocks) {
    const int G = row_lanes(p.d), ch = tid % G;
    const int n = blockIdx.x * (256 / G) + tid / G;
    const bool on = n < p.n && ch * 8 < p.d;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (on) load8(kv + ((size_t)h * p.kv_tokens + p.kv_off + n) * p.d + ch * 8, true, 8, v);
    unsigned amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, finite_bits(v[e]));
    for (int o = 1; o < G; o <<= 1) amax = max(amax, (unsigned)__shfl_xor((int)amax, o, kWave));
    if (!on) return;
    const unsigned e8 = scale_byte(amax);
    const float s = scale_of(e8);
    const size_t row = (size_t)h * p.c.tokens + p.c_off + n;
    u32x2 w;
    w[0] = to_e4m3(v[0], v[1], s) | to_e4m3(v[2], v[3], s) << 16;
    w[1] = to_e4m3(v[4], v[5], s) | to_e4m3(v[6], v[7], s) << 16;
    *reinterpret_cast<u32x2*>(vals + row * p.d + ch * 8) = w;
    if (ch == 0) exps[row] = (unsigned char)e8;
    return;
  }
  // V: thread (cl, tg) holds tokens 8 tg .. +8 of channels cl + 32 i
  __shared__ unsigned red[4][kTile];
  __shared__ __attribute__((aligned(16))) unsigned char tile[kTile * 136];
  const int n0 = (blockIdx.x - L.k_blocks) * kTile;
  const int tg = tid & 7, cl = tid >> 3, pitch = p.d + 8;
  const int count = min(max(p.n - n0 - 8 * tg, 0), 8);
  const T* vt = kv + p.kv_tokens * H + (size_t)h * p.d * p.kv_tokens + p.kv_off + n0 + 8 * tg;
  float v[4][8];
  unsigned amax[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = cl + 32 * i;
    if (c < p.d && count > 0) load8(vt + (size_t)c * p.kv_tokens, L.vec && count == 8, count, v[i]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax[e] = max(amax[e], finite_bits(v[i][e]));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) amax[e] = max(amax[e], (unsigned)__shfl_xor((int)amax[e], o, kWave));
    if ((tid & 63) < 8) red[tid >> 6][8 * tg + e] = amax[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = 8 * tg + e;
    const unsigned e8 = scale_byte(max(max(red[0][t], red[1][t]), max(red[2][t], red[3][t])));
    const float s = scale_of(e8);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (cl + 32 * i < p.d) tile[t * pitch + cl + 32 * i] = (unsigned char)to_e4m3(v[i][e], 0.0f, s);
    if (cl == 0 && e < count)
      exps[(size_t)(p.heads + h) * p.c.tokens + p.c_off + n0 + t] = (unsigned char)e8;
  }
  __syncthreads();
  unsigned char* dst = vals + ((size_t)(p.heads + h) * p.c.tokens + p.c_off + n0) * p.d;
  const int chunks = p.d / 8, total = min(kTile, p.n - n0) * chunks;
  for (int i = tid; i < total; i += 256) {
    const int t = i / chunks, ch = i - t * chunks;
    *reinterpret_cast<u32x2*>(dst + (size_t)i * 8) = *reinterpret_cast<const u32x2*>(tile + t * pitch + ch * 8);
  }
}

// the 8 values of two words of e4m3 bytes, times s
__device__ __forceinline__ void from_e4m3(u32x2 w, float s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], s, false);
    const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], s, true);
    v[4 * i] = lo[0];
    v[4 * i + 1] = lo[1];
    v[4 * i + 2] = hi[0];
    v[4 * i + 3] = hi[1];
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* dst, bool vec, int count, const float (&v)[8]) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  if (vec) {
    vec8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = from_f<T>(v[e]);
    *reinterpret_cast<vec8*>(dst) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) dst[e] = from_f<T>(v[e]);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void kv_dequantize_kernel(Launch L) {
  const KvCacheParams& p = L.p;
  const int b = blockIdx.y / p.heads, h = blockIdx.y - b * p.heads, tid = threadIdx.x;
  const size_t H = (size_t)p.heads * p.d;
  T* kv = reinterpret_cast<T*>(p.kv) + b * p.kv_bs;
  const unsigned char* vals = p.c.values + b * p.c.values_bs;
  const unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  if ((int)blockIdx.x < L.k_blocks) {
    const int G = row_lanes(p.d), ch = tid % G;
    const int n = blockIdx.x * (256 / G) + tid / G;
    if (n >= p.n || ch * 8 >= p.d) return;
    const size_t row = (size_t)h * p.c.tokens + p.c_off + n;
    float v[8];
    from_e4m3(*reinterpret_cast<const u32x2*>(vals + row * p.d + ch * 8), scale_of(exps[row]), v);
    store8(kv + ((size_t)h * p.kv_tokens + p.kv_off + n) * p.d + ch * 8, true, 8, v);
    return;
  }
  __shared__ __attribute__((aligned(16))) unsigned char tile[kTile * 136];
  const int n0 = (blockIdx.x - L.k_blocks) * kTile;
  const int chunks = p.d / 8, total = min(kTile, p.n - n0) * chunks, pitch = p.d + 8;
  const size_t row0 = (size_t)(p.heads + h) * p.c.tokens + p.c_off + n0;
  for (int i = tid; i < total; i += 256) {
    const int t = i / chunks, ch = i - t * chunks;
    *reinterpret_cast<u32x2*>(tile + t * pitch + ch * 8) = *reinterpret_cast<const u32x2*>(vals + row0 * p.d + (size_t)i * 8);
  }
  __syncthreads();
  const int tg = tid & 7, cl = tid >> 3;
  const int count = min(max(p.n - n0 - 8 * tg, 0), 8);
  if (count == 0) return;
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = scale_of(e < count ? exps[row0 + 8 * tg + e] : 127u);
  T* vt = kv + p.kv_tokens * H + (size_t)h * p.d * p.kv_tokens + p.kv_off + n0 + 8 * tg;
  for (int c = cl; c < p.d; c += 32) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = e < count ? __builtin_amdgcn_cvt_scalef32_f32_fp8((unsigned)tile[(8 * tg + e) * pitch + c], s[e], 0) : 0.0f;
    store8(vt + (size_t)c * p.kv_tokens, L.vec && count == 8, count, v);
  }
}

template <typename K>
hipError_t launch(K kern, const KvCacheParams& p, int esize, hipStream_t s) {
  if (p.n <= 0) return hipSuccess;
  Launch L;
  L.p = p;
  L.k_blocks = ceil_div(p.n, 256 / row_lanes(p.d));
  L.vec = p.kv_tokens % 8 == 0 && p.kv_off % 8 == 0;
  hipLaunchKernelGGL(kern, dim3(L.k_blocks + ceil_div(p.n, kTile), p.heads * p.B), dim3(256), 0, s, L);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_quantize(const KvCacheParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch(kv_quantize_kernel<bf16>, p, 2, s) : launch(kv_quantize_kernel<float>, p, 4, s);
}

hipError_t launch_kv_dequantize(const KvCacheParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch(kv_dequantize_kernel<bf16>, p, 2, s) : launch(kv_dequantize_kernel<float>, p, 4, s);
}

}  // namespace orch
