// The 8-bit K/V cache: a band's K/V quantised as they are written, and the cache
// read back into a K/V buffer of the operand type.
//
// A token's d channels of one head share the scale s, the smallest power of two
// with max |x| <= 448 s: x / s and value * s are exact, so rounding to e4m3 (4
// significant bits) is the only error: at most 2^-4 of a value down to 2^-6 s, 2^13.8 to 2^14.8 below the largest, and
// 2^-10 s below that.  A power of two loses nothing against max / 448
// there, takes one byte (E8M0), and is what the conversion instructions take as
// their scale.  K rows are contiguous in both layouts; V is transposed (V^T
// [d][tokens] in the buffer, token-major in the cache) through LDS in tiles of 64
// tokens, each lane with 8 tokens x 4 channels of it in registers.  One read and one write of every element: bound by
// memory.  d = 72, 2 x 16 heads, bf16: 16384 tokens written in 51 us (228 MB, 4.5 TB/s) and read back in 35 (6.5,
// part of it from the caches); 1664 tokens of 4096 written in 9.5-10 us (23 MB), 4096 read back in 9.5-10 (57 MB).
// Workgroups of 64 tokens of one head: the V ones take longer and start first.
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

// max over the 8 lanes of an aligned group, on the VALU
__device__ __forceinline__ unsigned max8(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, false));    // quad_perm 1, 0, 3, 2
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, false));    // quad_perm 2, 3, 0, 1
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, false));  // row_half_mirror
}

template <typename T>
__device__ __forceinline__ void load8(const T* src, float (&v)[8]) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  const vec8 x = *reinterpret_cast<const vec8*>(src);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_f<T>(x[e]);
}

template <typename T>
__device__ __forceinline__ void store8(T* dst, const float (&v)[8]) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  vec8 x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = from_f<T>(v[e]);
  *reinterpret_cast<vec8*>(dst) = x;
}

template <int D>
struct Geo {
  static constexpr int CPT = D / 8;              // 8-channel chunks of a token
  // K, writing: LPR lanes a row, chunks j, j + LPR, ...
  static constexpr int LPR = D == 72 ? 3 : D == 80 ? 2 : 4, CPR = CPT / LPR, RPW = 64 / LPR;   // rows of a wave
  // V: a thread holds 8 tokens x 4 channels
  static constexpr int QUADS = D / 4, THREADS = (QUADS * 8 + 63) / 64 * 64, WAVES = THREADS / 64;
  static constexpr int PITCH = D + 4;            // bytes of a token's row in LDS
  static constexpr int KROWS = WAVES * RPW;      // K rows of a workgroup, writing
  static constexpr int KCH = 4;                  // K chunks of a thread, reading back
};

struct Launch {
  KvCacheParams p;
  int v_blocks;      // workgroups of one (branch, head) on V tiles, first (they take longer); the rest take K
  int vec;           // V^T rows and offsets in whole 16-byte chunks
};

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_quantize_kernel(Launch L) {
  using G = Geo<D>;
  const KvCacheParams& p = L.p;
  const int b = blockIdx.y / p.heads, h = blockIdx.y - b * p.heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t H = (size_t)p.heads * D;
  const T* kv = reinterpret_cast<const T*>(p.kv) + b * p.kv_bs;
  unsigned char* vals = p.c.values + b * p.c.values_bs;
  unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  if ((int)blockIdx.x >= L.v_blocks) {
    const int kb = blockIdx.x - L.v_blocks;
    const int r = lane / G::LPR, j = lane - r * G::LPR, n = kb * G::KROWS + wave * G::RPW + r;
    const bool on = n < p.n && r < G::RPW;
    const T* src = kv + ((size_t)h * p.kv_tokens + p.kv_off + (on ? n : 0)) * D + j * 8;
    float v[G::CPR][8];
    unsigned amax = 0;
#pragma unroll
    for (int i = 0; i < G::CPR; ++i) load8(src + i * G::LPR * 8, v[i]);
#pragma unroll
    for (int i = 0; i < G::CPR; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = max(amax, finite_bits(v[i][e]));
    unsigned all = amax;
#pragma unroll
    for (int k = 1; k < G::LPR; ++k) all = max(all, (unsigned)__shfl((int)amax, r * G::LPR + (j + k) % G::LPR, kWave));
    if (!on) return;
    const unsigned e8 = scale_byte(all);
    const float s = scale_of(e8);
    const size_t row = (size_t)h * p.c.tokens + p.c_off + n;
#pragma unroll
    for (int i = 0; i < G::CPR; ++i) {
      u32x2 w;
      w[0] = to_e4m3(v[i][0], v[i][1], s) | to_e4m3(v[i][2], v[i][3], s) << 16;
      w[1] = to_e4m3(v[i][4], v[i][5], s) | to_e4m3(v[i][6], v[i][7], s) << 16;
      *reinterpret_cast<u32x2*>(vals + row * D + (j + i * G::LPR) * 8) = w;
    }
    if (j == 0) exps[row] = (unsigned char)e8;
    return;
  }
  // V: eight neighbouring lanes hold the same 8 tokens, 4 channels each
  __shared__ unsigned red[G::WAVES][kTile];
  __shared__ __attribute__((aligned(16))) unsigned char tile[kTile * G::PITCH];
  const int n0 = blockIdx.x * kTile;
  const int tg = lane >> 3, quad = wave * 8 + (lane & 7);
  const bool on = quad < G::QUADS;
  const int count = min(max(p.n - n0 - 8 * tg, 0), 8);
  const T* vt = kv + p.kv_tokens * H + ((size_t)h * D + 4 * (on ? quad : 0)) * p.kv_tokens + p.kv_off + n0 + 8 * tg;
  float v[4][8];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (L.vec && count == 8) {
      load8(vt + (size_t)c * p.kv_tokens, v[c]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = e < count ? to_f<T>(vt[(size_t)c * p.kv_tokens + e]) : 0.0f;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const unsigned m = max(max(finite_bits(v[0][e]), finite_bits(v[1][e])), max(finite_bits(v[2][e]), finite_bits(v[3][e])));
    const unsigned all = max8(on ? m : 0u);
    if ((lane & 7) == e) red[wave][8 * tg + e] = all;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = 8 * tg + e;
    unsigned amax = red[0][t];
#pragma unroll
    for (int w = 1; w < G::WAVES; ++w) amax = max(amax, red[w][t]);
    const unsigned e8 = scale_byte(amax);
    const float s = scale_of(e8);
    if (on) *reinterpret_cast<unsigned*>(tile + t * G::PITCH + 4 * quad) = to_e4m3(v[0][e], v[1][e], s) | to_e4m3(v[2][e], v[3][e], s) << 16;
    if (quad == 0 && e < count) exps[(size_t)(p.heads + h) * p.c.tokens + p.c_off + n0 + t] = (unsigned char)e8;
  }
  __syncthreads();
  unsigned char* dst = vals + ((size_t)(p.heads + h) * p.c.tokens + p.c_off + n0) * D;
  const int total = min(kTile, p.n - n0) * G::CPT;
  for (int i = tid; i < total; i += G::THREADS) {
    const unsigned* src = reinterpret_cast<const unsigned*>(tile + i / G::CPT * G::PITCH + i % G::CPT * 8);
    *reinterpret_cast<u32x2*>(dst + (size_t)i * 8) = u32x2{src[0], src[1]};
  }
}

// four values of a word of e4m3 bytes, times s
__device__ __forceinline__ void from_e4m3(unsigned w, float s, float (&v)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false);
  const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_dequantize_kernel(Launch L) {
  using G = Geo<D>;
  const KvCacheParams& p = L.p;
  const int b = blockIdx.y / p.heads, h = blockIdx.y - b * p.heads, tid = threadIdx.x;
  const size_t H = (size_t)p.heads * D;
  T* kv = reinterpret_cast<T*>(p.kv) + b * p.kv_bs;
  const unsigned char* vals = p.c.values + b * p.c.values_bs;
  const unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  if ((int)blockIdx.x >= L.v_blocks) {
    const int kb = blockIdx.x - L.v_blocks;
    // both sides contiguous: chunk after chunk
    const size_t row0 = (size_t)h * p.c.tokens + p.c_off;
    T* dst = kv + ((size_t)h * p.kv_tokens + p.kv_off) * D;
    const int first = kb * G::THREADS * G::KCH, total = p.n * G::CPT;
    u32x2 w[G::KCH];
    float s[G::KCH];
#pragma unroll
    for (int k = 0; k < G::KCH; ++k) {
      const int i = min(first + k * G::THREADS + tid, total - 1);
      w[k] = *reinterpret_cast<const u32x2*>(vals + row0 * D + (size_t)i * 8);
      s[k] = scale_of(exps[row0 + i / G::CPT]);
    }
#pragma unroll
    for (int k = 0; k < G::KCH; ++k) {
      const int i = first + k * G::THREADS + tid;
      float lo[4], hi[4];
      from_e4m3(w[k][0], s[k], lo);
      from_e4m3(w[k][1], s[k], hi);
      if (i < total) store8(dst + (size_t)i * 8, {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
    return;
  }
  __shared__ __attribute__((aligned(16))) unsigned char tile[kTile * G::PITCH];
  const int n0 = blockIdx.x * kTile;
  const int total = min(kTile, p.n - n0) * G::CPT;
  const size_t row0 = (size_t)(p.heads + h) * p.c.tokens + p.c_off + n0;
  const int lane = tid & 63, tg = lane >> 3, quad = (tid >> 6) * 8 + (lane & 7);
  const int count = min(max(p.n - n0 - 8 * tg, 0), 8);
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = scale_of(exps[row0 + (e < count ? 8 * tg + e : 0)]);
  for (int i = tid; i < total; i += G::THREADS) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(vals + row0 * D + (size_t)i * 8);
    unsigned* to = reinterpret_cast<unsigned*>(tile + i / G::CPT * G::PITCH + i % G::CPT * 8);
    to[0] = x[0];
    to[1] = x[1];
  }
  __syncthreads();
  if (count == 0 || quad >= G::QUADS) return;
  float v[4][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // (past the last token: bytes of another workgroup, not stored)
    float x[4];
    from_e4m3(*reinterpret_cast<const unsigned*>(tile + (8 * tg + e) * G::PITCH + 4 * quad), s[e], x);
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c][e] = x[c];
  }
  T* vt = kv + p.kv_tokens * H + ((size_t)h * D + 4 * quad) * p.kv_tokens + p.kv_off + n0 + 8 * tg;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (L.vec && count == 8) {
      store8(vt + (size_t)c * p.kv_tokens, v[c]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < count) vt[(size_t)c * p.kv_tokens + e] = from_f<T>(v[c][e]);
    }
  }
}

template <typename T, int D>
hipError_t launch_d(const KvCacheParams& p, bool back, hipStream_t s) {
  using G = Geo<D>;
  Launch L;
  L.p = p;
  const int k_blocks = back ? ceil_div(p.n * G::CPT, G::THREADS * G::KCH) : ceil_div(p.n, G::KROWS);
  L.v_blocks = ceil_div(p.n, kTile);
  L.vec = p.kv_tokens % 8 == 0 && p.kv_off % 8 == 0;
  const dim3 grid(L.v_blocks + k_blocks, p.heads * p.B), block(G::THREADS);
  if (back) hipLaunchKernelGGL((kv_dequantize_kernel<T, D>), grid, block, 0, s, L);
  else hipLaunchKernelGGL((kv_quantize_kernel<T, D>), grid, block, 0, s, L);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const KvCacheParams& p, bool back, hipStream_t s) {
  if (p.n <= 0) return hipSuccess;
  switch (p.d) {
    case 32: return launch_d<T, 32>(p, back, s);
    case 64: return launch_d<T, 64>(p, back, s);
    case 72: return launch_d<T, 72>(p, back, s);
    case 80: return launch_d<T, 80>(p, back, s);
    case 96: return launch_d<T, 96>(p, back, s);
    case 128: return launch_d<T, 128>(p, back, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv_quantize(const KvCacheParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch<bf16>(p, false, s) : launch<float>(p, false, s);
}

hipError_t launch_kv_dequantize(const KvCacheParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch<bf16>(p, true, s) : launch<float>(p, true, s);
}

}  // namespace orch
