// The pass between two blocks (norm after a block, gate, residual scale, norm
// before the next one, its modulation, optionally to 8-bit codes), and rows to
// 8-bit codes with a scale each.
//
//   h' = a h + g post(y),   u = pre(h') (1 + s) + t
//
// Bytes bound both: every element is read once and written once.  A row stays in
// the registers of the LPR lanes that share it (a part of a wave, a wave, or a
// workgroup), so the statistics are two-pass (mean, then squares about it) at no
// cost in memory.
//
// Measured (kernel times, three sets of inputs in turn, of which the last-level cache keeps a part; a
// large copy runs at 5.1 TB/s), RMS norm, gate, LayerNorm and modulation, no weights, bf16 y and u: 32768 x
// 1152 (453 MB) 85 us, 5.3 TB/s; 3328 x 1152 (46 MB) 11.2 us, 4.1 TB/s; 768 x 1152 5.3 us; into codes 78,
// 11.8 and 5.8; all fp32 32768 x 1152 (604 MB) 106, 3328 x 1152 12.5, 32 x 128 3.1.  With learned weights
// 32768 x 1152 92-95.  The smallest are a launch, one round trip to memory and the reductions' chain.
// Dropped: a load for each channel group behind a branch of its own, at which the compiler waits
// (1.5 times as long at 32768 rows, 1.6 at 3328, 4 at 768); one channel an access where rows lie at any
// address (513 x 1021: 2.8 times as long as the 5.4 us now).
// The quantiser: 3328 x 4608 bf16 (46 MB) 11.2 us, 19452 x 3881 fp32 at odd addresses (378 MB) 66,
// 333 x 1000 fp32 2.9.
#include "common.h"
#include "kernels.h"

namespace orch {
namespace norms {

constexpr int kThreads = 256;
// Workgroups of 1024 threads along x: a grid's threads are counted in 32 bits, so the rows past these go along y.
constexpr int kWideRows = 1 << 21;

// v of the lane that DPP control word C names
template <int C>
__device__ __forceinline__ unsigned dpp(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, C, 0xf, 0xf, true);
}

struct Sum {
  __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }
};
struct Max {
  __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); }
};

// f over the LPR lanes that share a row, the same bits in each: neighbours, quads,
// halves of 16 by DPP, rows of 16 by permlane swaps, waves by LDS
template <int LPR>
struct Group {
  static constexpr int NW = LPR > 64 ? LPR / 64 : 1;
  unsigned* lds;       // [2][NW], LPR > 64
  int turn = 0;

  template <typename F>
  __device__ __forceinline__ unsigned all(unsigned v, F f) {
    v = f(v, dpp<0xB1>(v));    // lane ^ 1
    v = f(v, dpp<0x4E>(v));    // lane ^ 2
    v = f(v, dpp<0x141>(v));   // 7 - lane of 8
    v = f(v, dpp<0x140>(v));   // 15 - lane of 16
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (LPR > 16) {
      const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
      v = f(r[0], r[1]);
    }
    if constexpr (LPR > 32) {
      const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
      v = f(s[0], s[1]);
    }
#endif
    if constexpr (NW > 1) {
      // (two sets of slots: one is read while the next reduction fills the other)
      unsigned* slot = lds + turn * NW;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
      __syncthreads();
      v = slot[0];
#pragma unroll
      for (int w = 1; w < NW; ++w) v = f(v, slot[w]);
    }
    return v;
  }
  __device__ __forceinline__ float sum(float v) { return __uint_as_float(all(__float_as_uint(v), Sum{})); }
  __device__ __forceinline__ unsigned top(unsigned v) { return all(v, Max{}); }
};

// V elements as they are held (anywhere that suits one of them), and as fp32
template <typename T, int V, bool Ragged>
struct Raw {
  typedef T W __attribute__((ext_vector_type(V), aligned(Ragged ? sizeof(T) : V * sizeof(T))));
  W w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const W*>(p); }
  __device__ __forceinline__ float operator[](int e) const { return to_f<T>(w[e]); }
};
template <typename T, bool Ragged>
struct Raw<T, 1, Ragged> {
  T w;
  __device__ __forceinline__ void load(const T* p) { w = *p; }
  __device__ __forceinline__ float operator[](int) const { return to_f<T>(w); }
};

// A lane's share of a row of n >= V channels: V of them from (lane + LPR i) V on, i < NV.  Ragged
// rows end anywhere and lie anywhere: the chunk that would pass the end begins at n - V, and its
// first elements, which are the chunk's before, stay out of everything (a branch for each load
// would wait for each).  Chunks past the row read its first channels.
template <int V, int NV, int LPR, bool Ragged>
struct Share {
  int lane, n;
  __device__ __forceinline__ int nominal(int i) const { return (lane + LPR * i) * V; }
  __device__ __forceinline__ int at(int i) const { return Ragged ? min(nominal(i), n - V) : nominal(i) < n ? nominal(i) : 0; }
  __device__ __forceinline__ bool in(int i, int e) const {
    return nominal(i) < n && (!Ragged || e >= nominal(i) + V - n);
  }
  template <typename T>
  __device__ __forceinline__ void load(Raw<T, V, Ragged> (&r)[NV], const T* row) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) r[i].load(row + at(i));
  }
  // f(i, e) of every element
  template <typename F>
  __device__ __forceinline__ static void each(F f) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) f(i, e);
  }
  // whole(i) for chunks within the row, one(i, e) for what a last shorter one holds
  template <typename F, typename G>
  __device__ __forceinline__ void put(F whole, G one) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (Ragged ? nominal(i) + V <= n : nominal(i) < n) {
        whole(i);
      } else if (Ragged && nominal(i) < n) {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (in(i, e)) one(i, e);
      }
    }
  }
};

template <typename T, int V, bool Ragged>
__device__ __forceinline__ void store(T* p, const float* x) {
  typedef T W __attribute__((ext_vector_type(V), aligned(Ragged ? sizeof(T) : V * sizeof(T))));
  if constexpr (V == 1) {
    *p = from_f<T>(x[0]);
  } else {
    W w;
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = from_f<T>(x[e]);
    *reinterpret_cast<W*>(p) = w;
  }
}

// A row's codes: q = x * (127 / top) to nearest, ties to even, quotient and product
// rounded to 32 bits; scale top / 127.  `bits`: the largest magnitude's.  Below 2^-64
// the quotient is taken of 2^64 x, which is exact, so that it stays finite.
// An infinity or NaN anywhere: codes 0 and scale NaN, so every product of the row is NaN.
struct Codes {
  float up, r, scale;
  __device__ __forceinline__ explicit Codes(unsigned bits) {
    const float top = __uint_as_float(bits);
    up = bits < 0x1F800000u ? 0x1p64f : 1.0f;
    r = bits == 0u || bits >= 0x7F800000u ? 0.0f : 127.0f / (top * up);
    scale = bits >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : top / 127.0f;
    finite = bits < 0x7F800000u;
  }
  bool finite;
  __device__ __forceinline__ int code(float x) const { return finite ? (int)rintf((x * up) * r) : 0; }
  template <int V>
  __device__ __forceinline__ void put(signed char* p, const float* x) const {
    if constexpr (V == 1) {
      *p = (signed char)code(x[0]);
    } else {
      unsigned w[V / 4];
#pragma unroll
      for (int i = 0; i < V / 4; ++i)
        w[i] = (code(x[4 * i]) & 0xff) | (code(x[4 * i + 1]) & 0xff) << 8 | (code(x[4 * i + 2]) & 0xff) << 16 |
               (unsigned)code(x[4 * i + 3]) << 24;
      if constexpr (V == 4) *reinterpret_cast<unsigned*>(p) = w[0];
      else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    }
  }
};

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// x of a row -> its norm times weight plus bias (32 bits); what is not in the share
// comes in as 0 and stays out of the sums
template <int V, int NV, int LPR, bool Ragged>
__device__ __forceinline__ void norm(float (&x)[NV][V], const Share<V, NV, LPR, Ragged>& sh, const Norm& n, Group<LPR>& g) {
  using S = Share<V, NV, LPR, Ragged>;
  if (n.kind != kNormNone) {
    const float inv = 1.0f / (float)sh.n;
    if (n.kind == kNormLayer) {
      float s = 0.0f;
      S::each([&](int i, int e) __attribute__((always_inline)) { s += x[i][e]; });
      const float mean = g.sum(s) * inv;
      S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] = sh.in(i, e) ? x[i][e] - mean : 0.0f; });
    }
    float s = 0.0f;
    S::each([&](int i, int e) __attribute__((always_inline)) { s = fmaf(x[i][e], x[i][e], s); });
    const float rstd = 1.0f / sqrtf(g.sum(s) * inv + n.eps);
    S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] *= rstd; });
  }
  if (n.weight) {
    Raw<float, V, Ragged> w[NV];
    sh.load(w, n.weight);
    S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] *= w[i][e]; });
  }
  if (n.bias) {
    Raw<float, V, Ragged> w[NV];
    sh.load(w, n.bias);
    S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] += w[i][e]; });
  }
}

template <typename T, int V, int LPR, int NV, bool Ragged>
__global__ __launch_bounds__(LPR > kThreads ? LPR : kThreads) void block_norms_kernel(BlockNormsParams p) {
  constexpr int RPB = LPR > kThreads ? 1 : kThreads / LPR;    // rows of a workgroup
  using S = Share<V, NV, LPR, Ragged>;
  __shared__ unsigned red[LPR > 64 ? 2 * LPR / 64 : 1];
  const int row = (LPR > kThreads ? blockIdx.y * kWideRows + blockIdx.x : blockIdx.x * RPB) + threadIdx.x / LPR;
  if (row >= p.rows) return;    // (the whole group of lanes; a group of several waves is a whole workgroup)
  const S sh{(int)(threadIdx.x % LPR), p.hidden};
  Group<LPR> g{red};
  const size_t b = row / p.rows_per_batch * p.mod_stride;
  // every load first, as far as the registers hold them
  constexpr bool EARLY = NV * V <= 24;
  Raw<float, V, Ragged> h[NV], gate[NV], shift[NV], scale[NV];
  Raw<T, V, Ragged> y[NV];
  if (EARLY || !p.y) sh.load(h, p.h + row * p.h_stride);
  if (p.y) sh.load(y, reinterpret_cast<const T*>(p.y) + row * p.y_stride);
  if (EARLY && p.gate) sh.load(gate, p.gate + b);
  if (EARLY && p.scale) sh.load(scale, p.scale + b);
  if (EARLY && p.shift) sh.load(shift, p.shift + b);
  float x[NV][V];
  if (p.y) {
    float z[NV][V];
    S::each([&](int i, int e) __attribute__((always_inline)) { z[i][e] = sh.in(i, e) ? y[i][e] : 0.0f; });
    norm<V, NV, LPR, Ragged>(z, sh, p.post, g);
    if (!EARLY && p.gate) sh.load(gate, p.gate + b);
    if (p.gate) S::each([&](int i, int e) __attribute__((always_inline)) { z[i][e] *= gate[i][e]; });
    if (!EARLY) sh.load(h, p.h + row * p.h_stride);
    S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] = fmaf(p.residual_scale, h[i][e], z[i][e]); });
  } else {
    S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] = p.residual_scale * h[i][e]; });
  }
  if (p.h_out) {
    float* o = p.h_out + row * p.h_out_stride;
    sh.put([&](int i) __attribute__((always_inline)) { store<float, V, Ragged>(o + sh.at(i), x[i]); },
           [&](int i, int e) __attribute__((always_inline)) { o[sh.at(i) + e] = x[i][e]; });
  }
  if (!p.out && !p.codes) return;
  S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] = sh.in(i, e) ? x[i][e] : 0.0f; });
  norm<V, NV, LPR, Ragged>(x, sh, p.pre, g);
  if (!EARLY && p.scale) sh.load(scale, p.scale + b);
  if (p.scale) S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] *= 1.0f + scale[i][e]; });
  if (!EARLY && p.shift) sh.load(shift, p.shift + b);
  if (p.shift) S::each([&](int i, int e) __attribute__((always_inline)) { x[i][e] += shift[i][e]; });
  if (p.out) {
    T* o = reinterpret_cast<T*>(p.out) + row * p.out_stride;
    sh.put([&](int i) __attribute__((always_inline)) { store<T, V, Ragged>(o + sh.at(i), x[i]); },
           [&](int i, int e) __attribute__((always_inline)) { o[sh.at(i) + e] = from_f<T>(x[i][e]); });
  }
  if (!p.codes) return;
  unsigned top = 0;
  S::each([&](int i, int e) __attribute__((always_inline)) { top = max(top, sh.in(i, e) ? magnitude(x[i][e]) : 0u); });
  const Codes q(g.top(top));
  signed char* o = p.codes + row * p.codes_stride;
  sh.put([&](int i) __attribute__((always_inline)) { q.put<V>(o + sh.at(i), x[i]); },
         [&](int i, int e) __attribute__((always_inline)) { o[sh.at(i) + e] = (signed char)q.code(x[i][e]); });
  if (sh.lane == 0) p.code_scales[row] = q.scale;
}

// Rows to codes.  NV 0: rows too long for the registers, read twice.
template <typename T, int V, int LPR, int NV, bool Ragged>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const T* __restrict__ x, size_t x_stride, int rows, int cols,
                                                                 signed char* __restrict__ codes, size_t codes_stride,
                                                                 float* __restrict__ scales) {
  __shared__ unsigned red[LPR > 64 ? 2 * LPR / 64 : 1];
  const int lane = threadIdx.x % LPR;
  const int row = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= rows) return;
  Group<LPR> g{red};
  const T* xr = x + row * x_stride;
  signed char* cr = codes + row * codes_stride;
  // (repeated elements do not change the largest)
  constexpr int C = NV > 0 ? NV : 4;
  using S = Share<V, C, LPR, Ragged>;
  unsigned top = 0;
  auto largest = [&](Raw<T, V, Ragged> (&v)[C], const S& sh) __attribute__((always_inline)) {
    sh.load(v, xr);
    S::each([&](int i, int e) __attribute__((always_inline)) { top = max(top, magnitude(v[i][e])); });
  };
  auto write = [&](Raw<T, V, Ragged> (&v)[C], const S& sh, const Codes& q) __attribute__((always_inline)) {
    sh.put(
        [&](int i) __attribute__((always_inline)) {
          float f[V];
#pragma unroll
          for (int e = 0; e < V; ++e) f[e] = v[i][e];
          q.put<V>(cr + sh.at(i), f);
        },
        [&](int i, int e) __attribute__((always_inline)) { cr[sh.at(i) + e] = (signed char)q.code(v[i][e]); });
  };
  Raw<T, V, Ragged> v[C];
  if constexpr (NV > 0) {
    const S sh{lane, cols};
    largest(v, sh);
    const Codes q(g.top(top));
    write(v, sh, q);
    if (lane == 0) scales[row] = q.scale;
  } else {
    for (int l = lane; l * V < cols; l += LPR * C) largest(v, S{l, cols});
    const Codes q(g.top(top));
    for (int l = lane; l * V < cols; l += LPR * C) {
      const S sh{l, cols};
      sh.load(v, xr);
      write(v, sh, q);
    }
    if (lane == 0) scales[row] = q.scale;
  }
}

static bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

template <typename T, int V, int LPR, int NV, bool Ragged>
static void launch_norms(const BlockNormsParams& p, hipStream_t s) {
  constexpr int threads = LPR > kThreads ? LPR : kThreads;
  const int groups = ceil_div(p.rows, threads / LPR);
  const dim3 grid = LPR > kThreads && groups > kWideRows ? dim3(kWideRows, ceil_div(groups, kWideRows)) : dim3(groups);
  hipLaunchKernelGGL((block_norms_kernel<T, V, LPR, NV, Ragged>), grid, dim3(threads), 0, s, p);
}

// As few lanes a row as keep to 20 channels each: more channels cost registers, and with them rows in
// flight, and lengthen the chain of a lone row; more lanes share out less (1152 channels in 64 lanes, in 32
// of 36 channels and in 256, no weights, bf16: 768 rows 5.4, 6.5 and 5.7 us, 3328 rows 11.4, 11.0 and
// 11.9, 32768 rows 85, 86 and 95).
template <typename T, bool Ragged>
static void launch_norms_width(const BlockNormsParams& p, hipStream_t s) {
  const int H = p.hidden;
  if (H <= 16 * 4 * 2) launch_norms<T, 4, 16, 2, Ragged>(p, s);
  else if (H <= 32 * 4 * 3) launch_norms<T, 4, 32, 3, Ragged>(p, s);
  else if (H <= 64 * 4 * 5) launch_norms<T, 4, 64, 5, Ragged>(p, s);
  else if (H <= 256 * 4 * 2) launch_norms<T, 4, 256, 2, Ragged>(p, s);
  else if (H <= 256 * 4 * 5) launch_norms<T, 4, 256, 5, Ragged>(p, s);
  else launch_norms<T, 4, 1024, 8, Ragged>(p, s);
}

template <typename T>
static void launch_norms_t(const BlockNormsParams& p, hipStream_t s) {
  bool even = p.hidden % 4 == 0 && p.mod_stride % 4 == 0;
  for (const void* q : {(const void*)p.gate, (const void*)p.shift, (const void*)p.scale, (const void*)p.post.weight,
                        (const void*)p.post.bias, (const void*)p.pre.weight, (const void*)p.pre.bias,
                        (const void*)p.h, (const void*)p.h_out})
    even = even && aligned(q, 16);
  even = even && aligned(p.y, 4 * sizeof(T)) && aligned(p.out, 4 * sizeof(T)) && p.h_stride % 4 == 0 &&
         p.h_out_stride % 4 == 0 && p.y_stride % 4 == 0 && p.out_stride % 4 == 0;
  if (p.hidden < 4) launch_norms<T, 1, 16, 1, false>(p, s);
  else if (even) launch_norms_width<T, false>(p, s);
  else launch_norms_width<T, true>(p, s);
}

template <typename T, int V, int LPR, int NV, bool Ragged>
static void launch_quant(const QuantizeRowsParams& p, hipStream_t s) {
  hipLaunchKernelGGL((quantize_rows_kernel<T, V, LPR, NV, Ragged>), dim3(ceil_div(p.rows, kThreads / LPR)), dim3(kThreads), 0, s,
                     reinterpret_cast<const T*>(p.x), p.x_stride, p.rows, p.cols, p.codes, p.codes_stride, p.scales);
}

template <typename T, bool Ragged>
static void launch_quant_width(const QuantizeRowsParams& p, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  if (p.cols <= 16 * V * 2) launch_quant<T, V, 16, 2, Ragged>(p, s);
  else if (p.cols <= 32 * V * 5) launch_quant<T, V, 32, 5, Ragged>(p, s);
  else if (p.cols <= 64 * V * 9) launch_quant<T, V, 64, 9, Ragged>(p, s);
  else if (p.cols <= 256 * V * 9) launch_quant<T, V, 256, 9, Ragged>(p, s);
  else launch_quant<T, V, 256, 0, Ragged>(p, s);
}

template <typename T>
static void launch_quant_t(const QuantizeRowsParams& p, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  if (p.cols < V) launch_quant<T, 1, 16, 1, false>(p, s);
  else if (p.cols % V == 0 && aligned(p.x, 16) && p.x_stride % V == 0) launch_quant_width<T, false>(p, s);
  else launch_quant_width<T, true>(p, s);
}

}  // namespace norms

hipError_t launch_block_norms(const BlockNormsParams& p, int dtype, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  if (dtype == kBF16) norms::launch_norms_t<bf16>(p, s);
  else norms::launch_norms_t<float>(p, s);
  return hipGetLastError();
}

hipError_t launch_quantize_rows(const QuantizeRowsParams& p, int dtype, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  if (dtype == kBF16) norms::launch_quant_t<bf16>(p, s);
  else norms::launch_quant_t<float>(p, s);
  return hipGetLastError();
}

}  // namespace orch
