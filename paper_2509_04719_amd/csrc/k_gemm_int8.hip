// Projections in 8-bit integers: y = (sum_k a[m][k] w[n][k]) sa[m] sw[n] + bias[n],
// with the epilogues of the other projections (plain store, GELU, gated residual,
// QKV scatter).  Sums are exact (int32), so no output depends on how k is split.
//
// Operands are int8 rows, k next to k; v_mfma_i32_32x32x32_i8 takes 16 bytes a lane
// of each, as the bf16 MFMA of half the k does, in the same time: the loops are those
// of the bf16 products counted in bytes.  Rows go straight to LDS 16 bytes a lane,
// 16-byte chunks XOR-swizzled by row.
//
// Any M, N and K: rows past M and N re-read the last one and are not stored; the
// bytes past K of the last k-tile are cleared in A's fragments (what W's hold
// there does not matter then: integers have no NaN).
//
// Measured (kernel times, median of 60 over three sets of inputs in turn, codes of normal deviates of
// uneven channels; the large ones move by 10% with the clock, which falls under their load; a large library
// product of int8 runs at 2110-2160 TOP/s, a large copy at 5.1 TB/s), us (TOP/s):
//   8192 x 8192 -> 8192    plain, bf16, uniform codes   475-520  (2120-2310)
//   32768 x 1152 -> 4608   plain, bf16   206-229  (1520-1690)     plain, fp32   263  (1320)
//                          GELU, bf16    230-257  (1350-1510)     GELU, fp32    305  (1140)
//   32768 x 4608 -> 1152   residual      241  (1440)
//   32205 x 2176 -> 1280   residual      157  (1140)
//   12288 x 1152 -> 3456   QKV, bf16     71  (1380)               QKV, fp32     105  (930)
//   12288 x 1152 -> 1152   residual      35-39  (840-930)
//   3328 x 1152 -> 3456    plain, bf16   19.9  (1330)    QKV, bf16   22.2  (1190)    QKV, fp32   29  (910)
//   3328 x 1152 -> 4608    GELU, bf16    28.0  (1260)
//   3328 x 4608 -> 1152    residual      25.8  (1370)
//   3328 x 1152 -> 1152    residual      14  (630)
//   768 x 1152 -> 4608     GELU, bf16    10.3  (790)
//   768 x 4608 -> 1152     residual      11.4  (710)
//   1 x 1152 -> 4608, GELU 5.0; 1 x 4608 -> 1152, residual 8.1; 96 x 384 -> 1152, QKV 4.6
// With K = 1152 a tile's products take 18400 cycles of the matrix cores and its outputs (scales, GELU,
// rounding) 19600 of the vector units, one after the other in the large tiles; smaller tiles, of which a
// CU holds two, overlap the two but pull more bytes from L2 than it gives (54 B per ns and CU).
#include <cmath>
#include <cstdlib>

#include "common.h"
#include "kernels.h"

namespace orch {
namespace i8 {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// GELU, tanh form: y / (1 + e^(-2u)), u = sqrt(2/pi) (y + 0.044715 y^3); where the
// result is rounded to bf16 on the fast reciprocal (2^-22 off)
template <typename T>
__device__ __forceinline__ float gelu(float y) {
  constexpr float c0 = -2.0f * 0.7978845608028654f * 1.4426950408889634f, c1 = c0 * 0.044715f;
  const float e = __builtin_amdgcn_exp2f(y * fmaf(c1, y * y, c0));
  return sizeof(T) == 2 ? y * __builtin_amdgcn_rcpf(1.0f + e) : y / (1.0f + e);
}

// m / rows_per_batch: a product with the rounded-up inverse, exact below 2^31
__device__ __forceinline__ int branch(const GemmI8Params& p, int m) {
  return (int)(((unsigned long long)(unsigned)m * p.rpb_inverse) >> p.rpb_shift);
}

// What a tile's epilogue reads beside its sums, in LDS: scales of its rows, scales
// and biases of its columns.
template <int BM, int BN>
struct Side {
  float sa[BM], sw[BN], bias[BN];
  struct Regs { float a, w, b; };
  // (loads first, LDS writes behind the prologue's other loads; at least 256 threads)
  __device__ __forceinline__ static void fetch(Regs& r, const GemmI8Params& p, int m0, int n0) {
    const int t = threadIdx.x;
    r.a = t < BM && m0 + t < p.M ? p.sa[m0 + t] : 0.0f;
    r.w = t < BN && n0 + t < p.N ? p.sw[n0 + t] : 0.0f;
    r.b = t < BN && n0 + t < p.N && p.bias ? p.bias[n0 + t] : 0.0f;
  }
  __device__ __forceinline__ void keep(const Regs& r) {
    const int t = threadIdx.x;
    if (t < BM) sa[t] = r.a;
    if (t < BN) sw[t] = r.w, bias[t] = r.b;
  }
  static_assert(BM <= 256 && BN <= 256, "one value a thread");
};

// The epilogue of a 32 x 32 block of sums from (m, n) on, straight from the registers.
// The MFMAs make transposed blocks: lane (lr, h) = (lane % 32, lane / 32) holds row lr,
// columns 8 g + 4 h + r.  In bf16 the halves h swap registers, so that a lane holds columns 16 h
// .. 16 h + 15 and every store is 16 bytes.  V^T wants tokens next to each other: its
// blocks (`Vt`) are made the other way round, so that a lane holds column lr and tokens 8 g + 4 h
// + r.
template <typename T, int EPI, bool Vt>
struct Block {
  const GemmI8Params& p;
  int lr, h;

  // columns' (Vt: the column's) scales and biases, and rows' scales, of the lane
  struct Cols { f32x4 w[Vt ? 1 : 4], b[Vt ? 1 : 4]; };
  __device__ __forceinline__ void cols(Cols& c, const float* sw, const float* bias) const {
    if constexpr (Vt) {
      c.w[0][0] = sw[lr];
      c.b[0][0] = bias[lr];
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        c.w[g] = *reinterpret_cast<const f32x4*>(sw + 8 * g + 4 * h);
        c.b[g] = *reinterpret_cast<const f32x4*>(bias + 8 * g + 4 * h);
      }
    }
  }

  // four bf16 as two words
  __device__ __forceinline__ static uint2 pack(const float* y) {
    const bf16x4 v = {(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    return __builtin_bit_cast(uint2, v);
  }
  // 16 bytes with what the other half holds of groups g (kept by h = 0) and g + 2 (by h = 1)
  __device__ __forceinline__ static uint4 join(uint2 x, uint2 y) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto a = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
    return make_uint4(a[0], b[0], a[1], b[1]);
#else
    return make_uint4(x.x, x.y, y.x, y.y);
#endif
  }

  // where (row m, column n) of Q, K or V^T lies
  __device__ __forceinline__ T* at(int b, int tok, int n) const {
    const int hidden = p.hidden, which = n >= 2 * hidden ? 2 : n >= hidden ? 1 : 0, nn = n - which * hidden;
    const int head = (int)__umulhi((unsigned)nn, p.hd_magic), dd = nn - head * p.head_dim;
    T* kv = reinterpret_cast<T*>(p.kv) + b * p.kv_bs;
    const size_t ntot = (size_t)p.kv_tokens, t = (size_t)(p.tok_offset + tok);
    if (which == 0) return reinterpret_cast<T*>(p.q) + (((size_t)b * p.heads + head) * p.rows_per_batch + tok) * p.head_dim + dd;
    if (which == 1) return kv + ((size_t)head * ntot + t) * p.head_dim + dd;
    return kv + ntot * hidden + ((size_t)head * p.head_dim + dd) * ntot + t;
  }

  // outputs of a block, before a gated residual
  __device__ __forceinline__ void values(float (&y)[4][4], const i32x16& acc, const Cols& c, const float* sa) const {
    const float own = Vt ? 0.0f : sa[lr];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 a;
      if constexpr (Vt) a = *reinterpret_cast<const f32x4*>(sa + 8 * g + 4 * h);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        y[g][r] = Vt ? fmaf((float)acc[4 * g + r] * a[r], c.w[0][0], c.b[0][0])
                     : fmaf((float)acc[4 * g + r] * own, c.w[Vt ? 0 : g][r], c.b[Vt ? 0 : g][r]);
        if (EPI == kEpiGelu) y[g][r] = gelu<T>(y[g][r]);
      }
    }
  }

  // what the residual stream and the gate hold at (m, n)
  struct Stream { f32x4 h, g; };
  __device__ __forceinline__ void fetch(Stream& s, int m, int n) const {
    if (EPI == kEpiResidual && m < p.M && n < p.N) {
      s.h = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p.out) + (size_t)m * p.N + n);
      s.g = *reinterpret_cast<const f32x4*>(p.gate + branch(p, m) * p.gate_stride + n);
    }
  }

  // 16 bytes of outputs from (m, n) on: channels (Vt: tokens) next to each other.  Rows of
  // `out` take 16-byte accesses (p.wide).  held: the same in LDS, where they are.
  __device__ __forceinline__ void sink(const uint4& v, const char* held, int m, int n, const Stream& was) const {
    constexpr int CE = 16 / sizeof(T);
    if (m >= p.M || n >= p.N) return;
    if constexpr (EPI == kEpiResidual) {
      const f32x4 y = __builtin_bit_cast(f32x4, v);
      f32x4 o;
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = fmaf(was.g[r], y[r], was.h[r]);
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p.out) + (size_t)m * p.N + n) = o;
    } else if constexpr (EPI == kEpiQkv) {
      const int b = branch(p, m), tok = m - b * p.rows_per_batch;
      T* d = at(b, tok, n);
      // whole: the 16 bytes lie next to each other (not so at a branch's end, or for V^T's columns
      // beside K's in one wave's blocks); V^T's at any token
      if (Vt ? m + CE <= p.M && tok + CE <= p.rows_per_batch : n < 2 * p.hidden) {
        typedef T Any __attribute__((ext_vector_type(CE), aligned(sizeof(T))));
        if constexpr (Vt) *reinterpret_cast<Any*>(d) = __builtin_bit_cast(Any, v);
        else *reinterpret_cast<uint4*>(d) = v;
      } else if (held) {
#pragma unroll 1
        for (int f = 0; f < CE; ++f) one(held_one(held, f), Vt ? m + f : m, Vt ? n : n + f);
      } else {
        typedef T W __attribute__((ext_vector_type(CE)));
        const W w = __builtin_bit_cast(W, v);
#pragma unroll
        for (int f = 0; f < CE; ++f) one(w[f], Vt ? m + f : m, Vt ? n : n + f);
      }
    } else {
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.out) + (size_t)m * p.N + n) = v;
    }
  }
  // element i of what is held in LDS (written there as 16-byte words)
  __device__ __forceinline__ static T held_one(const char* p, int i) {
    T x;
    __builtin_memcpy(&x, p + i * (int)sizeof(T), sizeof(T));
    return x;
  }
  // one output where rows of out take no 16-byte accesses
  __device__ __forceinline__ void element(T x, int m, int n) const {
    if (m >= p.M || n >= p.N) return;
    T* d = reinterpret_cast<T*>(p.out) + (size_t)m * p.N + n;
    if constexpr (EPI == kEpiResidual) *d = fmaf(p.gate[branch(p, m) * p.gate_stride + n], x, *d);
    else *d = x;
  }
  __device__ __forceinline__ void one(T x, int m, int n) const {
    const int b = branch(p, m);
    if (m < p.M && n < p.N) *at(b, m - b * p.rows_per_batch, n) = x;
  }

  // a block straight from the registers
  __device__ __forceinline__ void run(const i32x16& acc, const Cols& c, const float* sa, int m0, int n0, int split) const {
    if constexpr (EPI == kEpiPartial) {
      const int m = m0 + lr;
      int* d = p.ws + ((size_t)split * p.M + m) * p.N + n0;
      if (m < p.M) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int n = 8 * g + 4 * h;
          if (p.N % 4 == 0) {
            if (n0 + n < p.N)
              *reinterpret_cast<i32x4*>(d + n) = i32x4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (n0 + n + r < p.N) d[n + r] = acc[4 * g + r];
          }
        }
      }
    } else {
      float y[4][4];
      Stream was[4];
      if (p.wide)
#pragma unroll
        for (int g = 0; g < 4; ++g) fetch(was[g], m0 + lr, n0 + 8 * g + 4 * h);
      values(y, acc, c, sa);
      if (EPI != kEpiQkv && !p.wide) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) element(from_f<T>(y[g][r]), m0 + lr, n0 + 8 * g + 4 * h + r);
      } else if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint4 v = join(pack(y[e]), pack(y[e + 2]));
          const int x = 16 * h + 8 * e;
          if constexpr (Vt) sink(v, nullptr, m0 + x, n0 + lr, Stream{});
          else sink(v, nullptr, m0 + lr, n0 + x, Stream{});
        }
      } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const uint4 v = __builtin_bit_cast(uint4, f32x4{y[g][0], y[g][1], y[g][2], y[g][3]});
          const int x = 8 * g + 4 * h;
          if constexpr (Vt) sink(v, nullptr, m0 + x, n0 + lr, was[g]);
          else sink(v, nullptr, m0 + lr, n0 + x, was[g]);
        }
      }
    }
  }
};

// A wave's sums, FM x FN blocks from (m, n) on, whose rows' scales are at sa, columns'
// at sw and bias.
template <typename T, int EPI, bool Vt, int FM, int FN>
__device__ __forceinline__ void direct(const GemmI8Params& p, const i32x16 (&acc)[FM][FN], const float* sa, const float* sw,
                                       const float* bias, int lane, int m, int n, int split) {
  using B = Block<T, EPI, Vt>;
  const B blk{p, lane & 31, lane >> 5};
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    if (n + 32 * j >= p.N) break;
    typename B::Cols c;
    if constexpr (EPI != kEpiPartial) blk.cols(c, sw + 32 * j, bias + 32 * j);
#pragma unroll
    for (int i = 0; i < FM; ++i)
      if (m + 32 * i < p.M) blk.run(acc[i][j], c, sa + 32 * i, m + 32 * i, n + 32 * j, split);
  }
}

// The same by way of LDS, so that a store instruction writes whole 128-byte lines (eight
// rows of 64 bf16 or 32 fp32) and addresses are formed for one line at a time.  Stores straight from
// the registers write 32 bytes of 32 rows: 256 x 256 tiles spill (6 to 600 registers), 192 x 256 ones take,
// plain, bf16, 250 us for 235-244 at 32768 x 1152 -> 4608, 91.5 for 90 at 12288 rows, 19.1 for 19.9 where there is
// one round of tiles (3328 x 1152 -> 3456).  16 rows at a time in an area of the
// wave's own; rows 144 bytes apart spread over the banks.
constexpr int kLine = 144, kArea = 16 * kLine;

// What the lanes of the wave wrote to LDS before is what they read behind it.  (LDS takes a
// wave's accesses in order, so this is no instruction; but it keeps the compiler from sending
// lanes that write and lanes that do not through copies of the code one after the other.)
__device__ __forceinline__ void wave_sync() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#endif
}

template <typename T, int EPI, bool Vt, int FM, int FN>
__device__ __forceinline__ void staged(const GemmI8Params& p, const i32x16 (&acc)[FM][FN], char* area, const float* sa,
                                       const float* sw, const float* bias, int lane, int m, int n) {
  using B = Block<T, EPI, Vt>;
  const B blk{p, lane & 31, lane >> 5};
  const int lr = blk.lr, h = blk.h;
  // blocks side by side along the stored rows: two in bf16, one in fp32
  constexpr int SB = sizeof(T) == 2 ? 2 : 1, CE = 16 / sizeof(T);
  constexpr int O = Vt ? FN : FM, I = Vt ? FM : FN;       // blocks across and along the stored rows
#pragma unroll
  for (int i0 = 0; i0 < I; i0 += SB) {
    const int along = (Vt ? m : n) + 32 * i0;
    if (along >= (Vt ? p.M : p.N)) break;
    typename B::Cols c[Vt ? 1 : SB];
    if constexpr (!Vt) {
#pragma unroll
      for (int k = 0; k < SB; ++k)
        if (i0 + k < I) blk.cols(c[k], sw + 32 * (i0 + k), bias + 32 * (i0 + k));
    }
#pragma unroll
    for (int o = 0; o < O; ++o) {
      if ((Vt ? n : m) + 32 * o >= (Vt ? p.N : p.M)) break;
      if constexpr (Vt) blk.cols(c[0], sw + 32 * o, bias + 32 * o);
      // (this turn's addresses from this turn's copy: hoisted ones would not fit the registers)
      int at = lane;
      asm volatile("" : "+v"(at));
      const int nb = i0 + SB <= I ? SB : 1, ch8 = sizeof(T) == 2 ? 4 * nb : 8;    // (a last block of its own: half lines)
      typename B::Stream was[2][2];
      if (EPI == kEpiResidual && p.wide) {
#pragma unroll
        for (int x = 0; x < 4; ++x) blk.fetch(was[x >> 1][x & 1], m + 32 * o + 8 * x + at / 8, along + CE * (at % 8));
      }
      uint4 v[4];     // chunk 4 k + 2 h + e of block k in bf16, 2 g + h in fp32
#pragma unroll
      for (int k = 0; k < nb; ++k) {
        float y[4][4];
        if constexpr (Vt) blk.values(y, acc[i0 + k][o], c[0], sa + 32 * (i0 + k));
        else blk.values(y, acc[o][i0 + k], c[Vt ? 0 : k], sa + 32 * o);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < 2; ++e) v[2 * k + e] = B::join(B::pack(y[e]), B::pack(y[e + 2]));
        } else {
#pragma unroll
          for (int g = 0; g < 4; ++g) v[g] = __builtin_bit_cast(uint4, f32x4{y[g][0], y[g][1], y[g][2], y[g][3]});
        }
      }
#pragma unroll
      for (int pass = 0; pass < 2; ++pass) {
        wave_sync();
        if ((lr >> 4) == pass) {
#pragma unroll
          for (int x = 0; x < ch8 / 2; ++x)
            *reinterpret_cast<uint4*>(area + (lr & 15) * kLine +
                                      (sizeof(T) == 2 ? 4 * (x >> 1) + 2 * h + (x & 1) : 2 * x + h) * 16) = v[x];
        }
        wave_sync();
        const int across = (Vt ? n : m) + 32 * o + 16 * pass;
        if (EPI == kEpiQkv || p.wide) {
#pragma unroll
          for (int q = 0; q < ch8 / 4; ++q) {
            const int row = q * 8 + at / ch8, ch = at % ch8;
            const char* held = area + row * kLine + ch * 16;
            const uint4 w = *reinterpret_cast<const uint4*>(held);
            if constexpr (Vt) blk.sink(w, held, along + CE * ch, across + row, was[pass][q]);
            else blk.sink(w, held, across + row, along + CE * ch, was[pass][q]);
          }
        } else {        // (rows of out that 16 bytes do not fit: an element a lane)
          const int per = ch8 * CE;
#pragma unroll 2
          for (int q = 0; q < per / 4; ++q) {
            const int row = q * (64 / per) + at / per, c = at % per;
            blk.element(B::held_one(area + row * kLine, c), across + row, along + c);
          }
        }
      }
    }
  }
}

// Whether a wave's blocks from column n on are V^T's alone, and so made the other way round
template <int EPI>
__device__ __forceinline__ bool all_vt(const GemmI8Params& p, int n) {
  return EPI == kEpiQkv && n >= 2 * p.hidden;
}
template <bool Vt>
__device__ __forceinline__ i32x16 mfma(const i32x4& a, const i32x4& w, const i32x16& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (Vt) return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, w, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_i32_32x32x32_i8(w, a, c, 0, 0, 0);
#else
  return c;
#endif
}

// Which tile workgroup `pid` takes: XCD-major, then groups of GROUP tile rows, column-major
// inside.
template <int GROUP>
struct TileAt {
  int m, n;
  __device__ __forceinline__ TileAt(int tiles_m, int tiles_n, int pid) {
    const int per = tiles_m * tiles_n / 8;
    if (pid < per * 8) pid = (pid & 7) * per + (pid >> 3);
    const int gid = pid / (GROUP * tiles_n);
    const int first_m = gid * GROUP;
    const int gsz = min(tiles_m - first_m, GROUP);
    m = first_m + (pid % (GROUP * tiles_n)) % gsz;
    n = (pid % (GROUP * tiles_n)) / gsz;
  }
};

// all ones where byte 16 c + i of a k-tile with `left` bytes of k lies within them
__device__ __forceinline__ i32x4 within(int left, int c) {
  i32x4 m;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int n = left - 16 * c - 4 * d;
    m[d] = n >= 4 ? -1 : n <= 0 ? 0 : (int)((1u << (8 * n)) - 1u);
  }
  return m;
}

#if defined(__HIP_DEVICE_COMPILE__)
// `rows` rows of `base` from row r0 on (at most `most` are addressed): K bytes of
// each, the last one's to a multiple of 16, so that no load leaves the matrix
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const signed char* base, size_t ld, int r0, int rows, int most, int K) {
  const int n = min(rows - r0, most);
  return buffer_rsrc(base + r0 * ld, (size_t)(n - 1) * ld + (size_t)((K + 15) & ~15));
}
#endif

// ---------------------------------------------------------------------------
// BM x BN tile over WM x WN waves, k-tiles of 128 bytes in a ring of S stages: one barrier a
// k-tile; the loads of tile kt + S - 1 lie between the MFMAs of tile kt.
template <int BM, int BN, int WM, int WN, int S>
struct Geo {
  static constexpr int BK = 128, NW = WM * WN;
  static constexpr int TM = BM / WM, TN = BN / WN;  // wave tile
  static constexpr int FM = TM / 32, FN = TN / 32;  // 32x32 blocks per wave
  static constexpr int IA = BM / (8 * NW), LPT = IA + BN / (8 * NW);  // loads of A's rows, of all, per lane and k-tile
  static constexpr int STAGE = (BM + BN) * BK;
  static constexpr int KK = BK / 32;                // MFMA k-steps per k-tile
  static constexpr int LPK = S == 2 ? LPT : (LPT + KK - 1) / KK;
  static constexpr int RING = S * STAGE;
  static constexpr int LDS = RING + (int)sizeof(Side<BM, BN>);
  static_assert(NW >= 4 && TM % 32 == 0 && TN % 32 == 0, "wave tile");
  static_assert(BM % (NW * 8) == 0 && BN % (NW * 8) == 0, "rows per wave");
  static_assert(S >= 2 && LPT * (S - 1) < 60 && NW * kArea <= RING && LDS <= 160 * 1024, "LDS");
};

template <int BM, int BN, int WM, int WN, int S, int WPE, typename T, int EPI>
__global__ __launch_bounds__(64 * WM * WN, WPE) void ring_kernel(GemmI8Params p, int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  using G = Geo<BM, BN, WM, WN, S>;
  constexpr int BK = G::BK, FM = G::FM, FN = G::FN, KK = G::KK, IA = G::IA, LPT = G::LPT, LPK = G::LPK;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const TileAt<8> at(tiles_m, tiles_n, blockIdx.x);
  const int m0 = at.m * BM, n0 = at.n * BN;
  auto& side = *reinterpret_cast<Side<BM, BN>*>(smem + G::RING);
  typename Side<BM, BN>::Regs sr;
  side.fetch(sr, p, m0, n0);

  // load j covers tile rows (j NW + wave) 8 .. + 8 (A's first, then W's); chunk c of row r lies at
  // c ^ (r / 2 % 8)
  unsigned off[LPT];
#pragma unroll
  for (int j = 0; j < LPT; ++j) {
    const int r = ((j < IA ? j : j - IA) * G::NW + wave) * 8 + (lane >> 3);
    const unsigned ch = (unsigned)((lane & 7) ^ ((r >> 1) & 7)) * 16u;
    off[j] = j < IA ? (unsigned)min(r, p.M - 1 - m0) * (unsigned)p.lda + ch
                    : (unsigned)min(r, p.N - 1 - n0) * (unsigned)p.ldw + ch;
  }
  const __amdgpu_buffer_rsrc_t rA = rows_rsrc(p.A, p.lda, m0, p.M, BM, p.K);
  const __amdgpu_buffer_rsrc_t rW = rows_rsrc(p.W, p.ldw, n0, p.N, BN, p.K);

  i32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

  const int lrow = lane & 31, h = lane >> 5;
  int koff[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) koff[kk] = ((2 * kk + h) ^ ((lrow >> 1) & 7)) * 16;
  const int arow = (wm * G::TM + lrow) * BK, brow = BM * BK + (wn * G::TN + lrow) * BK;

  const int KT = (p.K + BK - 1) / BK;
  const int left = p.K - (KT - 1) * BK;           // bytes of k in the last k-tile

  // load j of k-tile t into its stage
  auto dma = [&](auto jc, int t) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
    constexpr int i = j < IA ? j : j - IA;
    char* dst = smem + t % S * G::STAGE + (j < IA ? 0 : BM * BK) + (i * G::NW + wave) * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(j < IA ? rA : rW, (ORCH_LDS void*)dst, 16, off[j],
                                             (unsigned)t * BK, 0, 0);
  };
  // the MFMAs of k-tile t, with ISSUE the loads of k-tile t + S - 1 between them: MFMA e of k-step
  // kk, then its share of the next k-step's fragments, then its share of the loads
  auto compute = [&](auto vt_c, auto issue_c, auto last_c, int t) __attribute__((always_inline)) {
    constexpr bool ISSUE = decltype(issue_c)::value;
    constexpr int NM = FM * FN, ND = FM + FN;
    const char* base = smem + t % S * G::STAGE;
    i32x4 a[2][FM], b[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) a[0][i] = *reinterpret_cast<const i32x4*>(base + arow + i * 32 * BK + koff[0]);
#pragma unroll
    for (int j = 0; j < FN; ++j) b[0][j] = *reinterpret_cast<const i32x4*>(base + brow + j * 32 * BK + koff[0]);
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, KK>([&](auto kkc) __attribute__((always_inline)) {
      constexpr int kk = decltype(kkc)::value, cur = kk & 1;
      constexpr int nd = kk + 1 < KK ? ND : 0;
      constexpr int l0 = cmin(kk * LPK, LPT), nl = ISSUE ? cmin(kk * LPK + LPK, LPT) - l0 : 0;
      if constexpr (decltype(last_c)::value) {
        if (left < BK) {
          const i32x4 m = within(left, 2 * kk + h);
#pragma unroll
          for (int i = 0; i < FM; ++i) a[cur][i] &= m;
        }
      }
      static_for<0, NM>([&](auto ec) __attribute__((always_inline)) {
        constexpr int e = decltype(ec)::value, i = e / FN, j = e % FN;
        acc[i][j] = mfma<decltype(vt_c)::value>(a[cur][i], b[cur][j], acc[i][j]);
        static_for<e * nd / NM, (e + 1) * nd / NM>([&](auto dc) __attribute__((always_inline)) {
          constexpr int d = decltype(dc)::value;
          if constexpr (d < FM) a[cur ^ 1][d] = *reinterpret_cast<const i32x4*>(base + arow + d * 32 * BK + koff[kk + 1]);
          else b[cur ^ 1][d - FM] = *reinterpret_cast<const i32x4*>(base + brow + (d - FM) * 32 * BK + koff[kk + 1]);
        });
        static_for<l0 + e * nl / NM, l0 + (e + 1) * nl / NM>([&](auto jc) __attribute__((always_inline)) { dma(jc, t + S - 1); });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };
  using No = std::false_type;
  using Yes = std::true_type;

#pragma unroll
  for (int s = 0; s < S - 1; ++s)
    if (s < KT) static_for<0, LPT>([&](auto jc) __attribute__((always_inline)) { dma(jc, s); });
  side.keep(sr);
  auto loop = [&](auto vt) __attribute__((always_inline)) {
    int t = 0;
    for (; t + S - 1 < KT; ++t) {
      wait_vmcnt<(S - 2) * LPT>();
      lds_barrier();
      compute(vt, Yes{}, No{}, t);
    }
    // the last S - 1 (or fewer): all loads are on their way
    for (; t + 1 < KT; ++t) {
      if (S > 3 && t + 3 == KT) wait_vmcnt<(S > 3 ? 2 : 0) * LPT>();
      else if (S > 2 && t + 2 == KT) wait_vmcnt<LPT>();
      else wait_vmcnt<0>();
      lds_barrier();
      compute(vt, No{}, No{}, t);
    }
    wait_vmcnt<0>();
    lds_barrier();
    compute(vt, No{}, Yes{}, t);
    __syncthreads();    // (the areas take the ring's place; the side's values are there)
    const int mw = wm * G::TM, nw = wn * G::TN;
    const float *sa = side.sa + mw, *sw = side.sw + nw, *bias = side.bias + nw;
    staged<T, EPI, decltype(vt)::value>(p, acc, smem + wave * kArea, sa, sw, bias, lane, m0 + mw, n0 + nw);
  };
  // (a wave's own choice: both loops meet the same barriers)
  if (all_vt<EPI>(p, n0 + wn * G::TN)) loop(Yes{});
  else loop(No{});
#endif
}

// ---------------------------------------------------------------------------
// BM x 256 tiles, BM 256 or 192, eight waves (2 x 4, BM / 2 x 64 outputs each), k-tiles of 128
// bytes in two LDS stages, one workgroup a CU that takes tiles until none is left.  The
// k-tiles of its tiles are one sequence: one barrier a k-tile, the next one's loads between the
// MFMAs, and behind a tile's last come the next one's first, whose loads are in flight while
// the outputs are written.  Behind the last tile the buffers of the loads are empty, so that
// they fetch nothing.
template <int BM>
struct BigGeo {
  static constexpr int BN = 256, BK = 128, KK = 4, STAGE = (BM + BN) * BK;
  // (groups of 4, 8 and 16 tile rows: 192 x 256 tiles, 3328 x 1152 -> 3456 20.0, 20.1, 20.2
  // us; 256 x 256, 12288 x 1152 -> 3456, QKV 71-78, 71-76, 75-76, 32768 x 1152 -> 4608, plain 213, 209-215, 218-221)
  static constexpr int GROUP = 4;
  static constexpr int FM = BM / 64, IA = BM / 64, LPT = IA + 4;    // blocks of a wave, loads of A's rows, of all
  static constexpr int SIDES = 2 * STAGE, AREAS = SIDES + 2 * (int)sizeof(Side<BM, BN>), LDS = AREAS + 8 * kArea;
  static_assert(BM % 64 == 0 && LDS <= 160 * 1024, "LDS");
};

template <int BM, typename T, int EPI>
__global__ __launch_bounds__(512, 2) void big_kernel(GemmI8Params p, int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  using G = BigGeo<BM>;
  constexpr int BN = G::BN, BK = G::BK, KK = G::KK, STAGE = G::STAGE, FM = G::FM, IA = G::IA, LPT = G::LPT;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, lr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int tiles = tiles_m * tiles_n, KT = (p.K + BK - 1) / BK;
  Side<BM, BN>* sides = reinterpret_cast<Side<BM, BN>*>(smem + G::SIDES);

  // The loads' place in the sequence: k-tile lk of tile lt.  Load j fills tile rows (8 j + wave)
  // 8 .. + 8, A's first, then W's; chunk c of row r lies at c ^ (r / 2 % 8).
  int lt = blockIdx.x, lk = 0, lside = 0;
  const int lrow = wave * 8 + (lane >> 3), chunk = (lane & 7) ^ ((lrow >> 1) & 7);
  unsigned off[LPT];
  __amdgpu_buffer_rsrc_t rA, rW;
  auto place = [&]() __attribute__((always_inline)) {
    if (lt >= tiles) {
      rA = buffer_rsrc(p.A, 0);
      rW = buffer_rsrc(p.W, 0);
      return;
    }
    const TileAt<G::GROUP> ta(tiles_m, tiles_n, lt);
    const int m0 = ta.m * BM, n0 = ta.n * BN;
#pragma unroll
    for (int j = 0; j < LPT; ++j)
      off[j] = (j < IA ? (unsigned)min(64 * j + lrow, p.M - 1 - m0) * (unsigned)p.lda
                       : (unsigned)min(64 * (j - IA) + lrow, p.N - 1 - n0) * (unsigned)p.ldw) + chunk * 16u;
    rA = rows_rsrc(p.A, p.lda, m0, p.M, BM, p.K);
    rW = rows_rsrc(p.W, p.ldw, n0, p.N, BN, p.K);
    // the tile's scales and biases: 64 values a load, twelve loads over the waves
    Side<BM, BN>& sd = sides[lside];
    const int part = (wave & 3) * 64;
    const unsigned o = (unsigned)(part + lane) * 4u;
    if (wave < 4) {
      const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(p.sa + m0, (size_t)min(p.M - m0, BM) * 4);
      const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(p.sw + n0, (size_t)min(p.N - n0, BN) * 4);
      if (part < BM) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (ORCH_LDS void*)(sd.sa + part), 4, o, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ORCH_LDS void*)(sd.sw + part), 4, o, 0, 0, 0);
    } else if (p.bias) {
      const __amdgpu_buffer_rsrc_t rb = buffer_rsrc(p.bias + n0, (size_t)min(p.N - n0, BN) * 4);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (ORCH_LDS void*)(sd.bias + part), 4, o, 0, 0, 0);
    } else {
      sd.bias[part + lane] = 0.0f;
    }
  };
  auto load = [&](auto jc, int st) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
    char* dst = smem + st * STAGE + (j * 8 + wave) * 1024;     // (W's rows follow A's)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(j < IA ? rA : rW, (ORCH_LDS void*)dst, 16, off[j],
                                             (unsigned)lk * BK, 0, 0);
  };
  auto next = [&]() __attribute__((always_inline)) {
    if (++lk == KT) {
      lk = 0;
      lt += gridDim.x;
      lside ^= 1;
      place();
    }
  };

  i32x16 acc[FM][2];
  int koff[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) koff[kk] = ((2 * kk + h) ^ ((lr >> 1) & 7)) * 16;
  const int arow = (wm * (BM / 2) + lr) * BK, brow = BM * BK + (wn * 64 + lr) * BK;
  const int left = p.K - (KT - 1) * BK;     // bytes of k in a tile's last k-tile
  // the MFMAs of stage st: MFMA e of k-step kk, then its share of the next k-step's fragments
  // and, in the first k-step, of the loads into the other stage.  first: on sums of 0; last: what lies
  // past K cleared
  auto compute = [&](auto vt, auto first_c, auto last_c, int st) __attribute__((always_inline)) {
    const i32x16 zero = {};
    const char* base = smem + st * STAGE;
    i32x4 a[2][FM], b[2][2];
#pragma unroll
    for (int i = 0; i < FM; ++i) a[0][i] = *reinterpret_cast<const i32x4*>(base + arow + i * 32 * BK + koff[0]);
#pragma unroll
    for (int j = 0; j < 2; ++j) b[0][j] = *reinterpret_cast<const i32x4*>(base + brow + j * 32 * BK + koff[0]);
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, KK>([&](auto kkc) __attribute__((always_inline)) {
      constexpr int kk = decltype(kkc)::value, cur = kk & 1, NM = 2 * FM, nd = kk + 1 < KK ? FM + 2 : 0;
      if constexpr (decltype(last_c)::value) {
        if (left < BK) {
          const i32x4 m = within(left, 2 * kk + h);
#pragma unroll
          for (int i = 0; i < FM; ++i) a[cur][i] &= m;
        }
      }
      static_for<0, NM>([&](auto ec) __attribute__((always_inline)) {
        constexpr int e = decltype(ec)::value, i = e / 2, j = e % 2;
        acc[i][j] = mfma<decltype(vt)::value>(a[cur][i], b[cur][j], decltype(first_c)::value && kk == 0 ? zero : acc[i][j]);
        static_for<e * nd / NM, (e + 1) * nd / NM>([&](auto dc) __attribute__((always_inline)) {
          constexpr int d = decltype(dc)::value;
          if constexpr (d < FM) a[cur ^ 1][d] = *reinterpret_cast<const i32x4*>(base + arow + d * 32 * BK + koff[kk + 1]);
          else b[cur ^ 1][d - FM] = *reinterpret_cast<const i32x4*>(base + brow + (d - FM) * 32 * BK + koff[kk + 1]);
        });
        if constexpr (kk == 0)
          static_for<e * LPT / NM, (e + 1) * LPT / NM>([&](auto jc) __attribute__((always_inline)) { load(jc, st ^ 1); });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };

  place();
  static_for<0, LPT>([&](auto jc) __attribute__((always_inline)) { load(jc, 0); });
  int st = 0, side = 0;
  for (int ct = blockIdx.x; ct < tiles; ct += gridDim.x) {
    const TileAt<G::GROUP> ta(tiles_m, tiles_n, ct);
    const int m0 = ta.m * BM + wm * (BM / 2), n0 = ta.n * BN + wn * 64;
    auto tile = [&](auto vt) __attribute__((always_inline)) {
      auto step = [&](auto first, auto last) __attribute__((always_inline)) {
        wait_vmcnt<0>();
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): a missing bias' zeros too
        lds_barrier();
        next();
        compute(vt, first, last, st);
        st ^= 1;
      };
      using Yes = std::true_type;
      using No = std::false_type;
      if (KT == 1) {
        step(Yes{}, Yes{});
      } else {
        step(Yes{}, No{});
        for (int kt = 2; kt < KT; ++kt) step(No{}, No{});
        step(No{}, Yes{});
      }
      const Side<BM, BN>& sd = sides[side];
      staged<T, EPI, decltype(vt)::value>(p, acc, smem + G::AREAS + wave * kArea, sd.sa + wm * (BM / 2), sd.sw + wn * 64,
                                          sd.bias + wn * 64, lane, m0, n0);
    };
    if (all_vt<EPI>(p, n0)) tile(std::true_type{});
    else tile(std::false_type{});
    side ^= 1;
  }
  wait_vmcnt<0>();    // (loads into LDS that is about to be another workgroup's)
#endif
}

// ---------------------------------------------------------------------------
// Few output tiles: four waves, (BM / 32) x (BN / 32) blocks of 32 x 32 x KG groups
// that share the k-tiles of 128 bytes (group g takes g, g + KG, ...; their sums meet in
// LDS).  A ring of S stages a group.
template <int BM, int BN, int KG, int S>
struct SmallGeo {
  static constexpr int NWG = 4 / KG, WN = BN / 32;
  static constexpr int STAGE = (BM + BN) * 128;
  static constexpr int LPT = (BM + BN) / 8 / NWG;         // 1 KB loads per wave and k-tile
  static constexpr int RING = KG * S * STAGE;
  static constexpr int LDS = RING + (int)sizeof(Side<BM, BN>);
  static constexpr int SUMS = (KG - 1) * NWG * 4096;
  static_assert((BM / 32) * (BN / 32) == NWG, "a 32 x 32 block per wave");
  static_assert((BM + BN) / 8 % NWG == 0 && (S - 1) * LPT < 60, "whole loads");
  static_assert(SUMS <= RING && LDS <= 160 * 1024, "LDS");
};

template <int BM, int BN, int KG, int S, typename T, int EPI>
__global__ __launch_bounds__(256) void small_kernel(GemmI8Params p, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  using G = SmallGeo<BM, BN, KG, S>;
  constexpr int LPT = G::LPT;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, lr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = wave % G::NWG, kg = wave / G::NWG;
  const int tiles = p.splits > 1 ? gridDim.x / p.splits : gridDim.x;
  const int split = blockIdx.x / tiles;
  // row-major tiles, an eighth of them in a row on each XCD
  int w = blockIdx.x - split * tiles;
  const int per = tiles / 8;
  if (w < per * 8) w = (w & 7) * per + (w >> 3);
  const int m0 = w / tiles_n * BM, n0 = w % tiles_n * BN;
  const int mw = wg / G::WN * 32, nw = wg % G::WN * 32;
  char* ring = smem + kg * S * G::STAGE;
  auto& side = *reinterpret_cast<Side<BM, BN>*>(smem + G::RING);
  typename Side<BM, BN>::Regs sr;
  if constexpr (EPI != kEpiPartial) side.fetch(sr, p, m0, n0);

  // load i of a k-tile: rows 8 (wg LPT + i) .. + 8 (A first, then W)
  unsigned off[LPT];
#pragma unroll
  for (int i = 0; i < LPT; ++i) {
    const int r0 = (wg * LPT + i) * 8, r = r0 + (lane >> 3);
    const unsigned ch = ((lane & 7) ^ ((r >> 1) & 7)) * 16u;
    off[i] = r0 < BM ? (unsigned)min(r, p.M - 1 - m0) * (unsigned)p.lda + ch
                     : (unsigned)min(r - BM, p.N - 1 - n0) * (unsigned)p.ldw + ch;
  }
  const __amdgpu_buffer_rsrc_t rA = rows_rsrc(p.A, p.lda, m0, p.M, BM, p.K);
  const __amdgpu_buffer_rsrc_t rW = rows_rsrc(p.W, p.ldw, n0, p.N, BN, p.K);
  const int all = (p.K + 127) / 128;
  const int kt0 = EPI == kEpiPartial ? (int)((long long)all * split / p.splits) : 0;
  const int KT = EPI == kEpiPartial ? (int)((long long)all * (split + 1) / p.splits) - kt0 : all;
  const int left = p.K - (kt0 + KT - 1) * 128;
  // this group's t-th k-tile
  auto issue = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      char* dst = ring + t % S * G::STAGE + (wg * LPT + i) * 1024;
      const unsigned k = (unsigned)(kt0 + kg + KG * t) * 128u;
      if ((wg * LPT + i) * 8 < BM) __builtin_amdgcn_raw_ptr_buffer_load_lds(rA, (ORCH_LDS void*)dst, 16, off[i], k, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(rW, (ORCH_LDS void*)dst, 16, off[i], k, 0, 0);
    }
  };
  const int arow = (mw + lr) * 128, wrow = (BM + nw + lr) * 128;
  int koff[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) koff[c] = ((2 * c + h) ^ ((lr >> 1) & 7)) * 16;
  i32x16 acc[1][1];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[0][0][r] = 0;

  // groups differ by at most one k-tile; all meet every barrier
  const int mine = (KT - kg + KG - 1) / KG, NIT = (KT + KG - 1) / KG;
#pragma unroll
  for (int t = 0; t < S - 1; ++t)
    if (t < mine) issue(t);
  if constexpr (EPI != kEpiPartial) side.keep(sr);
  const bool vt = all_vt<EPI>(p, n0 + nw);
  for (int t = 0; t < NIT; ++t) {
    if (t + S - 2 < mine) wait_vmcnt<(S - 2) * LPT>();
    else wait_vmcnt<0>();
    lds_barrier();
    if (t + S - 1 < mine) issue(t + S - 1);
    if (t >= mine) continue;
    const char* base = ring + t % S * G::STAGE;
    i32x4 a[4], b[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      a[c] = *reinterpret_cast<const i32x4*>(base + arow + koff[c]);
      b[c] = *reinterpret_cast<const i32x4*>(base + wrow + koff[c]);
    }
    if (left < 128 && kg + KG * t == KT - 1) {
#pragma unroll
      for (int c = 0; c < 4; ++c) a[c] &= within(left, 2 * c + h);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      // (the block of V^T the other way round: the operands change places)
      const i32x4 x = vt ? a[c] : b[c], y = vt ? b[c] : a[c];
      acc[0][0] = mfma<false>(y, x, acc[0][0]);
    }
  }
  __syncthreads();
  if constexpr (KG > 1) {
    if (kg > 0) {
      int* part = reinterpret_cast<int*>(smem + ((kg - 1) * G::NWG + wg) * 4096) + lane;
#pragma unroll
      for (int r = 0; r < 16; ++r) part[r * 64] = acc[0][0][r];
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int g = 0; g < KG - 1; ++g) {
      const int* part = reinterpret_cast<const int*>(smem + (g * G::NWG + wg) * 4096) + lane;
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][0][r] += part[r * 64];
    }
  }
  if (vt) direct<T, EPI, true>(p, acc, side.sa + mw, side.sw + nw, side.bias + nw, lane, m0 + mw, n0 + nw, split);
  else direct<T, EPI, false>(p, acc, side.sa + mw, side.sw + nw, side.bias + nw, lane, m0 + mw, n0 + nw, split);
#endif
}

// The k-splits' sums, then the caller's epilogue: a workgroup a block of 32 x 32, whose four
// waves share the splits (at most kMaxSplits, so that a wave's loads are in flight at once).
constexpr int kMaxSplits = 16;

template <typename T, int EPI>
__global__ __launch_bounds__(256) void split_sum_kernel(GemmI8Params p, int blocks_n) {
  __shared__ __attribute__((aligned(16))) Side<32, 32> sd;
  __shared__ int part[3][16][64];
  const int lane = threadIdx.x & 63, lr = lane & 31, h = lane >> 5, wave = threadIdx.x >> 6;
  const int m0 = blockIdx.x / blocks_n * 32, n0 = blockIdx.x % blocks_n * 32;
  typename Side<32, 32>::Regs sr;
  sd.fetch(sr, p, m0, n0);
  sd.keep(sr);
  const size_t MN = (size_t)p.M * p.N;
  const bool vt = all_vt<EPI>(p, n0);
  i32x16 acc[1][1];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[0][0][r] = 0;
#pragma unroll
  for (int i = 0; i < kMaxSplits / 4; ++i) {
    const int k = wave + 4 * i;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int x = 8 * (r >> 2) + 4 * h + (r & 3), m = m0 + (vt ? x : lr), n = n0 + (vt ? lr : x);
      if (k < p.splits && m < p.M && n < p.N) acc[0][0][r] += p.ws[k * MN + (size_t)m * p.N + n];
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave - 1][r][lane] = acc[0][0][r];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[0][0][r] += part[0][r][lane] + part[1][r][lane] + part[2][r][lane];
  if (vt) direct<T, EPI, true>(p, acc, sd.sa, sd.sw, sd.bias, lane, m0, n0, 0);
  else direct<T, EPI, false>(p, acc, sd.sa, sd.sw, sd.bias, lane, m0, n0, 0);
}

// ---------------------------------------------------------------------------
// ORCH_INT8_TILE=<index> forces a form (tuning, tests).
static int forced() {
  const char* s = getenv("ORCH_INT8_TILE");
  return s ? atoi(s) : -1;
}

template <typename K>
static hipError_t allow_lds(K kern, int lds) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

template <int BM, int BN, int WM, int WN, int S, int WPE, typename T, int EPI>
static hipError_t launch_ring(const GemmI8Params& p, hipStream_t s) {
  using G = Geo<BM, BN, WM, WN, S>;
  auto kern = ring_kernel<BM, BN, WM, WN, S, WPE, T, EPI>;
  static const hipError_t attr = allow_lds(kern, G::LDS);
  if (attr != hipSuccess) return attr;
  const int tm = ceil_div(p.M, BM), tn = ceil_div(p.N, BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn)), dim3(64 * WM * WN), G::LDS, s, p, tm, tn);
  return hipGetLastError();
}

template <int BM, int BN, int KG, int S, typename T, int EPI>
static hipError_t launch_small(const GemmI8Params& p, hipStream_t s) {
  using G = SmallGeo<BM, BN, KG, S>;
  auto kern = small_kernel<BM, BN, KG, S, T, EPI>;
  static const hipError_t attr = allow_lds(kern, G::LDS);
  if (attr != hipSuccess) return attr;
  const int tn = ceil_div(p.N, BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(p.M, BM) * tn * p.splits)), dim3(256), G::LDS, s, p, tn);
  return hipGetLastError();
}

// Tiles go round 256 workgroups, one a CU.
template <int BM, typename T, int EPI>
static hipError_t launch_big(const GemmI8Params& p, hipStream_t s) {
  using G = BigGeo<BM>;
  auto kern = big_kernel<BM, T, EPI>;
  static const hipError_t attr = allow_lds(kern, G::LDS);
  if (attr != hipSuccess) return attr;
  const int tm = ceil_div(p.M, BM), tn = ceil_div(p.N, G::BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)cmin(tm * tn, 256)), dim3(512), G::LDS, s, p, tm, tn);
  return hipGetLastError();
}

enum Form { k256x256, k192x256, k128x128, k128x128Alone, k64x64, k32x64, k32x32, kForms };

template <typename T, int EPI>
static hipError_t launch_form(int f, const GemmI8Params& p, hipStream_t s) {
  switch (f) {
    case k256x256:
      if constexpr (EPI != kEpiResidual) return launch_big<256, T, EPI>(p, s);
      else return hipErrorInvalidValue;     // (pick() does not take it)
    case k192x256:
      if constexpr (EPI != kEpiResidual) return launch_big<192, T, EPI>(p, s);
      else return hipErrorInvalidValue;     // (pick() does not take it)
    case k128x128: return launch_ring<128, 128, 2, 2, 2, 2, T, EPI>(p, s);
    case k128x128Alone: return launch_ring<128, 128, 4, 2, 4, 2, T, EPI>(p, s);
    case k64x64: return launch_ring<64, 64, 2, 2, 4, 2, T, EPI>(p, s);
    case k32x64: return launch_small<32, 64, 2, 3, T, EPI>(p, s);
    default: return launch_small<32, 32, 4, 3, T, EPI>(p, s);
  }
}

// The form with the least estimated time in us, T its tiles and KT the k-tiles of 128: fitted to M
// from 1 to 32768 at the DiT projections of hidden 384 and 1152 and K up to 4608 (one run each,
// stores of bf16).  Measured, us, 256 x 256 / 192 x 256 / 128 x 128 / alone / 64 x 64 / 32 x 64 / 32 x 32:
//   32768 x 1152 -> 4608  206-229 / 219 / 234 / 273 / 344 / 813 / 1710
//   3328 x 1152 -> 3456       22 /  20 /  24 /  26 /  28 /  58 /  132
//   3328 x 4608 -> 1152       47 /  40 /  29 /  23 /  30 /  50 /   95
//   768 x 4608 -> 1152        46 /  39 /  26 /  17 /  10 /  15 /   27
//   96 x 4608 -> 1152          - /   - /   - /   - / 9.0 / 11.6 / 7.5
// A CU holds one workgroup of the large tiles, of `alone` and of 32 x 32, two of the others, where
// one's outputs are written beside another's products.
struct Plan { int form, splits; };

static Plan pick(int M, int N, int K, int epi, size_t ws_elems) {
  const int f = forced(), kt = ceil_div(K, 128);
  if (f >= 0 && f < kForms && (f > k192x256 || epi != kEpiResidual)) return {f, 1};
  float best = 0.0f;
  int form = -1;
  auto tiles = [&](int bm, int bn) { return (float)ceil_div(M, bm) * ceil_div(N, bn); };
  auto rounds = [&](float t) { return ceilf(t / 256.0f); };
  auto take = [&](int c, float us) {
    if (form < 0 || us < best) form = c, best = us;
  };
  const float k = (float)kt, t128 = tiles(128, 128), t64 = tiles(64, 64), t3264 = tiles(32, 64), t32 = tiles(32, 32);
  // (not for the gated residual, whose stream a lone workgroup waits for: 32205 x 2176 -> 1280 172 us in 256 x 256
  // tiles, 161 in 192 x 256, 157 in 128 x 128; 12288 x 1152 -> 1152 36, 44 and 35-39)
  if (epi != kEpiResidual) {
    take(k256x256, 2.5f + rounds(tiles(256, 256)) * (8.0f + 1.4f * k));
    take(k192x256, 2.5f + rounds(tiles(192, 256)) * (6.5f + 1.1f * k));
  }
  take(k128x128, t128 <= 256 ? 5.5f + 0.65f * k : 3.0f + t128 / 512 * (4.0f + k));
  take(k128x128Alone, 2.0f + rounds(t128) * (2.5f + 0.3f * k) + t128 / 256 * (2.5f + 0.22f * k));
  take(k64x64, t64 <= 256 ? 3.5f + 0.2f * k : 3.0f + t64 / 512 * (1.0f + 0.45f * k));
  take(k32x64, t3264 <= 256 ? 3.2f + 0.22f * k : 3.0f + t3264 / 512 * (1.3f + 0.45f * k));
  take(k32x32, 2.9f + 0.105f * k + (rounds(t32) - 1) * (1.6f + 0.155f * k));
  // Few blocks of a long K: its k-tiles over more workgroups, 16 at least each, and a second launch
  // that adds their sums (32 x 18432 -> 128, plain: 18.2 us, in two launches 5.3 and 7.7; 131056: 113, 11.0 and 10.4)
  if (form == k32x32 && kt >= 96) {
    const int wgs = ceil_div(M, 32) * ceil_div(N, 32), sp = cmin(cmin(256 / cmin(wgs, 256), kMaxSplits), kt / 16);
    if (sp > 1 && (size_t)sp * M * N <= ws_elems) return {form, sp};
  }
  return {form, 1};
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, int EPI>
static hipError_t launch_t(const GemmI8Params& p0, hipStream_t s) {
  GemmI8Params p = p0;
  constexpr int ce = EPI == kEpiResidual ? 4 : 16 / (int)sizeof(T);
  p.wide = p.N % ce == 0 && aligned16(p.out) && (EPI != kEpiResidual || (aligned16(p.gate) && p.gate_stride % 4 == 0));
  if (EPI == kEpiQkv) p.hd_magic = (unsigned)((0x100000000ull + p.head_dim - 1) / p.head_dim);
  if (EPI == kEpiQkv || EPI == kEpiResidual) {
    int l = 0;
    while ((1ll << l) < p.rows_per_batch) ++l;
    p.rpb_shift = 31 + l;
    p.rpb_inverse = (unsigned)(((1ull << p.rpb_shift) + p.rows_per_batch - 1) / p.rows_per_batch);
  }
  const Plan pl = pick(p.M, p.N, p.K, EPI, p.ws ? p.ws_elems : 0);
  p.splits = pl.splits;
  if (pl.splits > 1) {
    if (const hipError_t e = launch_small<32, 32, 4, 3, T, kEpiPartial>(p, s); e != hipSuccess) return e;
    const int bn = ceil_div(p.N, 32), blocks = ceil_div(p.M, 32) * bn;
    hipLaunchKernelGGL((split_sum_kernel<T, EPI>), dim3(blocks), dim3(256), 0, s, p, bn);
    return hipGetLastError();
  }
  return launch_form<T, EPI>(pl.form, p, s);
}

template <typename T>
static hipError_t launch_epi(const GemmI8Params& p, int epi, hipStream_t s) {
  switch (epi) {
    case kEpiStore: return launch_t<T, kEpiStore>(p, s);
    case kEpiGelu: return launch_t<T, kEpiGelu>(p, s);
    case kEpiResidual: return launch_t<float, kEpiResidual>(p, s);
    case kEpiQkv: return launch_t<T, kEpiQkv>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace i8

size_t gemm_int8_workspace_bytes(int M, int N, int K) {
  const i8::Plan pl = i8::pick(M, N, K, kEpiStore, (size_t)-1);
  return pl.splits > 1 ? (size_t)pl.splits * M * N * 4 : 0;
}

hipError_t launch_gemm_int8(const GemmI8Params& p, int epi, int dtype, hipStream_t s) {
  if (p.M <= 0) return hipSuccess;
  return dtype == kBF16 ? i8::launch_epi<bf16>(p, epi, s) : i8::launch_epi<float>(p, epi, s);
}

}  // namespace orch
