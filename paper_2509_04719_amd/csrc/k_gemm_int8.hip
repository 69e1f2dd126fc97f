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

// What a tile's epilogue reads beside its sums, in LDS: scales of its rows, scales
// and biases of its columns.
template <int BM, int BN>
struct Side {
  float sa[BM], sw[BN], bias[BN];
  struct Regs { float a[(BM + 255) / 256], w[(BN + 255) / 256], b[(BN + 255) / 256]; };
  // (loads first, LDS writes behind the prologue's other loads; at least 256 threads)
  __device__ __forceinline__ static void fetch(Regs& r, const GemmI8Params& p, int m0, int n0) {
    const int t = threadIdx.x;
    r.a[0] = t < BM && m0 + t < p.M ? p.sa[m0 + t] : 0.0f;
    r.w[0] = t < BN && n0 + t < p.N ? p.sw[n0 + t] : 0.0f;
    r.b[0] = t < BN && n0 + t < p.N && p.bias ? p.bias[n0 + t] : 0.0f;
  }
  __device__ __forceinline__ void keep(const Regs& r) {
    const int t = threadIdx.x;
    if (t < BM) sa[t] = r.a[0];
    if (t < BN) sw[t] = r.w[0], bias[t] = r.b[0];
  }
  static_assert(BM <= 256 && BN <= 256, "one value a thread");
};

// 32 rows x TN columns of sums, staged in LDS (rows of TN + 4 ints, so that the
// 16-byte writes of 16 rows land in distinct banks), then walked in 16-byte chunks of
// the output's rows, or along V^T's tokens.
template <typename T, int TN, int EPI>
struct Strip {
  static constexpr int LS = TN + 4;
  static constexpr int BYTES = 32 * LS * 4;
  const GemmI8Params& p;
  const int* strip;
  const float *sa, *sw, *bias;   // of the strip's rows, of its columns
  int lane, m0, n0, split;       // its first row and column

  __device__ __forceinline__ float value(int s, float a, float w, float b) const { return fmaf((float)s * a, w, b); }

  __device__ __forceinline__ void rows_store() const {
    constexpr int CE = 16 / sizeof(T), CH = TN / CE, RQ = 64 / CH;
    static_assert(64 % CH == 0, "a lane's columns stay the same");
    const int c = lane % CH * CE, n = n0 + c;
    if (n >= p.N) return;
    float w[CE], b[CE];
#pragma unroll
    for (int e = 0; e < CE; ++e) w[e] = sw[c + e], b[e] = bias[c + e];
    T* out = reinterpret_cast<T*>(p.out);
#pragma unroll
    for (int q = 0; q < 32 / RQ; ++q) {
      const int r = q * RQ + lane / CH, m = m0 + r;
      if (m >= p.M) continue;
      T o[CE];
#pragma unroll
      for (int e = 0; e < CE; e += 4) {
        const i32x4 s = *reinterpret_cast<const i32x4*>(strip + r * LS + c + e);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const float y = value(s[f], sa[r], w[e + f], b[e + f]);
          o[e + f] = from_f<T>(EPI == kEpiGelu ? gelu<T>(y) : y);
        }
      }
      put<CE>(out + (size_t)m * p.N + n, o, p.N - n);
    }
  }

  // CE values to p, `left` of them within the row
  template <int CE, typename U>
  __device__ __forceinline__ void put(U* d, const U* o, int left) const {
    typedef U W __attribute__((ext_vector_type(CE)));
    if (p.wide) {
      W v;
#pragma unroll
      for (int e = 0; e < CE; ++e) v[e] = o[e];
      *reinterpret_cast<W*>(d) = v;
    } else {
#pragma unroll
      for (int e = 0; e < CE; ++e)
        if (e < left) d[e] = o[e];
    }
  }

  __device__ __forceinline__ void rows_residual() const {
    constexpr int CH = TN / 4, RQ = 64 / CH, IT = 32 / RQ;
    const int c = lane % CH * 4, n = n0 + c;
    if (n >= p.N) return;
    float* out = reinterpret_cast<float*>(p.out);
    const f32x4 w = *reinterpret_cast<const f32x4*>(sw + c), b = *reinterpret_cast<const f32x4*>(bias + c);
    const int left = p.N - n;
    int br = m0 / p.rows_per_batch;
    f32x4 h[IT], g[IT];
    // (all loads first: the stores may alias them as far as the compiler knows)
#pragma unroll
    for (int q = 0; q < IT; ++q) {
      const int m = min(m0 + q * RQ + lane / CH, p.M - 1);
      while (m >= (long long)(br + 1) * p.rows_per_batch) ++br;
      const float *hr = out + (size_t)m * p.N + n, *gr = p.gate + br * p.gate_stride + n;
      if (p.wide) {
        h[q] = *reinterpret_cast<const f32x4*>(hr);
        g[q] = *reinterpret_cast<const f32x4*>(gr);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) h[q][e] = e < left ? hr[e] : 0.0f, g[q][e] = e < left ? gr[e] : 0.0f;
      }
    }
#pragma unroll
    for (int q = 0; q < IT; ++q) {
      const int r = q * RQ + lane / CH, m = m0 + r;
      if (m >= p.M) continue;
      const i32x4 s = *reinterpret_cast<const i32x4*>(strip + r * LS + c);
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(g[q][e], value(s[e], sa[r], w[e], b[e]), h[q][e]);
      put<4>(out + (size_t)m * p.N + n, o, left);
    }
  }

  __device__ __forceinline__ void rows_qkv() const {
    const int hd = p.head_dim, hidden = p.hidden, rpb = p.rows_per_batch;
    const size_t ntot = (size_t)p.kv_tokens;
    T* qb = reinterpret_cast<T*>(p.q);
    T* kvb = reinterpret_cast<T*>(p.kv);
    const int b0 = m0 / rpb;
    // Q and K: 16 bytes of one head's row a lane
    if (n0 < 2 * hidden) {
      constexpr int CE = 16 / sizeof(T), CH = TN / CE, RQ = 64 / CH;
      const int c = lane % CH * CE, n = n0 + c;
      if (n < 2 * hidden) {
        const int which = n >= hidden, nn = n - which * hidden;
        const int head = (int)__umulhi((unsigned)nn, p.hd_magic), dd = nn - head * hd;
        float w[CE], bi[CE];
#pragma unroll
        for (int e = 0; e < CE; ++e) w[e] = sw[c + e], bi[e] = bias[c + e];
        int b = b0;
#pragma unroll
        for (int q = 0; q < 32 / RQ; ++q) {
          const int r = q * RQ + lane / CH, m = m0 + r;
          if (m >= p.M) continue;
          while (m >= (long long)(b + 1) * rpb) ++b;
          const int tok = m - b * rpb;
          T* dst = which == 0 ? qb + (((size_t)b * p.heads + head) * rpb + tok) * hd + dd
                              : kvb + b * p.kv_bs + ((size_t)head * ntot + p.tok_offset + tok) * hd + dd;
          typedef T W __attribute__((ext_vector_type(CE)));
          W o;
#pragma unroll
          for (int e = 0; e < CE; e += 4) {
            const i32x4 s = *reinterpret_cast<const i32x4*>(strip + r * LS + c + e);
#pragma unroll
            for (int f = 0; f < 4; ++f) o[e + f] = from_f<T>(value(s[f], sa[r], w[e + f], bi[e + f]));
          }
          *reinterpret_cast<W*>(dst) = o;
        }
      }
    }
    // V^T [head][d][token]: 8 consecutive tokens of one channel a lane, four lanes the
    // strip's 32.  Groups 2 and 3 read their tokens rotated by four (8 LS = 32 mod 64
    // banks would put them on the banks of groups 0 and 1; 4 LS = 16 mod 64 moves them
    // to the free ones), then swap the halves back.
    static_assert((4 * LS) % 64 == 16, "conflict-free V^T reads");
    if (n0 + TN > 2 * hidden) {
#pragma unroll
      for (int q = 0; q < TN / 16; ++q) {
        const int col = q * 16 + (lane >> 2), grp = lane & 3, n = n0 + col;
        if (n < 2 * hidden || n >= p.N) continue;
        const int rot = (grp >> 1) * 4;
        int s[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) s[t] = strip[(grp * 8 + ((t + rot) & 7)) * LS + col];   // token t ^ rot
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int x = s[t], y = s[t + 4];
          s[t] = rot ? y : x;
          s[t + 4] = rot ? x : y;
        }
        T o[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) o[t] = from_f<T>(value(s[t], sa[grp * 8 + t], sw[col], bias[col]));
        const int nn = n - 2 * hidden, head = (int)__umulhi((unsigned)nn, p.hd_magic), dd = nn - head * hd;
        T* vt = kvb + ntot * hidden + ((size_t)head * hd + dd) * ntot + p.tok_offset;
        const int m = m0 + grp * 8;
        int b = b0;
        if (m >= p.M) continue;
        while (m >= (long long)(b + 1) * rpb) ++b;
        const int tok = m - b * rpb;
        T* dst = vt + b * p.kv_bs + tok;
        if (m + 7 < p.M && tok + 7 < rpb && ((uintptr_t)dst & 15) == 0) {
          constexpr int CE = 16 / sizeof(T);
          typedef T W __attribute__((ext_vector_type(CE)));
#pragma unroll
          for (int e = 0; e < 8; e += CE) {
            W v;
#pragma unroll
            for (int f = 0; f < CE; ++f) v[f] = o[e + f];
            *reinterpret_cast<W*>(dst + e) = v;
          }
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const int mm = m + t;
            if (mm < p.M) {
              while (mm >= (long long)(b + 1) * rpb) ++b;
              vt[b * p.kv_bs + (mm - b * rpb)] = o[t];
            }
          }
        }
      }
    }
  }

  // a k-split's sums, rows of ws[split]
  __device__ __forceinline__ void rows_partial() const {
    constexpr int CH = TN / 4, RQ = 64 / CH;
    const int c = lane % CH * 4, n = n0 + c;
    if (n >= p.N) return;
    int* ws = p.ws + (size_t)split * p.M * p.N;
#pragma unroll
    for (int q = 0; q < 32 / RQ; ++q) {
      const int r = q * RQ + lane / CH, m = m0 + r;
      if (m >= p.M) continue;
      const i32x4 s = *reinterpret_cast<const i32x4*>(strip + r * LS + c);
      int* d = ws + (size_t)m * p.N + n;
      if (p.N % 4 == 0) {
        *reinterpret_cast<i32x4*>(d) = s;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.N) d[e] = s[e];
      }
    }
  }

  __device__ __forceinline__ void rows() const {
    if (m0 >= p.M) return;
    if constexpr (EPI == kEpiStore || EPI == kEpiGelu) rows_store();
    else if constexpr (EPI == kEpiResidual) rows_residual();
    else if constexpr (EPI == kEpiPartial) rows_partial();
    else rows_qkv();
  }
};

// Columns of a strip of a wave that holds FN blocks of 32
constexpr int strip_cols(int FN) { return FN % 2 ? 32 : 64; }
constexpr int strip_bytes(int FN) { return 32 * (strip_cols(FN) + 4) * 4; }

// A wave's sums, FM x FN blocks of 32 x 32 from (m0 + mw, n0 + nw) of the tile at (m0,
// n0); the MFMAs make transposed blocks: a lane holds row lane % 32, columns 8 g + 4
// (lane / 32) + 0 .. 3.
template <typename T, int EPI, int FM, int FN, int BM, int BN>
__device__ __forceinline__ void epilogue(const GemmI8Params& p, const i32x16 (&acc)[FM][FN], char* lds, const Side<BM, BN>& side,
                                         int lane, int m0, int n0, int mw, int nw, int split) {
  constexpr int SN = strip_cols(FN), SB = SN / 32;
  using S = Strip<T, SN, EPI>;
  int* strip = reinterpret_cast<int*>(lds);
  const int lr = lane & 31, h = lane >> 5;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int jb = 0; jb < FN; jb += SB) {
#pragma unroll
      for (int j = 0; j < SB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<i32x4*>(strip + lr * S::LS + j * 32 + 8 * g + 4 * h) =
              i32x4{acc[i][jb + j][4 * g], acc[i][jb + j][4 * g + 1], acc[i][jb + j][4 * g + 2], acc[i][jb + j][4 * g + 3]};
      const int mr = mw + 32 * i, nc = nw + 32 * jb;
      S{p, strip, side.sa + mr, side.sw + nc, side.bias + nc, lane, m0 + mr, n0 + nc, split}.rows();
    }
}

// Which tile a workgroup takes: workgroup b is in split b / T of T = tiles_m x
// tiles_n tiles; inside a split XCD-major, then groups of 8 tile rows, column-major
// inside.
struct TileAt {
  int split, m, n;
  __device__ __forceinline__ TileAt(int tiles_m, int tiles_n) {
    const int T = tiles_m * tiles_n;
    split = __builtin_amdgcn_readfirstlane(blockIdx.x / T);
    int pid = blockIdx.x - split * T;
    const int per = T / 8;
    if (pid < per * 8) pid = (pid & 7) * per + (pid >> 3);
    constexpr int GROUP = 8;
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
// BM x BN tile over WM x WN waves, k-tiles of BK bytes in a ring of S stages: one
// barrier a k-tile; the loads of tile kt + S - 1 lie between the MFMAs of tile kt.
template <int BM, int BN, int BK, int WM, int WN, int S>
struct Geo {
  static constexpr int NW = WM * WN;
  static constexpr int TM = BM / WM, TN = BN / WN;  // wave tile
  static constexpr int FM = TM / 32, FN = TN / 32;  // 32x32 blocks per wave
  static constexpr int CPR = BK / 16;               // 16-byte chunks per row
  static constexpr int RPL = 1024 / BK;             // rows per wave-level load
  static constexpr int Q = 256 / BK;                // rows per 256-byte bank sweep
  static constexpr int IA = BM / (NW * RPL), IB = BN / (NW * RPL);
  static constexpr int LPT = IA + IB;               // loads per lane per k-tile
  static constexpr int STAGE = (BM + BN) * BK;
  static constexpr int KK = BK / 32;                // MFMA k-steps per k-tile
  static constexpr int LPK = S == 2 ? LPT : (LPT + KK - 1) / KK;
  static constexpr int STRIPS = NW * strip_bytes(FN);
  static constexpr int RING = S * STAGE > STRIPS ? S * STAGE : STRIPS;   // the strips take the ring's place
  static constexpr int LDS = RING + (int)sizeof(Side<BM, BN>);
  static_assert(BK == 64 || BK == 128, "k-tile");
  static_assert(NW >= 4 && TM % 32 == 0 && TN % 32 == 0, "wave tile");
  static_assert(BM % (NW * RPL) == 0 && BN % (NW * RPL) == 0, "rows per wave");
  static_assert(S >= 2 && LPT * (S - 1) < 60 && LDS <= 160 * 1024, "pipeline depth");
};

template <int BM, int BN, int BK, int WM, int WN, int S, int WPE, typename T, int EPI>
__global__ __launch_bounds__(64 * WM * WN, WPE) void ring_kernel(GemmI8Params p, int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  using G = Geo<BM, BN, BK, WM, WN, S>;
  constexpr int FM = G::FM, FN = G::FN, KK = G::KK, IA = G::IA, LPT = G::LPT, LPK = G::LPK;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const TileAt at(tiles_m, tiles_n);
  const int m0 = at.m * BM, n0 = at.n * BN;
  auto& side = *reinterpret_cast<Side<BM, BN>*>(smem + G::RING);
  typename Side<BM, BN>::Regs sr;
  if constexpr (EPI != kEpiPartial) side.fetch(sr, p, m0, n0);

  // load j covers tile rows (j NW + wave) RPL .. + RPL - 1 (A's first, then W's)
  unsigned off[LPT];
#pragma unroll
  for (int j = 0; j < LPT; ++j) {
    const int r = ((j < IA ? j : j - IA) * G::NW + wave) * G::RPL + lane / G::CPR;
    const int ch = (lane % G::CPR) ^ ((r / G::Q) % G::CPR);
    off[j] = j < IA ? (unsigned)min(r, p.M - 1 - m0) * (unsigned)p.lda + ch * 16u
                    : (unsigned)min(r, p.N - 1 - n0) * (unsigned)p.ldw + ch * 16u;
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
  for (int kk = 0; kk < KK; ++kk) koff[kk] = ((2 * kk + h) ^ ((lrow / G::Q) % G::CPR)) * 16;
  const int arow = (wm * G::TM + lrow) * BK, brow = BM * BK + (wn * G::TN + lrow) * BK;

  // this split's k-tiles
  const int all = (p.K + BK - 1) / BK;
  const int kt0 = EPI == kEpiPartial ? (int)((long long)all * at.split / p.splits) : 0;
  const int KT = EPI == kEpiPartial ? (int)((long long)all * (at.split + 1) / p.splits) - kt0 : all;
  const int left = p.K - (kt0 + KT - 1) * BK;     // bytes of k in its last one

  // load j of its k-tile kt into stage st
  auto dma = [&](auto jc, int kt, int st) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
    constexpr int i = j < IA ? j : j - IA;
    char* dst = smem + st * G::STAGE + (j < IA ? 0 : BM * BK) + (i * G::NW + wave) * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(j < IA ? rA : rW, (ORCH_LDS void*)dst, 16, off[j],
                                             (unsigned)(kt0 + kt) * BK, 0, 0);
  };
  // the MFMAs of stage st, with ISSUE the loads of k-tile ikt into stage ist between
  // them: MFMA e of k-step kk, then its share of the next k-step's fragments, then its
  // share of the loads
  auto compute = [&](int st, auto issue_c, auto last_c, int ikt, int ist) __attribute__((always_inline)) {
    constexpr bool ISSUE = decltype(issue_c)::value;
    constexpr int NM = FM * FN, ND = FM + FN;
    const char* base = smem + st * G::STAGE;
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
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[cur][j], a[cur][i], acc[i][j], 0, 0, 0);
        static_for<e * nd / NM, (e + 1) * nd / NM>([&](auto dc) __attribute__((always_inline)) {
          constexpr int d = decltype(dc)::value;
          if constexpr (d < FM) a[cur ^ 1][d] = *reinterpret_cast<const i32x4*>(base + arow + d * 32 * BK + koff[kk + 1]);
          else b[cur ^ 1][d - FM] = *reinterpret_cast<const i32x4*>(base + brow + (d - FM) * 32 * BK + koff[kk + 1]);
        });
        static_for<l0 + e * nl / NM, l0 + (e + 1) * nl / NM>([&](auto jc) __attribute__((always_inline)) { dma(jc, ikt, ist); });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };
  using No = std::false_type;
  using Yes = std::true_type;

#pragma unroll
  for (int s = 0; s < S - 1; ++s)
    if (s < KT) static_for<0, LPT>([&](auto jc) __attribute__((always_inline)) { dma(jc, s, s); });
  if constexpr (EPI != kEpiPartial) side.keep(sr);
  int kt = 0;
  for (; kt + S - 1 < KT; ++kt) {
    wait_vmcnt<(S - 2) * LPT>();
    lds_barrier();
    compute(kt % S, Yes{}, No{}, kt + S - 1, (kt + S - 1) % S);
  }
  // the last S - 1 (or fewer): all loads are on their way
  for (; kt + 1 < KT; ++kt) {
    if (S > 3 && kt + 3 == KT) wait_vmcnt<(S > 3 ? 2 : 0) * LPT>();
    else if (S > 2 && kt + 2 == KT) wait_vmcnt<LPT>();
    else wait_vmcnt<0>();
    lds_barrier();
    compute(kt % S, No{}, No{}, 0, 0);
  }
  wait_vmcnt<0>();
  lds_barrier();
  compute(kt % S, No{}, Yes{}, 0, 0);

  __syncthreads();
  epilogue<T, EPI>(p, acc, smem + wave * strip_bytes(FN), side, lane, m0, n0, wm * G::TM, wn * G::TN, at.split);
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
  static constexpr int STRIP = strip_bytes(1);
  static_assert((BM / 32) * (BN / 32) == NWG, "a 32 x 32 block per wave");
  static_assert((BM + BN) / 8 % NWG == 0 && (S - 1) * LPT < 60, "whole loads");
  static_assert(SUMS + NWG * STRIP <= RING && LDS <= 160 * 1024, "LDS");
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
    for (int c = 0; c < 4; ++c) acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[c], a[c], acc[0][0], 0, 0, 0);
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
  // (the strips lie past the groups' sums)
  epilogue<T, EPI>(p, acc, smem + G::SUMS + wg * G::STRIP, side, lane, m0, n0, mw, nw, split);
#endif
}

// The k-splits' sums, then the caller's epilogue: a strip of 32 x 64 a wave.
template <typename T, int EPI>
__global__ __launch_bounds__(256) void split_sum_kernel(GemmI8Params p, int strips_n, int strips) {
  using S = Strip<T, 64, EPI>;
  __shared__ __attribute__((aligned(16))) int lds[4][S::BYTES / 4];
  __shared__ __attribute__((aligned(16))) float sides[4][32 + 64 + 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int id = blockIdx.x * 4 + wave;
  if (id >= strips) return;
  const int m0 = id / strips_n * 32, n0 = id % strips_n * 64;
  int* strip = lds[wave];
  float* sd = sides[wave];
  if (lane < 32) sd[lane] = m0 + lane < p.M ? p.sa[m0 + lane] : 0.0f;
  sd[32 + lane] = n0 + lane < p.N ? p.sw[n0 + lane] : 0.0f;
  sd[96 + lane] = n0 + lane < p.N && p.bias ? p.bias[n0 + lane] : 0.0f;
  const size_t MN = (size_t)p.M * p.N;
  const int n = n0 + lane;
  for (int r = 0; r < 32; ++r) {
    int s = 0;
    if (m0 + r < p.M && n < p.N)
      for (int k = 0; k < p.splits; ++k) s += p.ws[k * MN + (size_t)(m0 + r) * p.N + n];
    strip[r * S::LS + lane] = s;
  }
  S{p, strip, sd, sd + 32, sd + 96, lane, m0, n0, 0}.rows();
}

// ---------------------------------------------------------------------------
// ORCH_INT8_TILE=<index> forces a form (tuning, tests).
static int forced() {
  const char* s = getenv("ORCH_INT8_TILE");
  return s ? atoi(s) : -1;
}

template <typename K>
static void allow_lds(K kern, int lds) {
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

template <int BM, int BN, int BK, int WM, int WN, int S, int WPE, typename T, int EPI>
static void launch_ring(const GemmI8Params& p, hipStream_t s) {
  using G = Geo<BM, BN, BK, WM, WN, S>;
  auto kern = ring_kernel<BM, BN, BK, WM, WN, S, WPE, T, EPI>;
  static const bool once = (allow_lds(kern, G::LDS), true);
  (void)once;
  const int tm = ceil_div(p.M, BM), tn = ceil_div(p.N, BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn * p.splits)), dim3(64 * WM * WN), G::LDS, s, p, tm, tn);
}

template <int BM, int BN, int KG, int S, typename T, int EPI>
static void launch_small(const GemmI8Params& p, hipStream_t s) {
  using G = SmallGeo<BM, BN, KG, S>;
  auto kern = small_kernel<BM, BN, KG, S, T, EPI>;
  static const bool once = (allow_lds(kern, G::LDS), true);
  (void)once;
  const int tn = ceil_div(p.N, BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(p.M, BM) * tn * p.splits)), dim3(256), G::LDS, s, p, tn);
}

enum Form { k256x128, k128x128, k64x64, k32x64, k32x32, kForms };

template <typename T, int EPI>
static void launch_form(int f, const GemmI8Params& p, hipStream_t s) {
  switch (f) {
    case k256x128: launch_ring<256, 128, 64, 2, 2, 3, 2, T, EPI>(p, s); break;
    case k128x128: launch_ring<128, 128, 128, 2, 2, 2, 2, T, EPI>(p, s); break;
    case k64x64: launch_small<64, 64, 1, 3, T, EPI>(p, s); break;
    case k32x64: launch_small<32, 64, 2, 3, T, EPI>(p, s); break;
    default: launch_small<32, 32, 4, 3, T, EPI>(p, s); break;
  }
}

struct Plan { int form, splits; };

static Plan pick(int M, int N, int K, size_t ws_elems) {
  const int f = forced();
  if (f >= 0 && f < kForms) return {f, 1};
  const long long blocks = (long long)ceil_div(M, 32) * ceil_div(N, 32);
  if (blocks <= 512) return {k32x32, 1};
  if (blocks <= 2048) return {k32x64, 1};
  if (blocks <= 4096) return {k64x64, 1};
  return {(long long)ceil_div(M, 256) * ceil_div(N, 128) >= 256 ? k256x128 : k128x128, 1};
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, int EPI>
static hipError_t launch_t(const GemmI8Params& p0, hipStream_t s) {
  GemmI8Params p = p0;
  constexpr int ce = EPI == kEpiResidual ? 4 : 16 / (int)sizeof(T);
  p.wide = p.N % ce == 0 && aligned16(p.out) && (EPI != kEpiResidual || (aligned16(p.gate) && p.gate_stride % 4 == 0));
  if (EPI == kEpiQkv) p.hd_magic = (unsigned)((0x100000000ull + p.head_dim - 1) / p.head_dim);
  const Plan pl = pick(p.M, p.N, p.K, p.ws ? p.ws_elems : 0);
  p.splits = pl.splits;
  if (pl.splits > 1) {
    launch_form<T, kEpiPartial>(pl.form, p, s);
    const int sn = ceil_div(p.N, 64), strips = ceil_div(p.M, 32) * sn;
    hipLaunchKernelGGL((split_sum_kernel<T, EPI>), dim3(ceil_div(strips, 4)), dim3(256), 0, s, p, sn, strips);
  } else {
    launch_form<T, EPI>(pl.form, p, s);
  }
  return hipGetLastError();
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
  const i8::Plan pl = i8::pick(M, N, K, (size_t)-1);
  return pl.splits > 1 ? (size_t)pl.splits * M * N * 4 : 0;
}

hipError_t launch_gemm_int8(const GemmI8Params& p, int epi, int dtype, hipStream_t s) {
  if (p.M <= 0) return hipSuccess;
  return dtype == kBF16 ? i8::launch_epi<bf16>(p, epi, s) : i8::launch_epi<float>(p, epi, s);
}

}  // namespace orch
