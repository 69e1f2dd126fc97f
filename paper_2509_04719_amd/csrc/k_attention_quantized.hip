// Attention of a band's queries over the whole image, K/V of the band's own tokens
// fresh (operand type) and of every other token in the 8-bit cache.
//
// Flash style on the matrix cores.  A workgroup of NW waves takes 32 NW queries
// of one (branch, head), a wave 32 of them, 64 keys a tile.  Scores are formed
// transposed, S^T = K Q^T, so that a lane owns one query column and the running
// max and sum of the softmax stay in the lane.
#include <cfloat>

#include "common.h"
#include "kernels.h"

namespace orch {

namespace q8attn {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 16 bytes at any element's address (fresh V^T rows start anywhere)
typedef unsigned u32x4_u __attribute__((ext_vector_type(4), aligned(2)));

constexpr int BKV = 64;

__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// key of row r of a 32-key half of S^T: bits 2 and 3 swapped, so that the eight scores a lane
// holds of a 16-key chunk are consecutive keys
__device__ __forceinline__ int kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// every LDS operation of the wave done, then the workgroup's barrier; loads from memory stay in flight
__device__ __forceinline__ void lds_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------
// bf16
template <int D, int NW>
struct Geo {
  static constexpr int NC = (D + 15) / 16;       // 16-channel chunks of a score
  static constexpr bool M32 = D % 32 == 0;       // PV on 32x32x16, else on 16x16x32
  static constexpr int NT = M32 ? D / 32 : NC;   // row tiles of O^T
  static constexpr int KP = NC * 32 + 16;        // bytes of a K row: an odd number of 16-byte chunks
  static constexpr int VP = M32 ? (D * 2 % 128 == 64 ? D * 2 : D * 2 + 64) : NC * 32;   // of a V row
  static constexpr int KT = BKV * KP, VT = BKV * VP;
  static constexpr int LDS = 2 * (KT + VT);
  static constexpr int THREADS = 64 * NW;
  static constexpr int CPT = D / 8;              // 8-channel chunks of a token
  static constexpr int SL = (BKV * CPT + THREADS - 1) / THREADS;   // chunks of a thread, K and V each
  static constexpr int WPC = cmin(8 / NW, 160 * 1024 / LDS);       // workgroups of a CU
  static constexpr int WPE = (WPC * NW + 3) / 4;                   // waves of a SIMD
  static constexpr bool EVEN = THREADS % CPT == 0;                 // a thread's chunks are THREADS / CPT keys apart
  static constexpr bool FRESH = NW == 4;         // fresh tiles are fetched ahead too
};

struct Split {
  int ns;            // workgroups that share a query tile's keys
  float* part_o;     // fp32 [tiles * ns][32 NW][D], unnormalised
  float2* part_ml;   // (max, sum)
};

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, (Geo<D, NW>::WPE)) void attn_q8_kernel(AttnQParams p, Split sp) {
  using G = Geo<D, NW>;
  constexpr int NC = G::NC, NT = G::NT, SL = G::SL, CPT = G::CPT, TH = G::THREADS;
  constexpr bool M32 = G::M32;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, h = lane >> 5;
  const int i16 = lane & 15, g16 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // workgroups in the order (branch, head, query tile, split); an eighth of them in a row on
  // each XCD, so that those that read the same K/V share an L2
  const int n_qt = (p.n_q + 32 * NW - 1) / (32 * NW);
  const int NWG = gridDim.x;
  int w = blockIdx.x;
  if (w < NWG / 8 * 8) w = (w & 7) * (NWG / 8) + (w >> 3);
  const int unit = w / sp.ns, part = w - unit * sp.ns;
  const int pair = unit / n_qt, q0 = (unit - pair * n_qt) * 32 * NW + 32 * wave;
  const int b = pair / p.heads, head = pair - b * p.heads;
  const int N = p.c.tokens, fb = p.fresh_begin, nf = p.n_fresh;
  const int nkt = (N + BKV - 1) / BKV;
  const int t0 = (int)((long long)nkt * part / sp.ns), NIT = (int)((long long)nkt * (part + 1) / sp.ns) - t0;
  const size_t H = (size_t)p.heads * D;
  const unsigned char* k8 = p.c.values + b * p.c.values_bs + (size_t)head * N * D;
  const unsigned char* v8 = p.c.values + b * p.c.values_bs + (size_t)(p.heads + head) * N * D;
  const unsigned char* ke = p.c.exps + b * p.c.exps_bs + (size_t)head * N;
  const unsigned char* ve = p.c.exps + b * p.c.exps_bs + (size_t)(p.heads + head) * N;
  const bf16 *kf = nullptr, *vf = nullptr;
  if (nf > 0) {
    kf = reinterpret_cast<const bf16*>(p.kv_fresh) + b * p.fresh_bs + (size_t)head * nf * D;
    vf = reinterpret_cast<const bf16*>(p.kv_fresh) + b * p.fresh_bs + nf * H + (size_t)head * D * nf;
  }

  // K rows' padding channels [D, 16 NC) and V's: zero, never written again
  if constexpr (D % 16 != 0) {
    for (int i = tid; i < 2 * BKV; i += TH) {
      *reinterpret_cast<u32x4*>(smem + (i / BKV) * G::KT + (i % BKV) * G::KP + 2 * D) = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>(smem + 2 * G::KT + (i / BKV) * G::VT + (i % BKV) * G::VP + 2 * D) = u32x4{0, 0, 0, 0};
    }
  }

  // Staging.  A tile of 64 tokens is contiguous in the cache: chunk id (8 channels) of key
  // id / CPT.  Key k of the tile goes to K row k, and to V row vrow(k): the transposing reads
  // below take keys 8 g + 4 x + r, r = 0 .. 3, of several g at once, which then lie in
  // consecutive rows.
  auto vrow = [](int k) __attribute__((always_inline)) { return (k & 32) | (k & 4) << 2 | (k & 24) >> 1 | (k & 3); };
  constexpr int KS = TH / CPT;                              // EVEN: keys from slot to slot
  static_assert(!G::EVEN || (KS & (KS - 1)) == 0, "a slot's rows are a constant away");
  int k_dst_[G::EVEN ? 1 : SL], v_dst_[G::EVEN ? 1 : SL], key_[G::EVEN ? 1 : SL];
#pragma unroll
  for (int i = 0; i < (G::EVEN ? 1 : SL); ++i) {
    const int id = i * TH + tid, key = id / CPT, ch = id - key * CPT;
    key_[i] = key;
    k_dst_[i] = (key & 63) * G::KP + ch * 16;
    v_dst_[i] = 2 * G::KT + vrow(key & 63) * G::VP + ch * 16;
  }
  auto key_of = [&](int i) __attribute__((always_inline)) { return G::EVEN ? key_[0] + i * KS : key_[i]; };
  auto k_dst = [&](int i) __attribute__((always_inline)) { return G::EVEN ? k_dst_[0] + i * KS * G::KP : k_dst_[i]; };
  auto v_dst = [&](int i) __attribute__((always_inline)) { return G::EVEN ? v_dst_[0] + vrow(i * KS) * G::VP : v_dst_[i]; };
  const bool last_on = (SL - 1) * TH + tid < BKV * CPT;     // the last slot's chunk exists
  auto on = [&](int i) __attribute__((always_inline)) { return (BKV * CPT) % TH == 0 || i + 1 < SL || last_on; };

  enum { kStale = 0, kFresh = 1, kMixed = 2 };
  auto type_of = [&](int t) {
    const int n0 = t * BKV;
    if (n0 + BKV <= N && (n0 + BKV <= fb || n0 >= fb + nf)) return (int)kStale;
    if (G::FRESH && n0 >= fb && n0 + BKV <= fb + nf) return (int)kFresh;
    return (int)kMixed;
  };
  typedef unsigned raw __attribute__((ext_vector_type(G::FRESH ? 4 : 2)));
  raw kraw[SL], vraw[SL];
  unsigned kexp[SL], vexp[SL];
  auto set = [](raw& r, const u32x4& x) __attribute__((always_inline)) {
    if constexpr (G::FRESH) r = x;
  };
  auto get = [](const raw& r) __attribute__((always_inline)) {
    if constexpr (G::FRESH) return r;
    else return u32x4{r[0], r[1], 0, 0};
  };
  auto load_k = [&](int t) {
    const int type = type_of(t);
    if (type == kStale) {
      const unsigned char* src = k8 + (size_t)t * BKV * D;
      const unsigned char* e = ke + t * BKV;
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) {
          const u32x2 x = *reinterpret_cast<const u32x2*>(src + (i * TH + tid) * 8);
          kraw[i][0] = x[0];
          kraw[i][1] = x[1];
          kexp[i] = e[key_of(i)];
        }
    } else if (G::FRESH && type == kFresh) {
      const bf16* src = kf + (size_t)(t * BKV - fb) * D;
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) set(kraw[i], *reinterpret_cast<const u32x4*>(src + (i * TH + tid) * 8));
    }
  };
  auto load_v = [&](int t) {
    const int type = type_of(t);
    if (type == kStale) {
      const unsigned char* src = v8 + (size_t)t * BKV * D;
      const unsigned char* e = ve + t * BKV;
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) {
          const u32x2 x = *reinterpret_cast<const u32x2*>(src + (i * TH + tid) * 8);
          vraw[i][0] = x[0];
          vraw[i][1] = x[1];
          vexp[i] = e[key_of(i)];
        }
    } else if (G::FRESH && type == kFresh) {
      // channel id / 8, keys 8 (id % 8) .. +8
      const bf16* src = vf + (t * BKV - fb);
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) {
          const int id = i * TH + tid;
          const u32x4_u x = *reinterpret_cast<const u32x4_u*>(src + (size_t)(id >> 3) * nf + (id & 7) * 8);
          set(vraw[i], u32x4{x[0], x[1], x[2], x[3]});
        }
    }
  };
  auto widen = [](unsigned x0, unsigned x1, unsigned e) {
    const float s = scale_of(e);
    u32x4 r;
    r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, s, false));
    r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, s, true));
    r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, s, false));
    r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, s, true));
    return r;
  };
  // a chunk of a tile that the band's edge or the last key crosses
  auto mixed = [&](int t, int i, bool isk) {
    const int n = t * BKV + key_of(i), f = n - fb, ch = i * TH + tid - key_of(i) * CPT;
    u32x4 r = {0, 0, 0, 0};
    if ((unsigned)f < (unsigned)nf) {
      if (isk) {
        r = *reinterpret_cast<const u32x4*>(kf + (size_t)f * D + ch * 8);
      } else {
        const unsigned short* src = reinterpret_cast<const unsigned short*>(vf) + (size_t)ch * 8 * nf + f;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = src[(size_t)2 * e * nf] | (unsigned)src[(size_t)(2 * e + 1) * nf] << 16;
      }
    } else if (n < N) {
      const u32x2 x = *reinterpret_cast<const u32x2*>((isk ? k8 : v8) + (size_t)n * D + ch * 8);
      r = widen(x[0], x[1], (isk ? ke : ve)[n]);
    }
    return r;
  };
  auto store_k = [&](int t) {
    const int type = type_of(t);
    char* dst = smem + (t & 1) * G::KT;
#pragma unroll
    for (int i = 0; i < SL; ++i)
      if (on(i)) {
        u32x4 x;
        if (type == kStale) x = widen(kraw[i][0], kraw[i][1], kexp[i]);
        else if (G::FRESH && type == kFresh) x = get(kraw[i]);
        else x = mixed(t, i, true);
        *reinterpret_cast<u32x4*>(dst + k_dst(i)) = x;
      }
  };
  auto store_v = [&](int t) {
    const int type = type_of(t);
    char* dst = smem + (t & 1) * G::VT;
    if (G::FRESH && type == kFresh) {
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) {
          const int id = i * TH + tid;
          const u32x4 x = get(vraw[i]);
          unsigned short* col = reinterpret_cast<unsigned short*>(dst + 2 * G::KT + vrow((id & 7) * 8) * G::VP) + (id >> 3);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            col[vrow(e) * (G::VP / 2)] = (unsigned short)(x[e >> 1] >> (16 * (e & 1)));
        }
    } else {
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(i)) {
          u32x4 x;
          if (type == kStale) x = widen(vraw[i][0], vraw[i][1], vexp[i]);
          else x = mixed(t, i, false);
          *reinterpret_cast<u32x4*>(dst + v_dst(i)) = x;
        }
    }
  };

  // this lane's query (B operand): channels 16 c + 8 h .. +8
  const int qrow = min(q0 + lc, p.n_q - 1);
  const bf16* qp = reinterpret_cast<const bf16*>(p.q) + (((size_t)b * p.heads + head) * p.n_q + qrow) * D;
  bf16x8 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (16 * c + 8 * h < D) {
      qf[c] = *reinterpret_cast<const bf16x8*>(qp + 16 * c + 8 * h);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[c][e] = (bf16)0.0f;
    }
  }
  const float scale = 1.4426950408889634f / sqrtf((float)D);   // log2(e) / sqrt(d)

  // fragment reads: K row of key 32 sub + kperm(lc), chunk 2 c + h; V rows by the transposing
  // read (lane i of 16 points at four channels of row i / 4 and gets channel i of the four rows)
  const int k_rd = kperm(lc) * G::KP + 16 * h;
  const int v_rd = 2 * G::KT + (M32 ? (4 * h + (i16 >> 2)) * G::VP + (g16 & 1) * 32 : (4 * g16 + (i16 >> 2)) * G::VP) + (i16 & 3) * 8;
  auto k_frag = [&](int t, int sub, int c) __attribute__((always_inline)) {
    return *reinterpret_cast<const bf16x8*>(smem + (t & 1) * G::KT + sub * 32 * G::KP + k_rd + 32 * c);
  };
  // O^T tile tt; M32: keys 16 ci .. +16 of the half, else all its 32
  auto v_frag = [&](int t, int sub, int tt, int ci) __attribute__((always_inline)) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const char* a = smem + (t & 1) * G::VT + v_rd + (sub * 32 + (M32 ? 8 * ci : 0)) * G::VP + tt * (M32 ? 64 : 32);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORCH_LDS s16x4*)(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORCH_LDS s16x4*)(a + 16 * G::VP));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  // O^T.  M32: tile t (channels 32 t ..) of the lane's query, 16 registers.  Else tile t (channels 16
  // t ..) of queries 16 j + (lane & 15): four registers at 4 (f % 4) of oo[f / 4], f = 2 t + j.
  constexpr int NO = M32 ? NT : (2 * NT + 3) / 4;
  f32x16 oo[NO];
  const f32x16 zero16 = {};
#pragma unroll
  for (int k = 0; k < NO; ++k) oo[k] = zero16;
  auto pv = [&](auto tc, auto jc, const bf16x8& v, const bf16x8& pp) __attribute__((always_inline)) {
    constexpr int t = decltype(tc)::value, j = decltype(jc)::value;
    if constexpr (M32) {
      oo[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pp, oo[t], 0, 0, 0);
    } else {
      constexpr int f = 2 * t + j;
      f32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = oo[f / 4][4 * (f % 4) + i];
      r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pp, r, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) oo[f / 4][4 * (f % 4) + i] = r[i];
    }
  };
  // the probabilities of a half from the score layout (chunk ci, lane half h: keys 16 ci + 8 h .. +8
  // of query lane & 31) to the B operand of the 16x16x32 MFMA (pp[j]: keys 8 (lane >> 4) .. +8 of
  // query 16 j + (lane & 15)): the 32-lane swap, then the 16-lane swap
  auto p_swap = [&](bf16x8(&pp)[2]) __attribute__((always_inline)) {
    if constexpr (!M32) {
      const u32x4 x = __builtin_bit_cast(u32x4, pp[0]), y = __builtin_bit_cast(u32x4, pp[1]);
      u32x4 a, c;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(x[i], y[i], false, false);
        const auto t = __builtin_amdgcn_permlane16_swap(r[0], r[1], false, false);
        a[i] = t[0];
        c[i] = t[1];
      }
      pp[0] = __builtin_bit_cast(bf16x8, a);
      pp[1] = __builtin_bit_cast(bf16x8, c);
    }
  };
  auto rescale = [&](float alpha) __attribute__((always_inline)) {
    if constexpr (M32) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) oo[t][r] *= alpha;
    } else {
      float aj[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) aj[j] = __shfl(alpha, 16 * j + i16, kWave);
#pragma unroll
      for (int f = 0; f < 2 * NT; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) oo[f / 4][4 * (f % 4) + r] *= aj[f & 1];
    }
  };
  // a query's largest score of a half, in log2 units (the rounded product)
  auto query_max = [&](const f32x16& v) __attribute__((always_inline)) {
    float mx = fmaxf(fmaxf(v[0], v[1]), v[2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) mx = fmaxf(fmaxf(mx, v[r]), v[r + 1]);
    return max_xhalf(fmaxf(mx, v[15])) * scale;
  };

  // Running max m_run (log2 units).  A raise puts it kLead above the largest score so far, and the next
  // comes when a probability reaches 2, seen by one bit of the rounded probabilities, so
  // no max is taken in the common case.  `careful` halves (the first one; while a query has had no
  // score above minus infinity; maxima past 2^20, where score * scale - max in one rounding is
  // not 0 for the largest score) take the max first and the difference of the rounded product.
  constexpr float kLead = 7.0f, kHuge = 0x1p20f;
  float m_run = -INFINITY, l_run = 0.0f;
  bool careful = true;
  auto lead = [&](float mx) __attribute__((always_inline)) { return fabsf(mx) < kHuge ? ceilf(mx) + kLead : mx; };
  auto raised = [&](float mx) __attribute__((always_inline)) { return mx > m_run && !(mx < m_run + 1.0f); };
  auto needs_care = [&]() __attribute__((always_inline)) { return __any(!(fabsf(m_run) <= 2 * kHuge)); };

  // One 32-key half: exponentials of its scores sc between the MFMAs of the next half's scores
  // (NEXT: tile nt, half nsub, into sn) and of the previous half's O^T += V^T P^T (pp; V
  // of tile pt, half psub).  Its probabilities go to pc.
  auto step = [&](auto next_c, bool first, f32x16& sc, int nt, int nsub, f32x16& sn, int pt, int psub,
                  bf16x8(&pp)[2], bf16x8(&pc)[2]) __attribute__((always_inline)) {
    constexpr bool NEXT = decltype(next_c)::value;
    constexpr int VF = M32 ? 2 : 1;
    bf16x8 vp[VF][NT], kn[NEXT ? NC : 1];
#pragma unroll
    for (int tt = 0; tt < NT; ++tt) vp[0][tt] = v_frag(pt, psub, tt, 0);
    if constexpr (NEXT) {
#pragma unroll
      for (int c = 0; c < NC / 2; ++c) kn[c] = k_frag(nt, nsub, c);
    }
    // (the rest between the MFMAs of the first chunk)
    auto later = [&]() __attribute__((always_inline)) {
      if constexpr (NEXT) {
#pragma unroll
        for (int c = NC / 2; c < NC; ++c) kn[c] = k_frag(nt, nsub, c);
      }
      if constexpr (M32) {
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) vp[VF - 1][tt] = v_frag(pt, psub, tt, 1);
      }
    };
    bool gone = false;
    p_swap(pp);
    float cm = scale, ms = m_run;
    if (__builtin_expect(careful, 0)) {
#pragma clang fp contract(off)
      const float mx = query_max(sc);
      const bool up = raised(mx);
      const float mn = up ? lead(mx) : m_run;
      const float alpha = up ? __builtin_amdgcn_exp2f(m_run - mn) : 1.0f;
      // the probabilities of the previous half, not yet in O, are of the old max: they go
      // in here, and nothing below (zeros on both sides: 0 V would be a NaN where V is infinite)
      if (!first)
        static_for<0, NT>([&](auto tc) {
          constexpr int tt = decltype(tc)::value;
          pv(tc, std::integral_constant<int, 0>{}, vp[0][tt], pp[0]);
          pv(tc, std::integral_constant<int, 1>{}, M32 ? v_frag(pt, psub, tt, 1) : vp[0][tt], pp[1]);
        });
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pp[0][e] = pp[1][e] = (bf16)0.0f;
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) vp[0][tt][e] = (bf16)0.0f;
      }
      gone = true;
      m_run = mn;
      l_run *= alpha;
      rescale(alpha);
      const bool none = mn == -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float s = sc[r] * scale;
        sc[r] = none ? s : s - mn;
      }
      cm = 1.0f;
      ms = 0.0f;
      careful = needs_care();
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    static_for<0, 2>([&](auto cc) {
      constexpr int ci = decltype(cc)::value;
      constexpr int c0 = ci * NC / 2, c1 = (ci + 1) * NC / 2;
      constexpr int NSM = NEXT ? c1 - c0 : 0, NM = NSM + NT, NB = cmin(NSM, NT);
      static_for<0, NM>([&](auto gc) {
        constexpr int g = decltype(gc)::value;
        constexpr bool is_pv = g < 2 * NB ? g % 2 == 0 : NT > NSM;
        constexpr int idx = g < 2 * NB ? g / 2 : g - NB;
        if constexpr (is_pv)
          pv(std::integral_constant<int, idx>{}, cc, vp[M32 ? ci : 0][idx], pp[ci]);
        else
          sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kn[c0 + idx], qf[c0 + idx], c0 + idx == 0 ? zero16 : sn, 0, 0, 0);
        if constexpr (ci == 0 && g == 0) later();
        if constexpr (M32 && ci == 0 && g == NM - 1) {
          if (__builtin_expect(gone, 0)) {
#pragma unroll
            for (int tt = 0; tt < NT; ++tt)
#pragma unroll
              for (int e = 0; e < 8; ++e) vp[VF - 1][tt][e] = (bf16)0.0f;
          }
        }
        static_for<g * 4 / NM, (g + 1) * 4 / NM>([&](auto pc_) {
          constexpr int pr = decltype(pc_)::value;
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[e] = __builtin_amdgcn_exp2f(fmaf(sc[8 * ci + 2 * pr + e], cm, -ms));
            pc[ci][2 * pr + e] = (bf16)x[e];
          }
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      asm volatile("" ::"v"(pc[ci]));   // (keeps the exponentials here, between the MFMAs)
    });
    __builtin_amdgcn_s_setprio(0);
    // a probability of 2 or more, or not finite: bf16 exponent bit 7
    const u32x4 a = __builtin_bit_cast(u32x4, pc[0]), c = __builtin_bit_cast(u32x4, pc[1]);
    const unsigned any = a[0] | a[1] | a[2] | a[3] | c[0] | c[1] | c[2] | c[3];
    if (__builtin_expect(__any((any & 0x40004000u) != 0u), 0)) {
#pragma clang fp contract(off)
      // (a careful half is at or below its max: here for what is not finite, nothing to raise)
      const float mx = cm == scale ? query_max(sc) : -INFINITY;
      const bool up = raised(mx);
      const float mn = up ? lead(mx) : m_run;
      const float alpha = up ? __builtin_amdgcn_exp2f(m_run - mn) : 1.0f;
      m_run = mn;
      l_run *= alpha;
      rescale(alpha);
      if (up) ms = mn;
      const bool huge = !(fabsf(ms) <= 2 * kHuge);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = sc[8 * j + e] * cm;
          pc[j][e] = (bf16)__builtin_amdgcn_exp2f(huge ? s - ms : fmaf(sc[8 * j + e], cm, -ms));
        }
      careful = needs_care();
    }
    // the sum of the rounded probabilities, in fp32
    const bf16x2 one2 = {(bf16)1.0f, (bf16)1.0f};
    const u32x4 pa = __builtin_bit_cast(u32x4, pc[0]), pb = __builtin_bit_cast(u32x4, pc[1]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned x = pa[e], y = pb[e];
      l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), one2, l_run, false);
      l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, y), one2, l_run, false);
    }
  };
  // keys past the last: no score
  auto mask = [&](int t, int sub, f32x16& sc) __attribute__((always_inline)) {
    if (__builtin_expect((t + 1) * BKV > N, 0)) {
      const int left = N - t * BKV - 32 * sub - 8 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (16 * (r >> 3) + (r & 7) >= left) sc[r] = -INFINITY;
    }
  };

  // K has two stages, V two: after the barrier between the halves of tile t, K of tile
  // t + 2 takes the place of tile t's and V of t + 1 that of t - 1's; their loads were
  // issued a whole tile earlier, into registers.
  load_k(t0);
  load_v(t0);
  store_k(t0);
  store_v(t0);
  if (1 < NIT) {
    load_k(t0 + 1);
    load_v(t0 + 1);
    store_k(t0 + 1);
  }
  if (2 < NIT) load_k(t0 + 2);
  lds_sync();
  f32x16 s0, s1;
  s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(t0, 0, 0), qf[0], zero16, 0, 0, 0);
#pragma unroll
  for (int c = 1; c < NC; ++c) s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(t0, 0, c), qf[c], s0, 0, 0, 0);
  bf16x8 pa[2], pb[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) pa[j][e] = (bf16)0.0f;
  int t = t0;
  for (; t + 1 < t0 + NIT; ++t) {
    mask(t, 0, s0);
    step(std::true_type{}, t == t0, s0, t, 1, s1, t == t0 ? t : t - 1, t == t0 ? 0 : 1, pa, pb);
    lds_sync();
    if (t + 2 < t0 + NIT) store_k(t + 2);
    store_v(t + 1);
    if (t + 3 < t0 + NIT) load_k(t + 3);
    if (t + 2 < t0 + NIT) load_v(t + 2);
    mask(t, 1, s1);
    step(std::true_type{}, false, s1, t + 1, 0, s0, t, 0, pb, pa);
  }
  mask(t, 0, s0);
  step(std::true_type{}, t == t0, s0, t, 1, s1, t == t0 ? t : t - 1, t == t0 ? 0 : 1, pa, pb);
  mask(t, 1, s1);
  step(std::false_type{}, false, s1, 0, 0, s0, t, 0, pb, pa);
  p_swap(pa);
  static_for<0, NT>([&](auto tc) {
    pv(tc, std::integral_constant<int, 0>{}, v_frag(t, 1, decltype(tc)::value, 0), pa[0]);
    pv(tc, std::integral_constant<int, 1>{}, v_frag(t, 1, decltype(tc)::value, 1), pa[1]);
  });

  // a lane holds channels 32 t + 8 g + 4 h .. +4 of query lane & 31 (M32), or 16 t + 4 (lane >> 4)
  // .. +4 of queries 16 j + (lane & 15)
  l_run += __shfl_xor(l_run, 32, kWave);
  const bool whole = sp.ns == 1;
  auto put = [&](int ql, int c, float l, float x0, float x1, float x2, float x3) __attribute__((always_inline)) {
    const int q = q0 + ql;
    if (q >= p.n_q) return;
    if (whole) {
      const float inv = 1.0f / l;
      bf16x4 v = {(bf16)(x0 * inv), (bf16)(x1 * inv), (bf16)(x2 * inv), (bf16)(x3 * inv)};
      *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16*>(p.out) + ((size_t)b * p.n_q + q) * H + (size_t)head * D + c) = v;
    } else {
      *reinterpret_cast<f32x4*>(sp.part_o + (((size_t)unit * sp.ns + part) * (32 * NW) + 32 * wave + ql) * D + c) = f32x4{x0, x1, x2, x3};
    }
  };
  if constexpr (M32) {
#pragma unroll
    for (int tt = 0; tt < NT; ++tt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        put(lc, 32 * tt + 8 * g + 4 * h, l_run, oo[tt][4 * g], oo[tt][4 * g + 1], oo[tt][4 * g + 2], oo[tt][4 * g + 3]);
  } else {
    float lj[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) lj[j] = __shfl(l_run, 16 * j + i16, kWave);
#pragma unroll
    for (int f = 0; f < 2 * NT; ++f)
      if (16 * (f / 2) + 4 * g16 < D)
        put(16 * (f & 1) + i16, 16 * (f / 2) + 4 * g16, lj[f & 1], oo[f / 4][4 * (f % 4)], oo[f / 4][4 * (f % 4) + 1],
            oo[f / 4][4 * (f % 4) + 2], oo[f / 4][4 * (f % 4) + 3]);
  }
  if (!whole && h == 0 && q0 + lc < p.n_q)
    sp.part_ml[((size_t)unit * sp.ns + part) * (32 * NW) + 32 * wave + lc] = make_float2(m_run, l_run);
}

// ---------------------------------------------------------------------------
// fp32: v_mfma_f32_32x32x2_f32, 32 keys a tile.  Its two k are channels 8 g + e and 8 g + 4 + e of the
// scores, and keys 8 g + e and 8 g + 4 + e of the PV product, which score register 4 g + e holds in the two
// lane halves: the probabilities need no movement, and V is read token-major, 32 channels of a key by 32 lanes.
template <int D, int NW>
struct Geo32 {
  static constexpr int BK = 32, NG = D / 8, DT = (D + 31) / 32, CPT = D / 8, THREADS = 64 * NW;
  static constexpr int KP = 4 * D + 16;          // bytes of a K row: an odd number of 16-byte chunks
  static constexpr int VP = 128 * DT + 32;       // of a V row: four rows apart are the other 32 banks
  static constexpr int LDS = BK * (KP + VP);
  static constexpr int SL = (BK * CPT + THREADS - 1) / THREADS;
  static constexpr int WPC = cmin(8 / NW, 160 * 1024 / LDS);
};

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, NW == 1 ? 1 : 2) void attn_q8_f32_kernel(AttnQParams p, Split sp) {
#pragma clang fp contract(off)
  using G = Geo32<D, NW>;
  constexpr int SL = G::SL, CPT = G::CPT, TH = G::THREADS, BK = G::BK, DT = G::DT;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  char* sk = smem;
  char* sv = smem + BK * G::KP;
  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, h = lane >> 5, wave = tid >> 6;
  const int n_qt = (p.n_q + 32 * NW - 1) / (32 * NW);
  const int unit = blockIdx.x / sp.ns, part = blockIdx.x - unit * sp.ns;
  const int pair = unit / n_qt, q0 = (unit - pair * n_qt) * 32 * NW + 32 * wave;
  const int b = pair / p.heads, head = pair - b * p.heads;
  const int N = p.c.tokens, fb = p.fresh_begin, nf = p.n_fresh;
  const int nkt = (N + BK - 1) / BK;
  const int t0 = (int)((long long)nkt * part / sp.ns), t1 = (int)((long long)nkt * (part + 1) / sp.ns);
  const size_t H = (size_t)p.heads * D;
  const unsigned char* k8 = p.c.values + b * p.c.values_bs + (size_t)head * N * D;
  const unsigned char* v8 = p.c.values + b * p.c.values_bs + (size_t)(p.heads + head) * N * D;
  const unsigned char* ke = p.c.exps + b * p.c.exps_bs + (size_t)head * N;
  const unsigned char* ve = p.c.exps + b * p.c.exps_bs + (size_t)(p.heads + head) * N;
  const float *kf = nullptr, *vf = nullptr;
  if (nf > 0) {
    kf = reinterpret_cast<const float*>(p.kv_fresh) + b * p.fresh_bs + (size_t)head * nf * D;
    vf = reinterpret_cast<const float*>(p.kv_fresh) + b * p.fresh_bs + nf * H + (size_t)head * D * nf;
  }
  // V's padding channels: zero, never written again
  if constexpr (32 * DT > D)
    for (int i = tid; i < BK * (32 * DT - D); i += TH)
      *reinterpret_cast<float*>(sv + i / (32 * DT - D) * G::VP + (D + i % (32 * DT - D)) * 4) = 0.0f;

  // chunk i * TH + tid of a tile: channels 8 ch .. +8 of key `key`
  auto chunk = [&](int i, int& key, int& ch) {
    const int id = i * TH + tid;
    key = id / CPT;
    ch = id - key * CPT;
    return key < BK;
  };
  u32x4 kr[SL][2], vr[SL][2];
  auto wide = [](u32x2 x, unsigned e, u32x4(&r)[2]) {
    const float s = scale_of(e);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x[i], s, false);
      const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x[i], s, true);
      r[i] = u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(c[0]), __float_as_uint(c[1])};
    }
  };
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      int key, ch;
      if (!chunk(i, key, ch)) continue;
      const int n = t * BK + key, f = n - fb;
      kr[i][0] = kr[i][1] = vr[i][0] = vr[i][1] = u32x4{0, 0, 0, 0};
      if ((unsigned)f < (unsigned)nf) {
        const u32x4* src = reinterpret_cast<const u32x4*>(kf + (size_t)f * D + ch * 8);
        kr[i][0] = src[0];
        kr[i][1] = src[1];
        const float* col = vf + (size_t)ch * 8 * nf + f;
#pragma unroll
        for (int e = 0; e < 8; ++e) vr[i][e >> 2][e & 3] = __float_as_uint(col[(size_t)e * nf]);
      } else if (n < N) {
        wide(*reinterpret_cast<const u32x2*>(k8 + (size_t)n * D + ch * 8), ke[n], kr[i]);
        wide(*reinterpret_cast<const u32x2*>(v8 + (size_t)n * D + ch * 8), ve[n], vr[i]);
      }
    }
  };
  auto store = [&]() {
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      int key, ch;
      if (!chunk(i, key, ch)) continue;
      u32x4* dk = reinterpret_cast<u32x4*>(sk + key * G::KP + ch * 32);
      u32x4* dv = reinterpret_cast<u32x4*>(sv + key * G::VP + ch * 32);
      dk[0] = kr[i][0];
      dk[1] = kr[i][1];
      dv[0] = vr[i][0];
      dv[1] = vr[i][1];
    }
  };

  const int qrow = min(q0 + lc, p.n_q - 1);
  const float* qp = reinterpret_cast<const float*>(p.q) + (((size_t)b * p.heads + head) * p.n_q + qrow) * D;
  f32x4 qf[G::NG];
#pragma unroll
  for (int g = 0; g < G::NG; ++g) qf[g] = *reinterpret_cast<const f32x4*>(qp + 8 * g + 4 * h);
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  f32x16 oo[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) oo[t][r] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;

  load(t0);
  for (int t = t0; t < t1; ++t) {
    store();
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
    f32x16 sc = {};
#pragma unroll
    for (int g = 0; g < G::NG; ++g) {
      const f32x4 k = *reinterpret_cast<const f32x4*>(sk + lc * G::KP + 32 * g + 16 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[g][e], sc, 0, 0, 0);
    }
    // register r: key 8 (r / 4) + 4 h + r % 4
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = t * BK + 8 * (r >> 2) + 4 * h + (r & 3) < N ? sc[r] * scale : -INFINITY;
      mx = fmaxf(mx, sc[r]);
    }
    mx = max_xhalf(mx);
    // (the difference of rounded products: equal scores cancel at any size.  While no score is above minus
    // infinity the subtrahend is 0, and every probability 0)
    if (mx > m_run) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      m_run = mx;
      l_run *= alpha;
#pragma unroll
      for (int tt = 0; tt < DT; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oo[tt][r] *= alpha;
    }
    const float ms = m_run == -INFINITY ? 0.0f : m_run;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(sc[r] - ms);
      l_run += sc[r];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float* row = reinterpret_cast<const float*>(sv + (8 * (r >> 2) + 4 * h + (r & 3)) * G::VP) + lc;
#pragma unroll
      for (int tt = 0; tt < DT; ++tt)
        oo[tt] = __builtin_amdgcn_mfma_f32_32x32x2f32(row[32 * tt], sc[r], oo[tt], 0, 0, 0);
    }
    __syncthreads();
  }
  l_run += __shfl_xor(l_run, 32, kWave);
  if (q0 + lc >= p.n_q) return;
  const size_t slot = ((size_t)unit * sp.ns + part) * (32 * NW) + 32 * wave + lc;
  const float inv = sp.ns == 1 ? 1.0f / l_run : 1.0f;
  float* orow = sp.ns == 1 ? reinterpret_cast<float*>(p.out) + ((size_t)b * p.n_q + q0 + lc) * H + (size_t)head * D
                           : sp.part_o + slot * D;
#pragma unroll
  for (int tt = 0; tt < DT; ++tt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * tt + 8 * g + 4 * h;
      if (c < D) *reinterpret_cast<f32x4*>(orow + c) = f32x4{oo[tt][4 * g] * inv, oo[tt][4 * g + 1] * inv, oo[tt][4 * g + 2] * inv, oo[tt][4 * g + 3] * inv};
    }
  if (sp.ns > 1 && h == 0) sp.part_ml[slot] = make_float2(m_run, l_run);
}

// The parts of a query tile whose keys ns workgroups shared: O = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s
// - m) l_s, m = max_s m_s.  A thread per 4 channels of a query, the parts in their order.
template <typename T>
__global__ __launch_bounds__(256) void attn_q8_merge_kernel(AttnQParams p, Split sp, int rows) {
  const int quads = p.d / 4, n_qt = (p.n_q + rows - 1) / rows;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long query = i / quads;                 // (branch, head, query)
  const int c = 4 * (int)(i - query * quads);
  if (query >= (long long)p.B * p.heads * p.n_q) return;
  const int pair = (int)(query / p.n_q), q = (int)(query - (long long)pair * p.n_q);
  const size_t slot = ((size_t)pair * n_qt + q / rows) * sp.ns * rows + q % rows;
  const float2* ml = sp.part_ml + slot;
  const float* po = sp.part_o + slot * p.d + c;
  float m = -INFINITY;
  for (int s = 0; s < sp.ns; ++s) m = fmaxf(m, ml[(size_t)s * rows].x);
  float l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  for (int s = 0; s < sp.ns; ++s) {
    const float2 x = ml[(size_t)s * rows];
    const float f = __builtin_amdgcn_exp2f(x.x - m);
    const f32x4 y = *reinterpret_cast<const f32x4*>(po + (size_t)s * rows * p.d);
    l = fmaf(f, x.y, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(f, y[e], o[e]);
  }
  const float inv = 1.0f / l;
  typedef T quad __attribute__((ext_vector_type(4)));
  quad v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = from_f<T>(o[e] * inv);
  const int b = pair / p.heads, head = pair - b * p.heads;
  *reinterpret_cast<quad*>(reinterpret_cast<T*>(p.out) + ((size_t)b * p.n_q + q) * p.heads * p.d + (size_t)head * p.d + c) = v;
}

// ---------------------------------------------------------------------------
// Waves of a workgroup by the number of queries, and workgroups that share a query tile's keys: the ns
// that minimises the rounds of resident workgroups times a workgroup's key tiles (and two more for
// its start), with the merge's cost where ns > 1.
struct Plan {
  int nw, ns;
  size_t tiles;
};

constexpr int few_waves(int d, bool f32) { return !f32 && d <= 80 ? 1 : 2; }

template <typename G>
Plan plan_geo(int nw, int bk, int B, int heads, int n_q, int n_kv) {
  const long long tiles = (long long)ceil_div(n_q, 32 * nw) * heads * B, slots = 256 * G::WPC;
  const int nkt = ceil_div(n_kv, bk);
  int best = 1;
  double cost = 1e300;
  for (int ns = 1; ns <= nkt && ns <= 64; ++ns) {
    const double rounds = (double)((tiles * ns + slots - 1) / slots);
    const double c = rounds * (ceil_div(nkt, ns) + 2.0) + (ns > 1 ? 6.0 : 0.0);
    if (c < cost) {
      cost = c;
      best = ns;
    }
  }
  return {nw, best, (size_t)tiles};
}

template <typename F>
void with_d(int d, F&& f) {
  switch (d) {
    case 32: f(std::integral_constant<int, 32>{}); break;
    case 64: f(std::integral_constant<int, 64>{}); break;
    case 72: f(std::integral_constant<int, 72>{}); break;
    case 80: f(std::integral_constant<int, 80>{}); break;
    case 96: f(std::integral_constant<int, 96>{}); break;
    case 128: f(std::integral_constant<int, 128>{}); break;
  }
}

// f(dimension, waves) with both as constants
template <typename F>
void with_shape(int d, int n_q, int dtype, F&& f) {
  with_d(d, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    if (n_q > 64) f(dc, std::integral_constant<int, 4>{});
    else if (dtype == kBF16) f(dc, std::integral_constant<int, few_waves(D, false)>{});
    else f(dc, std::integral_constant<int, few_waves(D, true)>{});
  });
}

Plan plan(int B, int heads, int n_q, int n_kv, int d, int dtype) {
  Plan r{0, 1, 0};
  with_shape(d, n_q, dtype, [&](auto dc, auto nc) {
    constexpr int D = decltype(dc)::value, NW = decltype(nc)::value;
    if (dtype == kBF16) {
      if constexpr (NW == 4 || NW == few_waves(D, false)) r = plan_geo<Geo<D, NW>>(NW, BKV, B, heads, n_q, n_kv);
    } else if constexpr (NW == 4 || NW == few_waves(D, true)) {
      r = plan_geo<Geo32<D, NW>>(NW, Geo32<D, NW>::BK, B, heads, n_q, n_kv);
    }
  });
  return r;
}

size_t part_floats(const Plan& pl, int d) { return pl.tiles * pl.ns * 32 * pl.nw * d; }

template <typename K>
hipError_t launch(K kern, int lds, int threads, size_t groups, const AttnQParams& p, const Split& sp, hipStream_t s) {
  hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(threads), lds, s, p, sp);
  return hipGetLastError();
}

}  // namespace q8attn

size_t attention_quantized_workspace_bytes(int B, int heads, int n_q, int n_kv, int d, int dtype) {
  using namespace q8attn;
  if (n_q <= 0) return 0;
  const Plan pl = plan(B, heads, n_q, n_kv, d, dtype);
  if (pl.nw == 0 || pl.ns == 1) return 0;
  return part_floats(pl, d) * 4 + pl.tiles * pl.ns * 32 * pl.nw * sizeof(float2);
}

hipError_t launch_attention_quantized(const AttnQParams& p, int dtype, hipStream_t s) {
  using namespace q8attn;
  if (p.n_q <= 0) return hipSuccess;
  Plan pl = plan(p.B, p.heads, p.n_q, p.c.tokens, p.d, dtype);
  if (pl.nw == 0) return hipErrorInvalidValue;
  if (!p.ws) pl.ns = 1;
  if (pl.tiles * pl.ns > 0x7fffffff) return hipErrorInvalidValue;
  Split sp{pl.ns, nullptr, nullptr};
  if (pl.ns > 1) {
    sp.part_o = reinterpret_cast<float*>(p.ws);
    sp.part_ml = reinterpret_cast<float2*>(sp.part_o + part_floats(pl, p.d));
  }
  hipError_t rc = hipErrorInvalidValue;
  with_shape(p.d, p.n_q, dtype, [&](auto dc, auto nc) {
    constexpr int D = decltype(dc)::value, NW = decltype(nc)::value;
    if (dtype == kBF16) {
      if constexpr (NW == 4 || NW == few_waves(D, false)) {
        constexpr int lds = Geo<D, NW>::LDS;
        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_q8_kernel<D, NW>),
                                                           hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        rc = attr != hipSuccess ? attr : launch(attn_q8_kernel<D, NW>, lds, 64 * NW, pl.tiles * pl.ns, p, sp, s);
      }
    } else if constexpr (NW == 4 || NW == few_waves(D, true)) {
      rc = launch(attn_q8_f32_kernel<D, NW>, Geo32<D, NW>::LDS, 64 * NW, pl.tiles * pl.ns, p, sp, s);
    }
  });
  if (rc != hipSuccess || pl.ns == 1) return rc;
  const size_t threads = (size_t)p.B * p.heads * p.n_q * (p.d / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (dtype == kBF16) hipLaunchKernelGGL(attn_q8_merge_kernel<bf16>, grid, dim3(256), 0, s, p, sp, 32 * pl.nw);
  else hipLaunchKernelGGL(attn_q8_merge_kernel<float>, grid, dim3(256), 0, s, p, sp, 32 * pl.nw);
  return hipGetLastError();
}

}  // namespace orch
