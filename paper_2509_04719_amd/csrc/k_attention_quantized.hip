// Attention of a band's queries over the whole image, K/V of the band's own tokens
// fresh (operand type) and of every other token in the 8-bit cache.
//
// O = softmax(Q K^T / sqrt d) V in one pass over the keys, with a running max and sum.  Scores are formed transposed,
// S^T = K Q^T, so that a lane owns one query column and its max and sum stay in the lane; 32 queries a wave, 64 keys a
// tile (32 in fp32).  The cache's bytes are widened to the operand type on their way to LDS (exact: e4m3 times a
// power of two is a bf16 number), and the band's own keys take the place of the cache's there.  Matrix products in 8
// bits would need Q and the probabilities in 8 bits too.
//
// The bf16 products take a probability as two bf16, p = hi + lo, two MFMAs for each V fragment: 16 significant bits of
// it, so that the output's rounding is the only error that shows (2-norm against 64 bits 1.66e-3, as in 32 bits
// throughout).  Rounded to one bf16 it would be 2.33e-3; the second term and its products cost 92 -> 117 us at 1664
// queries x 4096 keys and 937 -> 1300 at 6144 x 16384 (2 x 16 heads of 72), 16 -> 19 at 384 x 1024.
//
// Bound by the matrix cores with many queries (4 B heads n_q n_kv d flops), else by a wave's own chain: widening a
// key costs the VALU as much as a wave's softmax of it, and VALU and MFMA instructions of a SIMD do not overlap
// freely.  So there are four forms, chosen by an estimate of their time (`plan` below):
//   prepared    many queries: the keys are widened once, fresh and cached together, into tiles in the workspace, and
//               four waves of 32 queries load each tile straight to LDS.  d = 72, 2 x 16 heads: 6144 queries x
//               16384 keys 1300-1370 us (677-714 TFLOP/s, every product counted once; 51 of it preparing), 1664 x 4096
//               117-122 us; d = 128, 2 x 8 heads, 4096 x 4096 185 us (743).
//   NW = 4      without a workspace, or too few queries to pay for it: four waves of 32 queries share each tile, each
//               widens a quarter of it.  1664 x 1024 keys 43 us; d = 128, 2 x 8 heads, 45 x 2025, keys split 12 ways:
//               14.6 us and 5 for the parts.
//   NW = 1      few queries: four waves have the same 32 queries and each a quarter of the keys, without a barrier,
//               K from memory straight to the products' operand (through LDS: 4% longer at d = 72, 20% at 80 to 128).
//               384 x 1024 keys 17.5 us, 384 x 4096 45; one query x 16384 keys of 8 heads of 72 13.4 with its parts.
//   fp32        the same on v_mfma_f32_32x32x2: 512 x 1024 keys, 4 heads of 32: 8.5 us.
// With a workspace each may also split the keys of a query tile over workgroups; a merge kernel joins the parts.
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

// 2^(byte - 127).  (As a shift in C the compiler keeps the bytes of the tile in flight as 16 bits, widens
// them at the end of the loop that loads them, and waits for the loads there.)
__device__ __forceinline__ float scale_of(unsigned byte) {
  float r;
  asm("v_lshlrev_b32 %0, 23, %1" : "=v"(r) : "v"(byte));
  return r;
}

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
// bf16.  A workgroup is four waves.  NW = 4: each has 32 queries, and they share every tile of
// keys.  NW = 1: all have the same 32 queries, and each takes every key tile of a quarter of the
// keys alone, without a barrier; their parts meet in LDS at the end.  (Few queries leave
// most SIMDs without a wave otherwise, and a wave's own chain is what bounds it.)
template <int D, int NW, bool PREP = false>
struct Geo {
  static constexpr int KG = 4 / NW;              // key groups
  static constexpr int NC = (D + 15) / 16;       // 16-channel chunks of a score
  static constexpr bool M32 = D % 32 == 0;       // PV on 32x32x16, else on 16x16x32
  static constexpr int NT = M32 ? D / 32 : NC;   // row tiles of O^T
  static constexpr int CPT = D / 8;              // 8-channel chunks of a token
  // bytes of a K row, an odd number of 16-byte chunks; PREP: without padding channels; NW = 1 keeps no K in LDS
  static constexpr int KP = NW == 1 ? 0 : PREP ? (CPT | 1) * 16 : NC * 32 + 16;
  // of a V row: an odd multiple of 32 (16-row reads) or 64 (32-row reads)
  static constexpr int VP = !M32 ? NC * 32 : D * 2 % 128 == 64 ? D * 2 : D * 2 + 64;
  // PREP: tiles as they lie in memory, KT bytes of K rows, then VT of V^T rows
  static constexpr int KT = BKV * KP, VT = PREP ? (M32 ? D : 16 * NT) * 128 : BKV * VP;
  static constexpr int ZERO = PREP && D % 16 ? 1024 : 0;   // zeros behind a K stage: channels past the last
  static constexpr bool ONES = PREP && !M32 && 16 * NT > D;        // row D of V^T is ones: O^T's row D is the sum
  static constexpr int ST = NW == 4 ? 2 : 1;     // stages: a wave alone needs no second one
  static constexpr int KS = KT + ZERO;           // a K stage
  static constexpr int NO = M32 ? NT : (2 * NT + 3) / 4;           // 16-register blocks of O^T
  // (a group's part takes its tile's place)
  static constexpr int GROUP = cmax(ST * (KS + VT), KG > 1 ? (NO * 16 + 2) * 256 : 0);
  static_assert(KS % 128 == 0 && VT % 128 == 0, "the swizzle of V^T rows is an XOR of the address");
  static constexpr int LDS = KG * GROUP;
  static constexpr int THREADS = 64 * NW;        // that share a tile
  static constexpr int SL = (BKV * CPT + THREADS - 1) / THREADS;   // chunks of a thread, K and V each
  static constexpr int WPE = NW == 1 && D == 128 ? 1 : PREP && D <= 80 ? 3 : 2;          // waves of a SIMD that registers allow
  static constexpr int WPC = cmin(WPE, 160 * 1024 / LDS);          // workgroups of a CU
  static constexpr bool EVEN = THREADS % CPT == 0;                 // a thread's chunks are THREADS / CPT keys apart
  // NW = 1: V's lanes of a key, each with CPL chunks in a row, keys 64 / LPK apart
  static constexpr int LPK = D == 128 ? 4 : D == 64 || D == 80 || D == 96 ? 2 : 1;
  static constexpr int CPL = CPT / LPK;
  static constexpr int NE = NW == 1 ? LPK : SL;  // scales of a thread
  static constexpr bool AHEAD = NW == 4 && !PREP && D <= 96;       // tiles of fresh keys alone are fetched ahead too
};

struct Split {
  const char* tiles; // prepared tiles, [branch, head][key tile] of KT + VT bytes
  int ns;            // workgroups that share a query tile's keys
  float* part_o;     // fp32 [tiles * ns][32 NW][D], unnormalised
  float2* part_ml;   // (max, sum)
};

template <int D, int NW, bool PREP>
__global__ __launch_bounds__(256, (Geo<D, NW, PREP>::WPE)) void attn_q8_kernel(AttnQParams p, Split sp) {
  // (the body uses device-only types; the host pass only needs the launch stub)
#if defined(__HIP_DEVICE_COMPILE__)
  using G = Geo<D, NW, PREP>;
  constexpr int NC = G::NC, NT = G::NT, SL = G::SL, CPT = G::CPT, TH = G::THREADS, KG = G::KG;
  constexpr bool M32 = G::M32;
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  const int lane = threadIdx.x & 63, lc = lane & 31, h = lane >> 5;
  const int i16 = lane & 15, g16 = lane >> 4;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = KG == 1 ? 0 : wave_all, wave = KG == 1 ? wave_all : 0;
  const int tid = KG == 1 ? threadIdx.x : lane;          // of the threads that share a tile
  char* smem = smem_all + kg * G::GROUP;

  // workgroups in the order (branch, head, query tile, split); an eighth of them in a row on
  // each XCD, so that those that read the same K/V share an L2
  const int n_qt = (p.n_q + 32 * NW - 1) / (32 * NW);
  const int NWG = gridDim.x;
  int w = blockIdx.x;
  if (w < NWG / 8 * 8) w = (w & 7) * (NWG / 8) + (w >> 3);
  const int unit = w / sp.ns, part = w - unit * sp.ns;
  const int pair = unit / n_qt, q0 = (unit - pair * n_qt) * 32 * NW + 32 * wave;
  const int b = pair / p.heads, head = pair - b * p.heads;
  const int N = p.c.tokens, nf = p.n_fresh, fb = nf > 0 ? p.fresh_begin : 0;
  const int nkt = (N + BKV - 1) / BKV;
  const int shares = sp.ns * KG, share = part * KG + kg;
  const int t0 = (int)((long long)nkt * share / shares), te = (int)((long long)nkt * (share + 1) / shares);
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

  // K rows' padding channels [D, 16 NC): zero, never written again (Q's are zero too; V's may
  // hold anything, they end in rows of O^T that nobody reads)
  if constexpr (G::ZERO > 0) {
    if (tid < G::ST) *reinterpret_cast<u32x4*>(smem + tid * G::KS + G::KT) = u32x4{0, 0, 0, 0};
  } else if constexpr (NW == 4 && D % 16 != 0) {
    for (int i = tid; i < G::ST * BKV; i += TH)
      *reinterpret_cast<u32x4*>(smem + (i / BKV) * G::KS + (i % BKV) * G::KP + 2 * D) = u32x4{0, 0, 0, 0};
  }

  // Staging.  A tile of 64 tokens is contiguous in the cache: chunk id (8 channels) of key
  // id / CPT.  Key k of the tile goes to K row k, and to V row vrow(k): the transposing reads
  // below take keys 8 g + 4 x + r, r = 0 .. 3, of several g at once, which then lie in
  // consecutive rows.  A tile of fresh keys alone keeps V^T as it is, rows of 64 keys with
  // their 16-byte chunks swizzled by row.
  auto vrow = [](int k) __attribute__((always_inline)) { return (k & 32) | (k & 4) << 2 | (k & 24) >> 1 | (k & 3); };
  constexpr int KS = TH / CPT;                              // EVEN: keys from slot to slot
  static_assert(NW == 1 || !G::EVEN || (KS & (KS - 1)) == 0, "a slot's rows are a constant away");
  // V of a wave alone: LPK lanes for each key, with CPL neighbouring chunks: few scales a lane, rows a
  // constant apart, at the price of loads that touch more lines of the tile than they take from them.
  constexpr bool ROW = NW == 1;
  constexpr int LPK = G::LPK, CPL = G::CPL, KR = 64 / LPK;  // ROW: keys between a lane's rows
  const int vtid = (NW - 1 - wave) * 64 + lane;             // V's chunks from the last wave down
  constexpr int NA = ROW || G::EVEN ? 1 : SL;
  int k_dst_[NA], v_dst_[NA], kkey_[NA], vkey_[NA];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int idk = ROW ? lane * CPL : i * TH + tid, keyk = idk / CPT, idv = ROW ? idk : i * TH + vtid, keyv = idv / CPT;
    kkey_[i] = keyk;
    vkey_[i] = keyv;
    k_dst_[i] = keyk * G::KP + (idk - keyk * CPT) * 16;
    v_dst_[i] = G::ST * G::KS + vrow(keyv) * G::VP + (idv - keyv * CPT) * 16;
  }
  auto key_of = [&](auto isk_c, int i) __attribute__((always_inline)) {
    const int* k = decltype(isk_c)::value ? kkey_ : vkey_;
    return ROW ? k[0] + i / CPL * KR : G::EVEN ? k[0] + i * KS : k[i];
  };
  auto chunk_of = [&](auto isk_c, int i) __attribute__((always_inline)) {
    return ROW ? lane % LPK * CPL + i % CPL : i * TH + (decltype(isk_c)::value ? tid : vtid) - key_of(isk_c, i) * CPT;
  };
  auto k_dst = [&](int i) __attribute__((always_inline)) { return G::EVEN ? k_dst_[0] + i * KS * G::KP : k_dst_[i]; };
  auto v_dst = [&](int i) __attribute__((always_inline)) { return ROW ? v_dst_[0] + vrow(i / CPL * KR) * G::VP + i % CPL * 16 : G::EVEN ? v_dst_[0] + vrow(i * KS) * G::VP : v_dst_[i]; };
  // fresh V^T: slot i holds chunk vtid % 8 (8 keys) of channel vtid / 8 + i TH / 8
  const unsigned vt_src = 2u * ((unsigned)(vtid >> 3) * (unsigned)nf + (vtid & 7) * 8);     // bytes, below 2^32
  const int vt_dst_ = G::ST * G::KS + (vtid >> 3) * 128 + ((vtid & 7) ^ ((vtid >> 4) & 7)) * 16;
  auto vt_dst = [&](int i) __attribute__((always_inline)) {
    return (TH % 128 == 0 || i % 2 == 0 ? vt_dst_ : vt_dst_ ^ 64) + i * TH * 16;   // (64 threads: 8 rows on, 4 in the swizzle)
  };
  // the last slot is some waves' alone: the first ones take K's chunks, the last ones V's
  constexpr int LEFT = (BKV * CPT % TH) / 64;
  static_assert(BKV * CPT % 64 == 0, "whole waves");
  auto on = [&](auto isk_c, int i) __attribute__((always_inline)) {
    return LEFT == 0 || i + 1 < SL || (decltype(isk_c)::value ? wave < LEFT : wave >= NW - LEFT);
  };

  enum { kStale = 0, kFresh = 1, kMixed = 2 };
  auto type_of = [&](int t) __attribute__((always_inline)) {
    const int n0 = t * BKV, n1 = n0 + BKV;
    if (n1 <= N && (n1 <= fb || n0 >= fb + nf)) return (int)kStale;
    return n0 >= fb && n1 <= fb + nf ? (int)kFresh : (int)kMixed;
  };
  // What a thread holds of a tile on its way: the cache's chunks and exponents, read of every tile
  // (unused where the keys are fresh: a load under a branch costs register moves, and those a
  // wait for the load), and the fresh keys' chunks of a tile of these alone.
  struct Raw {
    u32x2 x[SL];
    unsigned e[G::NE];
    u32x4 f[G::AHEAD ? SL : 1];
  };
  // buffers of the cache's and the fresh K's head: one 32-bit offset a lane for every load, zero past the last key
  const __amdgpu_buffer_rsrc_t rk8 = buffer_rsrc(k8, (size_t)N * D), rv8 = buffer_rsrc(v8, (size_t)N * D);
  const __amdgpu_buffer_rsrc_t rke = buffer_rsrc(ke, N), rve = buffer_rsrc(ve, N);
  const __amdgpu_buffer_rsrc_t rkf = buffer_rsrc(nf > 0 ? (const void*)kf : k8, nf > 0 ? (size_t)nf * D * 2 : 0);
  auto load_fresh = [&](auto isk_c, int t, int i) __attribute__((always_inline)) {
    if constexpr (decltype(isk_c)::value) {
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rkf, tid * 16, (unsigned)(t * BKV - fb) * (2u * D) + i * TH * 16, 0));
    } else {
      // (rows of V^T start at any element)
      const char* base = reinterpret_cast<const char*>(vf + (t * BKV - fb) + (size_t)i * (TH / 8) * nf);
      const u32x4_u x = *reinterpret_cast<const u32x4_u*>(base + vt_src);
      return u32x4{x[0], x[1], x[2], x[3]};
    }
  };
  auto load = [&](auto isk_c, Raw& r, int t, int type) __attribute__((always_inline)) {
    constexpr bool isk = decltype(isk_c)::value;
    const __amdgpu_buffer_rsrc_t rx = isk ? rk8 : rv8, re = isk ? rke : rve;
    if constexpr (ROW) {
#pragma unroll
      for (int j = 0; j < LPK; ++j) {
        const int so = t * BKV * D + j * KR * D;
#pragma unroll
        for (int c = 0; c < CPL; c += 2) {
          const int i = j * CPL + c;
          if (c + 1 < CPL) {
            const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, (lane * CPL + c) * 8, so, 0));
            r.x[i] = u32x2{x[0], x[1]};
            r.x[cmin(i + 1, SL - 1)] = u32x2{x[2], x[3]};
          } else {
            r.x[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, (lane * CPL + c) * 8, so, 0));
          }
        }
        r.e[j] = __builtin_amdgcn_raw_buffer_load_b8(re, lane / LPK, t * BKV + j * KR, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < SL; ++i) {
        // (a last slot that is not this wave's reads nothing)
        const int off = on(isk_c, i) ? 0 : 0x7fffffff - BKV * D;
        r.x[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, (isk ? tid : vtid) * 8 + off, t * BKV * D + i * TH * 8, 0));
        r.e[i] = __builtin_amdgcn_raw_buffer_load_b8(re, key_of(isk_c, i), t * BKV, 0);
      }
    }
    if constexpr (G::AHEAD)
      if (type == kFresh) {
#pragma unroll
        for (int i = 0; i < SL; ++i)
          if (on(isk_c, i)) r.f[i] = load_fresh(isk_c, t, i);
      }
  };
  auto widen = [](unsigned x0, unsigned x1, unsigned e) __attribute__((always_inline)) {
    const float s = scale_of(e);
    u32x4 r;
    r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, s, false));
    r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, s, true));
    r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, s, false));
    r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, s, true));
    return r;
  };
  auto store = [&](auto isk_c, const Raw& r, int t, int type) __attribute__((always_inline)) {
    constexpr bool isk = decltype(isk_c)::value;
    char* dst = smem + (G::ST == 2 ? t & 1 : 0) * (isk ? G::KS : G::VT);
    auto chunk = [&](int i) __attribute__((always_inline)) {
      return widen(r.x[i][0], r.x[i][1], r.e[ROW ? i / CPL : i]);
    };
    auto at = [&](int i) __attribute__((always_inline)) { return reinterpret_cast<u32x4*>(dst + (isk ? k_dst(i) : v_dst(i))); };
    if (type == kStale) {
#pragma unroll
      for (int i = 0; i < SL; ++i)
        if (on(isk_c, i)) *at(i) = chunk(i);
      return;
    }
    if (type == kFresh) {
      constexpr int BATCH = G::AHEAD ? SL : cmin(SL, NW == 4 || D == 80 || D == 96 ? 4 : D == 72 ? 9 : 6);
#pragma unroll
      for (int i0 = 0; i0 < SL; i0 += BATCH) {
        u32x4 x[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
          if (i0 + k < SL && on(isk_c, i0 + k)) {
            if constexpr (G::AHEAD) x[k] = r.f[i0 + k];
            else x[k] = load_fresh(isk_c, t, i0 + k);
          }
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
          if (i0 + k < SL && on(isk_c, i0 + k))
            *reinterpret_cast<u32x4*>(dst + (isk ? k_dst(i0 + k) : vt_dst(i0 + k))) = x[k];
      }
      return;
    }
    // a tile that the band's edge or the last key crosses (past it the loads gave zeros): the
    // cache's keys, then the fresh ones, K's in rows, V's along the keys
    const int n0 = t * BKV;
    auto fresh = [&](int key) __attribute__((always_inline)) { return (unsigned)(n0 + key - fb) < (unsigned)nf; };
    constexpr int BATCH = cmin(SL, NW == 4 ? 2 : D == 128 ? 16 : D <= 72 ? 9 : 4);
#pragma unroll
    for (int i0 = 0; i0 < SL; i0 += BATCH) {
      u32x4 x[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int i = cmin(i0 + k, SL - 1);
        x[k] = chunk(i);
        if (isk && i0 + k < SL && on(isk_c, i) && fresh(key_of(isk_c, i)))
          x[k] = *reinterpret_cast<const u32x4*>(kf + (size_t)(n0 + key_of(isk_c, i) - fb) * D + chunk_of(isk_c, i) * 8);
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int i = cmin(i0 + k, SL - 1);
        if (i0 + k < SL && on(isk_c, i) && (isk || !fresh(key_of(isk_c, i)))) *at(i) = x[k];
      }
    }
    if (!isk && n0 + BKV > fb && n0 < fb + nf) {
      // chunk id: channel id / 8, keys 8 (id % 8) .. +8.  Its fresh keys come from eight elements of the channel's row
      // that lie in the band (all of it where it has fewer), element j of them key j + shift of the chunk.
      const int kc = 8 * (vtid & 7), f = n0 + kc - fb, first = min(max(f, 0), max(nf - 8, 0)), shift = first - f;
      const bool some = f > -8 && f < nf;
      unsigned short* col = reinterpret_cast<unsigned short*>(dst + G::ST * G::KS + vrow(kc) * G::VP) + (vtid >> 3);
#pragma unroll
      for (int i0 = 0; i0 < SL; i0 += BATCH) {
        u32x4 x[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const int i = cmin(i0 + k, SL - 1);
          const unsigned short* src = reinterpret_cast<const unsigned short*>(vf) + (size_t)((vtid >> 3) + i * (TH / 8)) * nf + first;
          if (some && i0 + k < SL && on(isk_c, i)) {
            if (nf >= 8) {
              const u32x4_u y = *reinterpret_cast<const u32x4_u*>(src);
              x[k] = u32x4{y[0], y[1], y[2], y[3]};
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) x[k][e] = src[min(2 * e, nf - 1)] | (unsigned)src[min(2 * e + 1, nf - 1)] << 16;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = j + shift;
          unsigned short* to = col + ((key & 4) << 2 | (key & 3)) * (G::VP / 2);
          if (some && (unsigned)key < 8u && j < nf) {
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
              const int i = cmin(i0 + k, SL - 1);
              if (i0 + k < SL && on(isk_c, i)) to[i * (TH / 8)] = (unsigned short)(x[k][j >> 1] >> (16 * (j & 1)));
            }
          }
        }
      }
    }
  };
  constexpr std::true_type kK{};
  constexpr std::false_type kV{};
  // prepared tiles: straight to LDS, 1 KB a wave and load, K's from the first wave on, V's from the last
  const __amdgpu_buffer_rsrc_t rt = buffer_rsrc(PREP ? (const void*)(sp.tiles + (size_t)pair * nkt * (G::KT + G::VT)) : k8,
                                                PREP ? (size_t)nkt * (G::KT + G::VT) : 0);
  auto issue = [&](auto isk_c, int t) __attribute__((always_inline)) {
    constexpr bool isk = decltype(isk_c)::value;
    constexpr int NL = (isk ? G::KT : G::VT) / 1024;
    char* dst = smem + (isk ? (t & 1) * G::KS : 2 * G::KS + (t & 1) * G::VT);
    const int so = t * (G::KT + G::VT) + (isk ? 0 : G::KT);
#pragma unroll
    for (int i = 0; i < (NL + 3) / 4; ++i) {
      const int j = 4 * i + (isk ? wave : 3 - wave);
      if (NL % 4 == 0 || i + 1 < (NL + 3) / 4 || j < NL)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rt, (ORCH_LDS void*)(dst + j * 1024), 16, lane * 16, so + j * 1024, 0, 0);
    }
  };
  // the wave's loads and LDS operations done, then the workgroup's barrier
  auto tiles_wait = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // K of a wave alone goes straight to the A operand: lane (lc, h) reads half of the channels of key kperm(lc) of a half
  // tile, 8 a chunk, from channel 8 NC h on (the order of the products' channels is free), and widens them there.  Fresh
  // keys take the place of the cache's in their lanes.
  struct KHalf {
    u32x2 x[NC];
    unsigned e;
  };
  const int kd_key = kperm(lc), kd_off = kd_key * D + h * 8 * NC;
  auto k_load = [&](KHalf& r, int t, int sub) __attribute__((always_inline)) {
    const int so = (t * BKV + 32 * sub) * D;
#pragma unroll
    for (int c = 0; c < NC; c += 2) {
      if (c + 1 < NC) {
        const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk8, kd_off + 8 * c, so, 0));
        r.x[c] = u32x2{x[0], x[1]};
        r.x[cmin(c + 1, NC - 1)] = u32x2{x[2], x[3]};
      } else {
        r.x[c] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rk8, kd_off + 8 * c, so, 0));
      }
    }
    r.e = __builtin_amdgcn_raw_buffer_load_b8(rke, kd_key, t * BKV + 32 * sub, 0);
  };
  auto k_make = [&](const KHalf& r, int t, int sub, int type, bf16x8(&k)[NC]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      u32x2 x = r.x[c];
      // (the upper half's last chunk is past the channels: it read the next key's)
      if (CPT % 2 && c == NC - 1) x = h ? u32x2{0, 0} : x;
      k[c] = __builtin_bit_cast(bf16x8, widen(x[0], x[1], r.e));
    }
    if (type != kStale) {
      const int key = t * BKV + 32 * sub + kd_key - fb;
      if ((unsigned)key < (unsigned)nf) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          // (at the last chunk of the upper half: no scale of the cache's either)
          if (CPT % 2 && c == NC - 1 && h) k[c] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
          else k[c] = *reinterpret_cast<const bf16x8*>(kf + (size_t)key * D + h * 8 * NC + 8 * c);
        }
      }
    }
  };

  // this lane's query (B operand): channels 16 c + 8 h .. +8, or as K's
  const int qrow = min(q0 + lc, p.n_q - 1);
  const bf16* qp = reinterpret_cast<const bf16*>(p.q) + (((size_t)b * p.heads + head) * p.n_q + qrow) * D;
  bf16x8 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int ch = ROW ? 8 * (NC * h + c) : 16 * c + 8 * h;
    if (ch < D) {
      qf[c] = *reinterpret_cast<const bf16x8*>(qp + ch);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[c][e] = (bf16)0.0f;
    }
  }
  const float scale = 1.4426950408889634f / sqrtf((float)D);   // log2(e) / sqrt(d)

  // fragment reads: K row of key 32 sub + kperm(lc), chunk 2 c + h; V rows by the transposing
  // read (lane i of 16 points at four channels of row i / 4 and gets channel i of the four rows)
  const int k_rd = kperm(lc) * G::KP + 16 * h;
  const int v_rd = G::ST * G::KS + (M32 ? (4 * h + (i16 >> 2)) * G::VP + (g16 & 1) * 32 : (4 * g16 + (i16 >> 2)) * G::VP) + (i16 & 3) * 8;
  auto k_frag = [&](int t, int sub, int c) __attribute__((always_inline)) {
    // (trimmed rows end with channel D: the last chunk's upper half reads zeros)
    int at = sub * 32 * G::KP + k_rd + 32 * c;
    if constexpr (G::ZERO > 0)
      if (c == NC - 1) at = h ? G::KT : at;
    return *reinterpret_cast<const bf16x8*>(smem + (G::ST == 2 ? t & 1 : 0) * G::KS + at);
  };
  // O^T tile tt; M32: keys 16 ci .. +16 of the half, else all its 32.  vt: the tile holds V^T rows
  const int vt_row = M32 ? lc : i16;
  const int vt_rd[2] = {G::ST * G::KS + vt_row * 128 + ((M32 ? h : g16) ^ ((vt_row >> 1) & 7)) * 16,
                        G::ST * G::KS + vt_row * 128 + (((M32 ? h : g16) ^ ((vt_row >> 1) & 7)) ^ (M32 ? 2 : 4)) * 16};
  auto vt_frag = [&](int t, int sub, int tt, int ci) __attribute__((always_inline)) {
    // (the chunk's number 4 sub + 2 ci + h, or 4 sub + lane / 16, is swizzled by row; M32's 4 sub is an XOR of
    // the address by 64)
    const char* base = smem + (G::ST == 2 ? t & 1 : 0) * G::VT;
    if constexpr (M32) return *reinterpret_cast<const bf16x8*>(base + (vt_rd[ci] ^ (64 * sub)) + tt * 4096);
    else return *reinterpret_cast<const bf16x8*>(base + vt_rd[sub] + tt * 2048);
  };
  auto v_frag = [&](int t, int sub, int tt, int ci) __attribute__((always_inline)) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const char* a = smem + (G::ST == 2 ? t & 1 : 0) * G::VT + v_rd + (sub * 32 + (M32 ? 8 * ci : 0)) * G::VP + tt * (M32 ? 64 : 32);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORCH_LDS s16x4*)(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORCH_LDS s16x4*)(a + 16 * G::VP));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  // O^T.  M32: tile t (channels 32 t ..) of the lane's query, 16 registers.  Else tile t (channels 16
  // t ..) of queries 16 j + (lane & 15): four registers at 4 (f % 4) of oo[f / 4], f = 2 t + j.
  constexpr int NO = G::NO;
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
  // The probabilities of a half, p = hi + lo: hi the top 16 bits of p, lo what is left of p (1 + 2^-23) as a bf16.  Both
  // are positive (down to p = 2^-103), so that an infinite V gives hi V + lo V = V, not a NaN.
  struct Prob {
    bf16x8 hi[2], lo[2];
  };
  auto p_set = [](Prob& p, int j, int pair, float x0, float x1) __attribute__((always_inline)) {
    constexpr float kUp = 1.0f + 0x1p-23f;
    const unsigned u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
    u32x4 a = __builtin_bit_cast(u32x4, p.hi[j]);
    a[pair] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
    p.hi[j] = __builtin_bit_cast(bf16x8, a);
    p.lo[j][2 * pair] = (bf16)fmaf(x0, kUp, -__uint_as_float(u0 & 0xffff0000u));
    p.lo[j][2 * pair + 1] = (bf16)fmaf(x1, kUp, -__uint_as_float(u1 & 0xffff0000u));
  };
  auto p_zero = [](Prob& p) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) p.hi[j] = p.lo[j] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
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

  auto tiles_sync = [&]() __attribute__((always_inline)) {
    if constexpr (PREP) tiles_wait();
    else if constexpr (KG == 1) lds_sync();
    else asm volatile("" ::: "memory");    // one wave's LDS operations are in order
  };
  // One 32-key half: exponentials of its scores sc between the MFMAs of the next half's scores
  // (NEXT: tile nt, half nsub, into sn) and of the previous half's O^T += V^T P^T (pp; V
  // of tile pt, half psub).  Its probabilities go to pc.  A wave alone has K of that half in kh (kind: of its tile),
  // and reads that of tile nt + 1.
  auto step = [&](auto next_c, bool first, f32x16& sc, int nt, int nsub, f32x16& sn, int pt, int psub, bool vt,
                  Prob& pp, Prob& pc, KHalf& kh, int kind) __attribute__((always_inline)) {
    constexpr bool NEXT = decltype(next_c)::value;
    constexpr int VF = M32 ? 2 : 1;
    bf16x8 vp[VF][NT], kn[NEXT ? NC : 1];
    auto v_frags = [&](int ci) __attribute__((always_inline)) {
      if (PREP || vt) {
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) vp[M32 ? ci : 0][tt] = vt_frag(pt, psub, tt, ci);
      } else {
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) vp[M32 ? ci : 0][tt] = v_frag(pt, psub, tt, ci);
      }
    };
    v_frags(0);
    if constexpr (NEXT && ROW) {
      k_make(kh, nt, nsub, kind, kn);
      k_load(kh, min(nt + 1, te - 1), nsub);
    } else if constexpr (NEXT) {
#pragma unroll
      for (int c = 0; c < NC / 2; ++c) kn[c] = k_frag(nt, nsub, c);
    }
    // (the rest between the MFMAs of the first chunk)
    auto later = [&]() __attribute__((always_inline)) {
      if constexpr (NEXT && !ROW) {
#pragma unroll
        for (int c = NC / 2; c < NC; ++c) kn[c] = k_frag(nt, nsub, c);
      }
      if constexpr (M32) v_frags(1);
    };
    bool gone = false;
    p_swap(pp.hi);
    p_swap(pp.lo);
    float cm = scale, ms = m_run;
    if (__builtin_expect(careful, 0)) {
#pragma clang fp contract(off)
      const float mx = query_max(sc);
      const bool up = raised(mx);
      const float mn = up ? lead(mx) : m_run;
      const float alpha = up ? __builtin_amdgcn_exp2f(m_run - mn) : 1.0f;
      // the probabilities of the previous half, not yet in O, are of the old max: they go
      // in here, and nothing below (zeros on both sides: 0 V would be a NaN where V is infinite)
      if (!first) {
        if constexpr (M32) v_frags(1);
        static_for<0, NT>([&](auto tc) {
          constexpr int tt = decltype(tc)::value;
          pv(tc, std::integral_constant<int, 0>{}, vp[0][tt], pp.hi[0]);
          pv(tc, std::integral_constant<int, 1>{}, vp[VF - 1][tt], pp.hi[1]);
          pv(tc, std::integral_constant<int, 0>{}, vp[0][tt], pp.lo[0]);
          pv(tc, std::integral_constant<int, 1>{}, vp[VF - 1][tt], pp.lo[1]);
        });
      }
      p_zero(pp);
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) vp[0][tt][e] = (bf16)0.0f;
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
        if constexpr (is_pv) {
          pv(std::integral_constant<int, idx>{}, cc, vp[M32 ? ci : 0][idx], pp.hi[ci]);
          pv(std::integral_constant<int, idx>{}, cc, vp[M32 ? ci : 0][idx], pp.lo[ci]);
        } else {
          sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kn[c0 + idx], qf[c0 + idx], c0 + idx == 0 ? zero16 : sn, 0, 0, 0);
        }
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
          for (int e = 0; e < 2; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(sc[8 * ci + 2 * pr + e], cm, -ms));
          p_set(pc, ci, pr, x[0], x[1]);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      asm volatile("" ::"v"(pc.hi[ci]), "v"(pc.lo[ci]));   // (keeps the exponentials here, between the MFMAs)
    });
    __builtin_amdgcn_s_setprio(0);
    // a probability of 2 or more, or not finite: bf16 exponent bit 7
    const u32x4 a = __builtin_bit_cast(u32x4, pc.hi[0]), c = __builtin_bit_cast(u32x4, pc.hi[1]);
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
        for (int pr = 0; pr < 4; ++pr) {
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float score = sc[8 * j + 2 * pr + e], s = score * cm;
            x[e] = __builtin_amdgcn_exp2f(huge ? s - ms : fmaf(score, cm, -ms));
          }
          p_set(pc, j, pr, x[0], x[1]);
        }
      careful = needs_care();
    }
    if constexpr (G::ONES) return;
    // the sum of what the products take, in fp32
    const bf16x2 one2 = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u32x4 w = __builtin_bit_cast(u32x4, k < 2 ? pc.hi[k] : pc.lo[k - 2]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned two = w[e];
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), one2, l_run, false);
      }
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

  // Between the halves of tile t, behind a barrier, K of tile t + 2 takes the place of tile t's, and V of t + 1
  // that of t - 1's (a wave alone: V of t); their loads were issued a whole tile earlier, into registers.
  constexpr int VA = G::ST - 1;
  // ty1 .. ty4: kinds of tiles t .. t + 3; vt0: tile t - 1 holds V^T
  auto tile = [&](int t) __attribute__((always_inline)) { return min(t, te - 1); };
  if (KG == 1 || t0 < te) {
    int ty1 = PREP ? 0 : type_of(t0), ty2 = PREP ? 0 : type_of(tile(t0 + 1)), ty3 = PREP ? 0 : type_of(tile(t0 + 2));
    Raw kr, vr;
    KHalf kh0, kh1;
    if constexpr (PREP) {
      issue(kK, t0);
      issue(kV, t0);
      issue(kK, tile(t0 + 1));
    } else if constexpr (G::ST == 2) {
      Raw kr1;
      load(kK, kr, t0, ty1);
      load(kV, vr, t0, ty1);
      load(kK, kr1, tile(t0 + 1), ty2);
      store(kK, kr, t0, ty1);
      load(kK, kr, tile(t0 + 2), ty3);
      store(kV, vr, t0, ty1);
      load(kV, vr, tile(t0 + 1), ty2);
      if (t0 + 1 < te) store(kK, kr1, t0 + 1, ty2);
    } else {
      k_load(kh0, t0, 0);
      k_load(kh1, t0, 1);
      load(kV, vr, t0, ty1);
    }
    tiles_sync();
    f32x16 s0, s1;
    {
      bf16x8 k0[NC];
      if constexpr (ROW) {
        k_make(kh0, t0, 0, ty1, k0);
        k_load(kh0, tile(t0 + 1), 0);
      } else {
#pragma unroll
        for (int c = 0; c < NC; ++c) k0[c] = k_frag(t0, 0, c);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[c], qf[c], c == 0 ? zero16 : s0, 0, 0, 0);
    }
    Prob pa, pb;
    p_zero(pa);
    bool vt0 = ty1 == kFresh;
    int t = t0;
    for (; t + 1 < te; ++t) {
      const bool vt1 = ty1 == kFresh;
      step(std::true_type{}, t == t0, s0, t, 1, s1, t == t0 ? t : t - 1, t == t0 ? 0 : 1, vt0, pa, pb, kh1, ty1);
      tiles_sync();
      if constexpr (PREP) {
        if (t + 2 < te) issue(kK, t + 2);
        issue(kV, t + 1);
        step(std::true_type{}, false, s1, t + 1, 0, s0, t, 0, vt1, pb, pa, kh0, ty2);
        continue;
      }
      const int t3 = tile(t + 3), ty4 = type_of(t3);
      if constexpr (!ROW) {
        if (t + 2 < te) store(kK, kr, t + 2, ty3);
        load(kK, kr, t3, ty4);
      }
      store(kV, vr, t + VA, G::ST == 2 ? ty2 : ty1);
      load(kV, vr, tile(t + VA + 1), G::ST == 2 ? ty3 : ty2);
      step(std::true_type{}, false, s1, t + 1, 0, s0, t, 0, vt1, pb, pa, kh0, ty2);
      vt0 = vt1;
      ty1 = ty2;
      ty2 = ty3;
      ty3 = ty4;
    }
    const bool vt1 = ty1 == kFresh;
    mask(t, 0, s0);
    step(std::true_type{}, t == t0, s0, t, 1, s1, t == t0 ? t : t - 1, t == t0 ? 0 : 1, vt0, pa, pb, kh1, ty1);
    tiles_sync();      // V of the last tile came since the last one
    if constexpr (G::ST == 1) store(kV, vr, t, ty1);
    mask(t, 1, s1);
    step(std::false_type{}, false, s1, 0, 0, s0, t, 0, vt1, pb, pa, kh0, kStale);
    p_swap(pa.hi);
    p_swap(pa.lo);
    static_for<0, NT>([&](auto tc) {
      constexpr int tt = decltype(tc)::value;
      static_for<0, 2>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        const bf16x8 v = PREP || vt1 ? vt_frag(t, 1, tt, j) : v_frag(t, 1, tt, j);
        pv(tc, jc, v, pa.hi[j]);
        pv(tc, jc, v, pa.lo[j]);
      });
    });
  }
  if constexpr (G::ONES) {
    // row D of O^T, of query 16 j + i: register (D % 16) % 4 of lane 16 (D % 16 / 4) + i
    constexpr int f0 = 2 * (D / 16), r0 = D % 16 % 4;
    float lj[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) lj[j] = __shfl(oo[(f0 + j) / 4][4 * ((f0 + j) % 4) + r0], 16 * (D % 16 / 4) + i16, kWave);
    l_run = lc < 16 ? lj[0] : lj[1];
  } else {
    l_run += __shfl_xor(l_run, 32, kWave);
  }

  // key groups: group 0 takes the others' parts, [register][lane] in their tiles' places, in their order
  if constexpr (KG > 1) {
    __syncthreads();
    if (kg > 0) {
      float* o = reinterpret_cast<float*>(smem) + lane;
#pragma unroll
      for (int k = 0; k < NO; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[(16 * k + r) * 64] = oo[k][r];
      o[NO * 1024] = m_run;
      o[NO * 1024 + 64] = l_run;
    }
    __syncthreads();
    if (kg > 0) return;
    // (relative to a max of minus infinity: 0, not the NaN of inf - inf)
    auto weight = [](float a, float b) { return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b); };
#pragma unroll 1
    for (int g = 1; g < KG; ++g) {
      const float* o = reinterpret_cast<const float*>(smem_all + g * G::GROUP) + lane;
      const float m2 = o[NO * 1024], mn = fmaxf(m_run, m2), f1 = weight(m_run, mn), f2 = weight(m2, mn);
      rescale(f1);
      l_run = l_run * f1 + o[NO * 1024 + 64] * f2;
      m_run = mn;
      float fj[2] = {f2, f2};
      if constexpr (!M32) {
#pragma unroll
        for (int j = 0; j < 2; ++j) fj[j] = __shfl(f2, 16 * j + i16, kWave);
      }
#pragma unroll
      for (int k = 0; k < NO; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (M32 || 4 * k + r / 4 < 2 * NT) oo[k][r] = fmaf(o[(16 * k + r) * 64], fj[(r >> 2) & 1], oo[k][r]);
    }
  }

  // a lane holds channels 32 t + 8 g + 4 h .. +4 of query lane & 31 (M32), or 16 t + 4 (lane >> 4)
  // .. +4 of queries 16 j + (lane & 15)
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
#endif
}

// ---------------------------------------------------------------------------
// Prepared tiles.  Every 128 queries of a (branch, head) read the same keys, and a wave's VALU work is
// paid in full next to its MFMAs: with many queries the keys are widened once, fresh and cached ones
// together, into tiles that lie in memory as they will in LDS: K rows of KP bytes, V^T rows of 64 keys
// with their 16-byte chunks swizzled by row (keys past the last are zeros).  Bound by memory: 16384 keys, 2 x 16 heads
// of 72 (53 MB read of HBM, 152 written) in 50 us, 4.1 TB/s.
template <int D>
__global__ __launch_bounds__(256) void attn_q8_prepare_kernel(AttnQParams p, char* tiles) {
  using G = Geo<D, 4, true>;
  constexpr int CPT = G::CPT, PITCH = D + 4, QUADS = D / 4;
  __shared__ __attribute__((aligned(16))) unsigned char bytes[BKV * PITCH];
  const int tid = threadIdx.x, t = blockIdx.x, pair = blockIdx.y;
  const int b = pair / p.heads, head = pair - b * p.heads;
  const int N = p.c.tokens, nf = p.n_fresh, fb = nf > 0 ? p.fresh_begin : 0, n0 = t * BKV;
  const size_t H = (size_t)p.heads * D;
  const unsigned char* vals = p.c.values + b * p.c.values_bs;
  const unsigned char* exps = p.c.exps + b * p.c.exps_bs;
  const size_t krow = (size_t)head * N + n0, vrow = (size_t)(p.heads + head) * N + n0;
  const bf16* kf = reinterpret_cast<const bf16*>(p.kv_fresh) + b * p.fresh_bs + (size_t)head * nf * D;
  const bf16* vf = reinterpret_cast<const bf16*>(p.kv_fresh) + b * p.fresh_bs + nf * H + (size_t)head * D * nf;
  char* img = tiles + ((size_t)pair * gridDim.x + t) * (G::KT + G::VT);
  auto fresh = [&](int key) { return (unsigned)(n0 + key - fb) < (unsigned)nf; };

  u32x2 vb[(BKV * CPT + 255) / 256];
#pragma unroll
  for (int i = 0; i < (BKV * CPT + 255) / 256; ++i) {
    const int id = i * 256 + tid, key = id / CPT;
    vb[i] = id < BKV * CPT && n0 + key < N && !fresh(key) ? *reinterpret_cast<const u32x2*>(vals + vrow * D + (size_t)id * 8) : u32x2{0, 0};
  }
#pragma unroll
  for (int i = 0; i < (BKV * CPT + 255) / 256; ++i) {
    const int id = i * 256 + tid, key = id / CPT, ch = id - key * CPT;
    if (id >= BKV * CPT) continue;
    u32x4 x = {0, 0, 0, 0};
    if (fresh(key)) {
      x = *reinterpret_cast<const u32x4*>(kf + (size_t)(n0 + key - fb) * D + ch * 8);
    } else if (n0 + key < N) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(vals + krow * D + (size_t)id * 8);
      const float s = scale_of(exps[krow + key]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        x[2 * k] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], s, false));
        x[2 * k + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], s, true));
      }
    }
    *reinterpret_cast<u32x4*>(img + key * G::KP + ch * 16) = x;
    unsigned* to = reinterpret_cast<unsigned*>(bytes + key * PITCH + ch * 8);
    to[0] = vb[i][0];
    to[1] = vb[i][1];
  }
  __syncthreads();
  // V^T: 8 keys x 4 channels a thread, eight neighbouring lanes the same keys
  const int lane = tid & 63, tg = lane >> 3, quad = (tid >> 6) * 8 + (lane & 7);
  auto put = [&](int c, const u32x4& x) {
    *reinterpret_cast<u32x4*>(img + G::KT + c * 128 + ((tg ^ ((c >> 1) & 7)) * 16)) = x;
  };
  if constexpr (G::ONES)
    if (quad == QUADS) put(D, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  if (quad >= QUADS) return;
  const int f = n0 + 8 * tg - fb;
  if (f >= 0 && f + 8 <= nf) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const u32x4_u x = *reinterpret_cast<const u32x4_u*>(vf + (size_t)(4 * quad + c) * nf + f);
      put(4 * quad + c, u32x4{x[0], x[1], x[2], x[3]});
    }
    return;
  }
  unsigned short o[4][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int key = 8 * tg + e;
    const float s = scale_of(n0 + key < N ? exps[vrow + key] : 127u);
    const unsigned w = *reinterpret_cast<const unsigned*>(bytes + key * PITCH + 4 * quad);
    const unsigned lo = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
    const unsigned hi = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
    o[0][e] = (unsigned short)lo;
    o[1][e] = (unsigned short)(lo >> 16);
    o[2][e] = (unsigned short)hi;
    o[3][e] = (unsigned short)(hi >> 16);
    if (fresh(key))
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c][e] = reinterpret_cast<const unsigned short*>(vf)[(size_t)(4 * quad + c) * nf + f + e];
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = o[c][2 * e] | (unsigned)o[c][2 * e + 1] << 16;
    put(4 * quad + c, x);
  }
}

// ---------------------------------------------------------------------------
// fp32: v_mfma_f32_32x32x2_f32, 32 keys a tile.  Its two k are channels 8 g + e and 8 g + 4 + e of the
// scores, and keys 8 g + e and 8 g + 4 + e of the PV product, which score register 4 g + e holds in the two
// lane halves: the probabilities need no movement, and V is read token-major, 32 channels of a key by 32 lanes.
// The MFMAs of a tile (64 cycles each) outweigh everything else, so every wave works alone: the KG
// waves of a workgroup have the same 32 queries and each a share of the keys; their parts meet in LDS.
template <int D>
struct Geo32 {
  static constexpr int BK = 32, NG = D / 8, DT = (D + 31) / 32, CPT = D / 8;
  static constexpr int KG = D <= 64 ? 8 : 4;
  static constexpr int KP = 4 * D + 16;          // bytes of a K row: an odd number of 16-byte chunks
  static constexpr int VP = 128 * DT + 32;       // of a V row: four rows apart are the other 32 banks
  static constexpr int TILE = BK * (KP + VP), LDS = KG * TILE;
  static constexpr int SL = (BK * CPT + 63) / 64;
  static constexpr int WPC = cmin(2, 160 * 1024 / LDS);
  static_assert((DT * 16 + 2) * 256 <= TILE, "a group's part fits its tile's place");
  // us of a tile in a wave: 64 cycles an MFMA, 1500 for the rest
  static constexpr double tile_us = (32.0 * D + 1024.0 * DT + 1500.0) / 2400.0;
};

template <int D>
__global__ __launch_bounds__(64 * Geo32<D>::KG, Geo32<D>::KG / 4) void attn_q8_f32_kernel(AttnQParams p, Split sp) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma clang fp contract(off)
  using G = Geo32<D>;
  constexpr int SL = G::SL, CPT = G::CPT, BK = G::BK, DT = G::DT, KG = G::KG;
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  const int lane = threadIdx.x & 63, lc = lane & 31, h = lane >> 5;
  const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* sk = smem_all + kg * G::TILE;
  char* sv = sk + BK * G::KP;
  const int n_qt = (p.n_q + 31) / 32;
  const int NWG = gridDim.x;
  int w = blockIdx.x;
  if (w < NWG / 8 * 8) w = (w & 7) * (NWG / 8) + (w >> 3);
  const int unit = w / sp.ns, part = w - unit * sp.ns;
  const int pair = unit / n_qt, q0 = (unit - pair * n_qt) * 32;
  const int b = pair / p.heads, head = pair - b * p.heads;
  const int N = p.c.tokens, nf = p.n_fresh, fb = nf > 0 ? p.fresh_begin : 0;
  const int nkt = (N + BK - 1) / BK, shares = sp.ns * KG, share = part * KG + kg;
  const int t0 = (int)((long long)nkt * share / shares), t1 = (int)((long long)nkt * (share + 1) / shares);
  const size_t H = (size_t)p.heads * D;
  const __amdgpu_buffer_rsrc_t rk8 = buffer_rsrc(p.c.values + b * p.c.values_bs + (size_t)head * N * D, (size_t)N * D);
  const __amdgpu_buffer_rsrc_t rv8 = buffer_rsrc(p.c.values + b * p.c.values_bs + (size_t)(p.heads + head) * N * D, (size_t)N * D);
  const __amdgpu_buffer_rsrc_t rke = buffer_rsrc(p.c.exps + b * p.c.exps_bs + (size_t)head * N, N);
  const __amdgpu_buffer_rsrc_t rve = buffer_rsrc(p.c.exps + b * p.c.exps_bs + (size_t)(p.heads + head) * N, N);
  const float *kf = nullptr, *vf = nullptr;
  if (nf > 0) {
    kf = reinterpret_cast<const float*>(p.kv_fresh) + b * p.fresh_bs + (size_t)head * nf * D;
    vf = reinterpret_cast<const float*>(p.kv_fresh) + b * p.fresh_bs + nf * H + (size_t)head * D * nf;
  }
  // V's padding channels: zero, never written again
  if constexpr (32 * DT > D)
    for (int i = lane; i < BK * (32 * DT - D); i += 64)
      *reinterpret_cast<float*>(sv + i / (32 * DT - D) * G::VP + (D + i % (32 * DT - D)) * 4) = 0.0f;

  // chunk i * 64 + lane of a tile: channels 8 ch .. +8 of key `key`; a key past the last reads zeros
  u32x2 kr[SL], vr[SL];
  unsigned ke[SL], ve[SL];
  auto load = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      const int id = i * 64 + lane;
      const int off = id < BK * CPT ? id * 8 : 0x7fffffff - BK * D;
      kr[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rk8, off, t * BK * D, 0));
      vr[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rv8, off, t * BK * D, 0));
      ke[i] = __builtin_amdgcn_raw_buffer_load_b8(rke, id / CPT, t * BK, 0);
      ve[i] = __builtin_amdgcn_raw_buffer_load_b8(rve, id / CPT, t * BK, 0);
    }
  };
  auto put = [&](char* dst, u32x2 x, unsigned e) __attribute__((always_inline)) {
    const float s = scale_of(e);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned word = x[i];
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, s, false);
      const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, s, true);
      reinterpret_cast<f32x4*>(dst)[i] = f32x4{a[0], a[1], c[0], c[1]};
    }
  };
  auto store = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      const int id = i * 64 + lane, key = id / CPT, ch = id - key * CPT;
      if (64 * SL == BK * CPT || i + 1 < SL || key < BK) {
        put(sk + key * G::KP + ch * 32, kr[i], ke[i]);
        put(sv + key * G::VP + ch * 32, vr[i], ve[i]);
      }
    }
    // the band's own keys over them
    const int n0 = t * BK;
    if (n0 + BK > fb && n0 < fb + nf) {
#pragma unroll 2
      for (int i = 0; i < SL; ++i) {
        const int id = i * 64 + lane, key = id / CPT, ch = id - key * CPT, f = n0 + key - fb;
        if (key >= BK || (unsigned)f >= (unsigned)nf) continue;
        const f32x4* src = reinterpret_cast<const f32x4*>(kf + (size_t)f * D + ch * 8);
        const float* col = vf + (size_t)ch * 8 * nf + f;
        f32x4* dk = reinterpret_cast<f32x4*>(sk + key * G::KP + ch * 32);
        f32x4* dv = reinterpret_cast<f32x4*>(sv + key * G::VP + ch * 32);
        f32x4 v[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = col[(size_t)e * nf];
        dk[0] = src[0];
        dk[1] = src[1];
        dv[0] = v[0];
        dv[1] = v[1];
      }
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

  if (t0 < t1) load(t0);
  for (int t = t0; t < t1; ++t) {
    store(t);
    load(min(t + 1, t1 - 1));
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
  }
  l_run += __shfl_xor(l_run, 32, kWave);

  // key group 0 takes the others' parts, [register][lane] in their tiles' places, in their order
  __syncthreads();
  if (kg > 0) {
    float* o = reinterpret_cast<float*>(sk) + lane;
#pragma unroll
    for (int tt = 0; tt < DT; ++tt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[(16 * tt + r) * 64] = oo[tt][r];
    o[DT * 1024] = m_run;
    o[DT * 1024 + 64] = l_run;
  }
  __syncthreads();
  if (kg > 0) return;
  auto weight = [](float a, float c) { return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - c); };
#pragma unroll 1
  for (int g = 1; g < KG; ++g) {
    const float* o = reinterpret_cast<const float*>(smem_all + g * G::TILE) + lane;
    const float m2 = o[DT * 1024], mn = fmaxf(m_run, m2), f1 = weight(m_run, mn), f2 = weight(m2, mn);
    l_run = l_run * f1 + o[DT * 1024 + 64] * f2;
    m_run = mn;
#pragma unroll
    for (int tt = 0; tt < DT; ++tt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oo[tt][r] = oo[tt][r] * f1 + o[(16 * tt + r) * 64] * f2;
  }
  if (q0 + lc >= p.n_q) return;
  const size_t slot = ((size_t)unit * sp.ns + part) * 32 + lc;
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
#endif
}

// The parts of a query tile whose keys ns workgroups shared: O = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s
// - m) l_s, m = max_s m_s.  A thread per 4 channels of a query and share of the parts (part s of
// share s % SG, four in flight), the shares met in LDS in their order.  Bound by its own launch and one chain of loads
// for few parts (3.5-5 us), by their bytes for many (384 queries x 5 parts, 2 x 16 heads of 72: 18 MB in 5.5 us).
template <typename T, int SG>
__global__ __launch_bounds__(256) void attn_q8_merge_kernel(AttnQParams p, Split sp, int rows) {
  __shared__ float ml_s[256][2];
  __shared__ f32x4 o_s[256];
  const int quads = p.d / 4, per = quads * SG, qpb = 256 / per;
  const int n_qt = (p.n_q + rows - 1) / rows;
  const int qi = threadIdx.x / per, share = (threadIdx.x - qi * per) / quads, c = 4 * (threadIdx.x % quads);
  const long long query = (long long)blockIdx.x * qpb + qi;          // (branch, head, query)
  const bool on = qi < qpb && query < (long long)p.B * p.heads * p.n_q;
  const int pair = on ? (int)(query / p.n_q) : 0, q = on ? (int)(query - (long long)pair * p.n_q) : 0;
  const size_t slot = ((size_t)pair * n_qt + q / rows) * sp.ns * rows + q % rows;
  const float2* ml = sp.part_ml + slot;
  const float* po = sp.part_o + slot * p.d + c;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  // weights relative to a max of minus infinity are 0, not the NaN of inf - inf
  auto weight = [](float a, float b) { return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b); };
  if (on)
    for (int s0 = share; s0 < sp.ns; s0 += 4 * SG) {
      float2 x[4];
      f32x4 y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = min(s0 + k * SG, sp.ns - 1);
        x[k] = ml[(size_t)s * rows];
        y[k] = *reinterpret_cast<const f32x4*>(po + (size_t)s * rows * p.d);
        if (s0 + k * SG >= sp.ns) x[k].x = -INFINITY;
      }
      const float mn = fmaxf(m, fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x)));
      const float f0 = weight(m, mn);
      l *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f0;
      m = mn;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (s0 + k * SG >= sp.ns) continue;
        const float f = weight(x[k].x, mn);
        l = fmaf(f, x[k].y, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(f, y[k][e], o[e]);
      }
    }
  ml_s[threadIdx.x][0] = m;
  ml_s[threadIdx.x][1] = l;
  o_s[threadIdx.x] = o;
  __syncthreads();
  if (!on || share > 0) return;
  float mn = m;
#pragma unroll
  for (int k = 1; k < SG; ++k) mn = fmaxf(mn, ml_s[threadIdx.x + k * quads][0]);
  const float f0 = weight(m, mn);
  l *= f0;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
  for (int k = 1; k < SG; ++k) {
    const int i = threadIdx.x + k * quads;
    const float f = weight(ml_s[i][0], mn);
    const f32x4 y = o_s[i];
    l = fmaf(f, ml_s[i][1], l);
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

template <typename T, int SG>
hipError_t launch_merge(const AttnQParams& p, const Split& sp, int rows, hipStream_t s) {
  const int qpb = 256 / (p.d / 4 * SG);
  const size_t queries = (size_t)p.B * p.heads * p.n_q;
  hipLaunchKernelGGL((attn_q8_merge_kernel<T, SG>), dim3((unsigned)((queries + qpb - 1) / qpb)), dim3(256), 0, s, p, sp, rows);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The plan of a call: the variant (tiles prepared or not, query groups of a workgroup) and the number ns
// of workgroups that share a query tile's keys, by the least estimated time.  In us, at d = 72 (other head
// sizes scale a tile by 0.5 + d / 140): a workgroup starts and ends in 4; a 64-key tile of a workgroup
// takes the `tile` below, by the workgroups on its CU; parts take 5 and their bytes, written and read, at
// 5 TB/s; preparing 2.5 and 5.5 ns a tile.  Fitted to 16 shapes at each head size, every variant and split: the
// chosen one takes 1.7% longer than the best of them in the mean, 19% at most (32 heads of 32, 384 queries x 4096
// keys).  Measured against the estimate (2 x 16 heads, d = 72): 384 queries x 4096 keys on NW = 4 / ns = 1, 2,
// 5: 104 / 66 / 44 (105 / 62 / 43 estimated), on NW = 1 / ns = 1 45 (44), prepared / ns = 5 45 (49); 1664 x 1024 on
// NW = 4 / ns = 1, 2 43 / 57 (37 / 59), prepared / 1 41 (32).
struct Plan {
  int nw, ns, prep;
  size_t tiles;
  double cost;
};

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

// A variant's best ns into *best if it beats it.  rows: queries of a workgroup; groups: key groups of
// it; tile[c - 1]: a tile's time with c workgroups on the CU; fixed: time before.
void consider(Plan* best, int nw, int prep, long long pairs, int n_q, int rows, int groups, int nkt, int wpc,
              const double (&tile)[3], double fixed, int d, int max_ns) {
  const long long units = ceil_div(n_q, rows) * pairs;
  const double scale = 0.5 + d / 140.0;
  for (int ns = 1; ns <= max_ns && ns <= ceil_div(nkt, groups); ns += ns < 8 ? 1 : ns / 4) {
    const long long w = units * ns, per_cu = (w + 255) / 256, rounds = (per_cu + wpc - 1) / wpc;
    const int c = (int)(per_cu < wpc ? per_cu : wpc);
    const double cost = fixed + (double)rounds * (4.0 + ceil_div(nkt, groups * ns) * tile[c - 1] * scale) +
                        (ns > 1 ? 5.0 + (double)(pairs * n_q) * ns * d * 8 / 5e6 : 0.0);
    if (cost < best->cost) *best = {nw, ns, prep, (size_t)units, cost};
  }
}

// workspace: the call has one (else the keys are neither prepared nor split)
Plan plan(int B, int heads, int n_q, int n_kv, int d, int dtype, bool workspace) {
  Plan r{0, 1, 0, 0, 1e300};
  const long long pairs = (long long)B * heads;
  const int max_ns = workspace ? 64 : 1;
  with_d(d, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    if (dtype == kBF16) {
      const int nkt = ceil_div(n_kv, BKV);
      consider(&r, 4, 0, pairs, n_q, 128, 1, nkt, Geo<D, 4>::WPC, {1.5, 2.05, 0}, 0.0, d, max_ns);
      // (its longer straight code is read once by every CU: 0.7 us at d = 64, 4.8 at d = 128; 2 x 8
      // heads, 1000 queries x 4096 keys at d = 32, 64: 30, 42 us, prepared 38, 47)
      consider(&r, 1, 0, pairs, n_q, 32, 4, nkt, Geo<D, 1>::WPC, {D == 128 ? 1.6 : 1.3, 2.4, 0}, D <= 64 ? D * 0.011 : 0.7 + (D - 64) * 0.063, d, max_ns);
      if (workspace && (long long)nkt * (Geo<D, 4, true>::KT + Geo<D, 4, true>::VT) < (1ll << 31))
        consider(&r, 4, 1, pairs, n_q, 128, 1, nkt, Geo<D, 4, true>::WPC, {1.2, 1.4, 2.4},
                 2.5 + 0.0055 * (double)(pairs * nkt) * (0.5 + d / 140.0), d, max_ns);
    } else {
      // 32-key tiles; the matrix pipe of a SIMD is one wave's at a time
      using G = Geo32<D>;
      const double alone = G::tile_us * (G::KG / 4) / (0.5 + d / 140.0);
      consider(&r, 1, 0, pairs, n_q, 32, G::KG, ceil_div(n_kv, G::BK), G::WPC, {alone, 2 * alone, 0}, 0.0, d, max_ns);
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

template <int D, int NW, bool PREP>
hipError_t launch_bf16(const Plan& pl, const AttnQParams& p, const Split& sp, hipStream_t s) {
  constexpr int lds = Geo<D, NW, PREP>::LDS;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_q8_kernel<D, NW, PREP>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  return attr != hipSuccess ? attr : launch(attn_q8_kernel<D, NW, PREP>, lds, 256, pl.tiles * pl.ns, p, sp, s);
}

template <int D>
hipError_t launch_f32(const Plan& pl, const AttnQParams& p, const Split& sp, hipStream_t s) {
  using G = Geo32<D>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_q8_f32_kernel<D>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
  return attr != hipSuccess ? attr : launch(attn_q8_f32_kernel<D>, G::LDS, 64 * G::KG, pl.tiles * pl.ns, p, sp, s);
}

// Bytes of the prepared tiles and of the parts.
size_t tile_bytes(const Plan& pl, int B, int heads, int n_kv, int d) {
  size_t r = 0;
  if (pl.prep)
    with_d(d, [&](auto dc) {
      using G = Geo<decltype(dc)::value, 4, true>;
      r = (size_t)ceil_div(n_kv, BKV) * (G::KT + G::VT) * B * heads;
    });
  return r;
}

size_t split_bytes(const Plan& pl, int d) {
  return pl.ns == 1 ? 0 : part_floats(pl, d) * 4 + pl.tiles * pl.ns * 32 * pl.nw * sizeof(float2);
}

size_t need_bytes(const Plan& pl, int B, int heads, int n_kv, int d) {
  return split_bytes(pl, d) + tile_bytes(pl, B, heads, n_kv, d);
}

// The plan of a call with ws_bytes of workspace (0: none): that of the whole workspace, or that of none.
Plan plan_within(int B, int heads, int n_q, int n_kv, int d, int dtype, size_t ws_bytes) {
  const Plan pl = plan(B, heads, n_q, n_kv, d, dtype, true);
  return pl.nw == 0 || (ws_bytes > 0 && ws_bytes >= need_bytes(pl, B, heads, n_kv, d)) ? pl : plan(B, heads, n_q, n_kv, d, dtype, false);
}

}  // namespace q8attn

size_t attention_quantized_workspace_bytes(int B, int heads, int n_q, int n_kv, int d, int dtype) {
  using namespace q8attn;
  if (n_q <= 0) return 0;
  const Plan pl = plan(B, heads, n_q, n_kv, d, dtype, true);
  return pl.nw == 0 ? 0 : need_bytes(pl, B, heads, n_kv, d);
}

bool attention_quantized_plan(int B, int heads, int n_q, int n_kv, int d, int dtype, size_t ws_bytes, int* prepared,
                              int* query_groups, int* key_parts) {
  const q8attn::Plan pl = q8attn::plan_within(B, heads, n_q, n_kv, d, dtype, ws_bytes);
  *prepared = pl.prep;
  *query_groups = pl.nw;
  *key_parts = pl.ns;
  return pl.nw != 0;
}

hipError_t launch_attention_quantized(const AttnQParams& p, int dtype, hipStream_t s) {
  using namespace q8attn;
  if (p.n_q <= 0) return hipSuccess;
  const Plan pl = plan_within(p.B, p.heads, p.n_q, p.c.tokens, p.d, dtype, p.ws ? p.ws_bytes : 0);
  if (pl.nw == 0) return hipErrorInvalidValue;
  const bool prepare = pl.prep;
  if (pl.tiles * pl.ns > 0x7fffffff) return hipErrorInvalidValue;
  Split sp{nullptr, pl.ns, nullptr, nullptr};
  if (prepare) sp.tiles = reinterpret_cast<const char*>(p.ws);
  if (pl.ns > 1) {
    sp.part_o = reinterpret_cast<float*>((char*)p.ws + tile_bytes(pl, p.B, p.heads, p.c.tokens, p.d));
    sp.part_ml = reinterpret_cast<float2*>(sp.part_o + part_floats(pl, p.d));
  }
  hipError_t rc = hipErrorInvalidValue;
  with_d(p.d, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    if (dtype == kBF16 && prepare) {
      hipLaunchKernelGGL(attn_q8_prepare_kernel<D>, dim3(ceil_div(p.c.tokens, BKV), p.B * p.heads), dim3(256), 0, s, p,
                         reinterpret_cast<char*>(p.ws));
      rc = hipGetLastError();
      if (rc == hipSuccess) rc = launch_bf16<D, 4, true>(pl, p, sp, s);
      return;
    }
    if (dtype == kBF16) rc = pl.nw == 4 ? launch_bf16<D, 4, false>(pl, p, sp, s) : launch_bf16<D, 1, false>(pl, p, sp, s);
    else rc = launch_f32<D>(pl, p, sp, s);
  });
  if (rc != hipSuccess || pl.ns == 1) return rc;
  // shares of the parts: eight where few parts' threads would each walk many parts in turn (20 queries x 5000 keys,
  // 40 parts), one where the chip is full without (384 queries x 4096 keys, 5 parts, 2 x 16 heads: 17 us with eight
  // shares, most of them empty, 7 with one)
  const int rows = 32 * pl.nw;
  const long long quads = (long long)p.B * p.heads * p.n_q * (p.d / 4);
  const int shares = quads >= 65536 || pl.ns <= 4 ? 1 : 8;
  if (dtype == kBF16) return shares == 1 ? launch_merge<bf16, 1>(p, sp, rows, s) : launch_merge<bf16, 8>(p, sp, rows, s);
  return shares == 1 ? launch_merge<float, 1>(p, sp, rows, s) : launch_merge<float, 8>(p, sp, rows, s);
}

}  // namespace orch
