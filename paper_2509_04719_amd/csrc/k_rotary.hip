// Rotary positions on a (frames, rows, columns) grid: pair i of a token's
// channels turns by the token's position on the pair's axis times the pair's
// frequency, x' = x cos - y sin, y' = x sin + y cos.
//
// The work is one read and one write of every element; what could cost more is
// the angle.  A thread owns one unit of a row (8 channels) of one token and walks a
// slice of the (tensor, branch, head) rows with it, so an angle is formed once
// for every row of the slice.  Angles are counted in turns: position x frequency /
// 2 pi in fp64 (off by at most three roundings, 3 2^-53 of the angle), the whole turns taken off (exact), the rest to
// fp32 (2^-26 of a turn: what is left of the error below positions of 10^7).  The frequencies come from the host in the kernel's arguments.
// Bound by memory: 46800 tokens, Q and K of 16 heads of 128 in bf16 (767 MB) in 149 us, 5.15 TB/s, what a copy reaches; 1664
// tokens of 2 x 16 heads of 72, Q and K (31 MB), in 8.8 us.
#include "common.h"
#include "kernels.h"

namespace orch {

// The kernel's arguments with the launch's split.
struct RotaryLaunch {
  RotaryParams p;
  int units, per, rows_total, rows0;   // rows0: rows (b, h) of the first tensor
};

// V channels (interleaved) or V pairs (halves) a unit; VEC: 16-byte (or V-element)
// aligned loads.
template <typename T, bool IL, int V, bool VEC>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryLaunch L) {
  const RotaryParams& p = L.p;
  constexpr int P = IL ? V / 2 : V;          // pairs of a unit
  constexpr int E = 2 * P;                   // its elements
  typedef T vec __attribute__((ext_vector_type(V)));
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int tok = i / L.units, u = i - tok * L.units;
  if (tok >= p.n_tok) return;
  const unsigned n = p.token_begin + tok;
  const unsigned line = n / (unsigned)p.cols;
  const unsigned idx[3] = {line / (unsigned)p.rows, line % (unsigned)p.rows, n % (unsigned)p.cols};

  // pair numbers count the axes' pairs one after the other; past them, channels pass through
  const int pair0 = u * P;
  const int rot = p.pairs[0] + p.pairs[1] + p.pairs[2];
  int c0 = pair0 * 2, c1 = 0;                // first channel (and that of the partners)
  if constexpr (!IL) {
    int left = pair0, base = 0, half = 0;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      half = a < 3 ? p.pairs[a] : p.d / 2 - rot;
      if (left < half || a == 3) break;
      left -= half;
      base += 2 * half;
    }
    c0 = base + left;
    c1 = c0 + half;
  }
  // the first rows are on their way while the angles are formed
  constexpr int RB = 4;
  T e[RB][E];
  T* o[RB];
  int r = blockIdx.y * L.per;
  const int r1 = min(r + L.per, L.rows_total);
  auto fetch = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < RB; ++k) {
      if (first + k >= r1) break;
      const bool second = first + k >= L.rows0;
      const RotaryTensor& t = p.t[second ? 1 : 0];
      const int rr = first + k - (second ? L.rows0 : 0);
      const int b = rr / t.heads, h = rr - b * t.heads;
      const T* x = reinterpret_cast<const T*>(t.x) + b * t.xs[0] + h * t.xs[1] + tok * t.xs[2];
      o[k] = reinterpret_cast<T*>(t.out) + b * t.os[0] + h * t.os[1] + tok * t.os[2];
      if constexpr (VEC) {
#pragma unroll
        for (int g = 0; g < E / V; ++g) {
          const vec v = *reinterpret_cast<const vec*>(x + (g ? c1 : c0));
#pragma unroll
          for (int j = 0; j < V; ++j) e[k][g * V + j] = v[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) e[k][j] = x[IL || j < V ? c0 + j : c1 + j - V];
      }
    }
  };
  fetch(r);
  float cs[P], sn[P];
  bool turn[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int k = pair0 + j;
    const int a = k < p.pairs[0] ? 0 : k < p.pairs[0] + p.pairs[1] ? 1 : 2;
    turn[j] = k < rot;
    const double pos = (double)idx[a] + p.origin[a];
    const double t = pos * p.turns[turn[j] ? k : 0];
    const float r = (float)(t - rint(t));
    sincospif(2.0f * r, &sn[j], &cs[j]);
  }

  for (; r < r1; r += RB) {
#pragma unroll
    for (int k = 0; k < RB; ++k) {
      if (r + k >= r1) break;
#pragma unroll
      for (int j = 0; j < P; ++j) {
        T &lo = e[k][IL ? 2 * j : j], &hi = e[k][IL ? 2 * j + 1 : V + j];
        const float a = to_f<T>(lo), c = to_f<T>(hi);
        if (turn[j]) {
          lo = from_f<T>(a * cs[j] - c * sn[j]);
          hi = from_f<T>(a * sn[j] + c * cs[j]);
        }
      }
      if constexpr (VEC) {
#pragma unroll
        for (int g = 0; g < E / V; ++g) {
          vec v;
#pragma unroll
          for (int j = 0; j < V; ++j) v[j] = e[k][g * V + j];
          *reinterpret_cast<vec*>(o[k] + (g ? c1 : c0)) = v;
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) o[k][IL || j < V ? c0 + j : c1 + j - V] = e[k][j];
      }
    }
    fetch(r + RB);
  }
}

template <typename T, bool IL, int V, bool VEC>
static hipError_t launch_rotary_v(const RotaryParams& p, hipStream_t s) {
  RotaryLaunch L;
  L.p = p;
  L.units = p.d / 2 / (IL ? V / 2 : V);
  L.rows0 = p.B * p.t[0].heads;
  L.rows_total = L.rows0 + (p.n_t > 1 ? p.B * p.t[1].heads : 0);
  const long long blocks = ((long long)p.n_tok * L.units + 255) / 256;
  // slices of the rows: up to eight rows an angle, fewer while that leaves under
  // 1024 workgroups (four a CU)
  L.per = (int)(blocks * L.rows_total / 1024);
  L.per = L.per < 1 ? 1 : L.per > 8 ? 8 : L.per;
  const int slices = ceil_div(L.rows_total, L.per);
  hipLaunchKernelGGL((rotary_kernel<T, IL, V, VEC>), dim3((unsigned)blocks, slices), dim3(256), 0, s, L);
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_rotary_t(const RotaryParams& p, hipStream_t s) {
  // elements that every row start, stride and segment is a multiple of
  size_t bits = p.interleaved ? 0 : p.pairs[0] | p.pairs[1] | p.pairs[2] | (p.d / 2 - p.pairs[0] - p.pairs[1] - p.pairs[2]);
  for (int k = 0; k < p.n_t; ++k) {
    bits |= (uintptr_t)p.t[k].x / sizeof(T) | (uintptr_t)p.t[k].out / sizeof(T);
    for (int a = 0; a < 3; ++a) bits |= p.t[k].xs[a] | p.t[k].os[a];
  }
  if (p.interleaved) {
    if (bits % 8 == 0) return launch_rotary_v<T, true, 8, true>(p, s);
    return launch_rotary_v<T, true, 8, false>(p, s);
  }
  if (bits % 8 == 0) return launch_rotary_v<T, false, 8, true>(p, s);
  if (bits % 4 == 0) return launch_rotary_v<T, false, 4, true>(p, s);
  if (bits % 2 == 0) return launch_rotary_v<T, false, 2, true>(p, s);
  return launch_rotary_v<T, false, 1, true>(p, s);
}

hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t s) {
  if (p.n_tok <= 0) return hipSuccess;
  return dtype == kBF16 ? launch_rotary_t<bf16>(p, s) : launch_rotary_t<float>(p, s);
}

}  // namespace orch
