// C ABI of the rotary positions, the 8-bit K/V cache and the attention that
// reads it: argument checks and launches.  Nothing here allocates or throws.
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/orch.h"
#include "common.h"
#include "kernels.h"

using namespace orch;

namespace orch_detail {
int set_error(int code, const char* msg);
}

namespace {

int fail(const char* fmt, ...) __attribute__((format(printf, 1, 2)));
int fail(const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return orch_detail::set_error(ORCH_EINVAL, buf);
}

int launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return ORCH_OK;
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return orch_detail::set_error(ORCH_EHIP, buf);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// `count` runs of `bytes` bytes, `stride` bytes apart: the branches of a buffer
struct Runs {
  const void* p;
  size_t bytes, stride;
  int count;
};

// A byte of both?  (The runs of one may lie between those of the other.)
bool overlap(const Runs& a, const Runs& b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t b0 = (uintptr_t)b.p;
  for (int i = 0; i < a.count; ++i) {
    const uintptr_t lo = (uintptr_t)a.p + (i ? i * a.stride : 0), hi = lo + a.bytes;
    // the first run of b that ends past lo
    const size_t j = lo < b0 + b.bytes ? 0 : b.count > 1 ? (lo - b0 - b.bytes) / b.stride + 1 : 1;
    if (j < (size_t)b.count && b0 + (j ? j * b.stride : 0) < hi) return true;
  }
  return false;
}

// No stride is as long as this (elements or bytes: 1 TB and more); below it no offset wraps.
constexpr size_t kFar = (size_t)1 << 40;

// heads, branches, head size and type that every entry point takes
int check_common(int B, int heads, int head_dim, int dtype) {
  if (B < 1 || heads < 1 || (long long)B * heads > 32767) return fail("bad shape: B and heads must be >= 1, B * heads <= 32767");
  if (!(head_dim == 32 || head_dim == 64 || head_dim == 72 || head_dim == 80 || head_dim == 96 || head_dim == 128))
    return fail("head_dim %d not supported", head_dim);
  if (dtype != ORCH_F32 && dtype != ORCH_BF16) return fail("bad dtype");
  return ORCH_OK;
}

// a cache of B branches; where its values and exponents lie
int check_cache(const orch_quantized_kv* c, int B, int heads, int d, Runs* values, Runs* exps) {
  if (!c || !c->values || !c->exponents) return fail("NULL cache");
  if (c->tokens < 1) return fail("the cache's tokens must be >= 1");
  if ((long long)c->tokens * d >= 1ll << 31) return fail("cache tokens * head_dim must be below 2^31");
  const size_t e = (size_t)2 * heads * c->tokens, v = e * d;
  if (B > 1 && (c->values_stride < v || c->exponents_stride < e || c->values_stride >= kFar || c->exponents_stride >= kFar))
    return fail("the cache's branch stride is too small or past 2^40");
  if (!aligned16(c->values) || (B > 1 && c->values_stride % 16)) return fail("cache values must be 16-byte aligned");
  *values = {c->values, v, c->values_stride, B};
  *exps = {c->exponents, e, c->exponents_stride, B};
  if (overlap(*values, *exps)) return fail("the cache's values and exponents overlap");
  return ORCH_OK;
}

// checks and parameters of writing and reading back
int kv_params(KvCacheParams* p, const void* kv, size_t kv_bs, int kv_tokens, int kv_off, const orch_quantized_kv* c,
              int c_off, int B, int heads, int n, int d, int dtype) {
  if (n != 0 && !kv) return fail("NULL pointer");
  int rc = check_common(B, heads, d, dtype);
  if (rc) return rc;
  Runs values, exps;
  rc = check_cache(c, B, heads, d, &values, &exps);
  if (rc) return rc;
  if (n < 0 || kv_off < 0 || c_off < 0 || kv_tokens < 1 || n > kv_tokens - kv_off || n > c->tokens - c_off)
    return fail("tokens [%d, %d + %d) of %d, [%d, %d + %d) of the cache's %d", kv_off, kv_off, n, kv_tokens, c_off,
                c_off, n, c->tokens);
  if ((long long)kv_tokens * d >= 1ll << 31) return fail("kv_tokens * head_dim must be below 2^31");
  const size_t es = dtype == ORCH_BF16 ? 2 : 4, H = (size_t)heads * d, elems = 2 * (size_t)kv_tokens * H;
  if (B > 1 && (kv_bs < elems || kv_bs >= kFar)) return fail("branch stride too small or past 2^40");
  if (!aligned16(kv) || (B > 1 && kv_bs * es % 16)) return fail("the K/V buffer must be 16-byte aligned");
  const Runs buffer = {kv, elems * es, kv_bs * es, B};
  if (overlap(buffer, values) || overlap(buffer, exps))
    return fail("the K/V buffer and the cache overlap");
  p->c.values = (unsigned char*)c->values; p->c.exps = (unsigned char*)c->exponents;
  p->c.values_bs = c->values_stride; p->c.exps_bs = c->exponents_stride; p->c.tokens = c->tokens;
  p->c_off = c_off; p->kv = const_cast<void*>(kv); p->kv_bs = kv_bs; p->kv_tokens = kv_tokens; p->kv_off = kv_off;
  p->B = B; p->heads = heads; p->d = d; p->n = n;
  return ORCH_OK;
}

}  // namespace

extern "C" {

int orch_op_rotary(const orch_rotary_axes* axes, const orch_rotary_tensor* tensors, int n_tensors, int B, int n_tok,
                   int token_begin, int head_dim, int dtype, void* hip_stream) {
  if (!axes || !tensors) return fail("NULL pointer");
  if (n_tensors < 1 || n_tensors > 2) return fail("n_tensors must be 1 or 2");
  int rc = check_common(B, 1, head_dim, dtype);
  if (rc) return rc;
  RotaryParams p{};
  long long tokens = 1;
  int channels = 0, pair = 0;
  if (!(axes->theta > 0.0) || !std::isfinite(axes->theta)) return fail("theta must be finite and > 0");
  const long double log_theta = std::log((long double)axes->theta);
  for (int a = 0; a < 3; ++a) {
    const int ch = axes->channels[a], ext = axes->extent[a];
    if (ch < 0 || ch % 2 || ch > head_dim - channels) return fail("axis channels must be even, >= 0 and at most head_dim in all");
    if (ext < 1 || ext > 0x7fffffffll / tokens) return fail("grid extents must be >= 1 and their product below 2^31");
    if (!std::isfinite(axes->origin[a]) || !std::isfinite(axes->step[a])) return fail("origin and step must be finite");
    channels += ch;
    tokens *= ext;
    p.pairs[a] = ch / 2;
    p.origin[a] = axes->origin[a];
    // theta^(-2 i / channels), one multiplication a pair in 80 bits: 64 roundings of 2^-64 and the
    // logarithm's (times its own size) leave fp64's rounding of the result alone (in fp64 the 64th would be off by 2^-46)
    const long double ratio = ch > 2 ? std::exp(log_theta * (-2.0L / ch)) : 1.0L;
    long double f = axes->step[a] / 6.283185307179586476925286766559L;
    for (int i = 0; i < ch / 2; ++i, f *= ratio) {
      const double turns = (double)f;
      if (!std::isfinite(turns * (std::fabs(axes->origin[a]) + ext))) return fail("an angle of axis %d is past fp64's range", a);
      p.turns[pair++] = turns;
    }
  }
  if (n_tok < 0 || token_begin < 0 || n_tok > tokens - token_begin)
    return fail("tokens [%d, %d + %d) not within the grid's %lld", token_begin, token_begin, n_tok, tokens);
  if ((long long)n_tok * head_dim >= 1ll << 31) return fail("n_tok * head_dim must be below 2^31");
  const size_t es = dtype == ORCH_BF16 ? 2 : 4;
  for (int k = 0; k < n_tensors; ++k) {
    const orch_rotary_tensor& t = tensors[k];
    if (n_tok > 0 && (!t.x || !t.out)) return fail("NULL pointer");
    if (t.heads < 1 || (long long)t.heads * B > 32767) return fail("bad shape: heads must be >= 1, B * heads <= 32767");
    if ((uintptr_t)t.x % es || (uintptr_t)t.out % es) return fail("tensors must be aligned to their elements");
    const int extent[3] = {B, t.heads, n_tok};
    for (int a = 0; a < 3; ++a)
      if (n_tok > 0 && extent[a] > 1 && (t.x_stride[a] < (size_t)head_dim || t.out_stride[a] < (size_t)head_dim ||
                                         t.x_stride[a] >= kFar || t.out_stride[a] >= kFar))
        return fail("strides must be at least head_dim and below 2^40");
    p.t[k].x = t.x; p.t[k].out = t.out; p.t[k].heads = t.heads;
    for (int a = 0; a < 3; ++a) {
      // (the stride of an extent of one is never used)
      p.t[k].xs[a] = extent[a] > 1 ? t.x_stride[a] : 0;
      p.t[k].os[a] = extent[a] > 1 ? t.out_stride[a] : 0;
      if (n_tok > 0 && t.x == t.out && p.t[k].xs[a] != p.t[k].os[a]) return fail("in place needs the same strides");
    }
  }
  if (n_tensors == 2 && n_tok > 0) {
    const orch_rotary_tensor &a = tensors[0], &c = tensors[1];
    if (a.out == c.out || a.out == c.x || a.x == c.out) return fail("the two tensors overlap");
  }
  p.n_t = n_tensors; p.B = B; p.n_tok = n_tok; p.d = head_dim; p.token_begin = token_begin;
  p.rows = axes->extent[1]; p.cols = axes->extent[2]; p.interleaved = axes->interleaved != 0;
  return launched(launch_rotary(p, dtype, (hipStream_t)hip_stream), "rotary launch");
}

int orch_op_kv_quantize(const void* kv, size_t kv_bs, int kv_tokens, int kv_off, const orch_quantized_kv* cache,
                        int tok_off, int B, int heads, int n_tok, int head_dim, int dtype, void* hip_stream) {
  KvCacheParams p{};
  int rc = kv_params(&p, kv, kv_bs, kv_tokens, kv_off, cache, tok_off, B, heads, n_tok, head_dim, dtype);
  if (rc) return rc;
  return launched(launch_kv_quantize(p, dtype, (hipStream_t)hip_stream), "K/V quantise launch");
}

int orch_op_kv_dequantize(const orch_quantized_kv* cache, int tok_off, void* kv, size_t kv_bs, int kv_tokens,
                          int kv_off, int B, int heads, int n_tok, int head_dim, int dtype, void* hip_stream) {
  KvCacheParams p{};
  int rc = kv_params(&p, kv, kv_bs, kv_tokens, kv_off, cache, tok_off, B, heads, n_tok, head_dim, dtype);
  if (rc) return rc;
  return launched(launch_kv_dequantize(p, dtype, (hipStream_t)hip_stream), "K/V read-back launch");
}

// (a shape that the call refuses needs no workspace and has no plan)
static bool attention_shape(int B, int heads, int n_q, int n_kv, int head_dim, int dtype) {
  return B >= 1 && heads >= 1 && (long long)B * heads <= 32767 && n_q >= 0 && n_kv >= 1 && head_dim >= 1 &&
         (dtype == ORCH_F32 || dtype == ORCH_BF16) && (long long)n_q * head_dim < 1ll << 31 && (long long)n_kv * head_dim < 1ll << 31;
}

size_t orch_attention_quantized_workspace_bytes(int B, int heads, int n_q, int n_kv, int head_dim, int dtype) {
  if (!attention_shape(B, heads, n_q, n_kv, head_dim, dtype)) return 0;
  return attention_quantized_workspace_bytes(B, heads, n_q, n_kv, head_dim, dtype);
}

int orch_attention_quantized_plan(int B, int heads, int n_q, int n_kv, int head_dim, int dtype, size_t workspace_bytes,
                                  int* prepared, int* query_groups, int* key_parts) {
  if (!prepared || !query_groups || !key_parts) return fail("NULL pointer");
  if (!attention_shape(B, heads, n_q, n_kv, head_dim, dtype) || n_q < 1 ||
      !attention_quantized_plan(B, heads, n_q, n_kv, head_dim, dtype, workspace_bytes, prepared, query_groups, key_parts))
    return fail("bad shape");
  return ORCH_OK;
}

int orch_op_attention_quantized(const void* q, const orch_quantized_kv* cache, const void* kv_fresh, size_t fresh_bs,
                                int fresh_begin, int n_fresh, int B, int heads, int n_q, int head_dim, void* out,
                                void* workspace, size_t workspace_bytes, int dtype, void* hip_stream) {
  if ((n_q != 0 && (!q || !out)) || (n_fresh > 0 && !kv_fresh)) return fail("NULL pointer");
  int rc = check_common(B, heads, head_dim, dtype);
  if (rc) return rc;
  Runs values, exps;
  rc = check_cache(cache, B, heads, head_dim, &values, &exps);
  if (rc) return rc;
  if (n_q < 0 || n_fresh < 0 || fresh_begin < 0 || n_fresh > cache->tokens - fresh_begin)
    return fail("bad shape: %d queries, fresh keys [%d, %d + %d) of %d", n_q, fresh_begin, fresh_begin, n_fresh, cache->tokens);
  if ((long long)n_q * head_dim >= 1ll << 31) return fail("n_q * head_dim must be below 2^31");
  const size_t es = dtype == ORCH_BF16 ? 2 : 4, H = (size_t)heads * head_dim;
  const size_t fresh_elems = 2 * (size_t)n_fresh * H, q_bytes = (size_t)B * n_q * H * es;
  if (n_fresh > 0 && B > 1 && (fresh_bs < fresh_elems || fresh_bs >= kFar)) return fail("branch stride too small or past 2^40");
  if (!aligned16(q) || !aligned16(out) || (n_fresh > 0 && (!aligned16(kv_fresh) || (B > 1 && fresh_bs * es % 16))) ||
      (workspace && !aligned16(workspace)))
    return fail("device buffers must be 16-byte aligned");
  const size_t ws_used = workspace ? workspace_bytes : 0;
  const Runs o = {out, q_bytes, 0, 1}, w = {workspace, ws_used, 0, 1};
  const Runs in[] = {{q, q_bytes, 0, 1}, values, exps, {kv_fresh, fresh_elems * es, fresh_bs * es, B}};
  for (const Runs& r : in)
    if (overlap(r, o) || overlap(r, w)) return fail("out or workspace overlaps an input");
  if (overlap(w, o)) return fail("out and workspace overlap");
  AttnQParams p{};
  p.q = q; p.out = out; p.kv_fresh = kv_fresh; p.fresh_bs = fresh_bs; p.fresh_begin = fresh_begin; p.n_fresh = n_fresh;
  p.c.values = (unsigned char*)cache->values; p.c.exps = (unsigned char*)cache->exponents;
  p.c.values_bs = cache->values_stride; p.c.exps_bs = cache->exponents_stride; p.c.tokens = cache->tokens;
  p.B = B; p.heads = heads; p.n_q = n_q; p.d = head_dim;
  p.ws = ws_used ? workspace : nullptr;
  p.ws_bytes = ws_used;
  return launched(launch_attention_quantized(p, dtype, (hipStream_t)hip_stream), "attention launch");
}

}  // extern "C"
