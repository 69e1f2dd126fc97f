// C ABI of the norms around a block, the quantiser of rows and the 8-bit integer
// products: argument checks and launches.  Nothing here allocates or throws.
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

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// No stride is as long as this (elements); how far rows reach is checked beside it (Rows::far).
constexpr size_t kFar = (size_t)1 << 40;
constexpr int kMaxRows = 1 << 24, kMaxHidden = 32768, kMaxCols = 131071;
constexpr size_t kMaxInt8Stride = (size_t)1 << 23;

// `rows` rows of `bytes` bytes, `stride` bytes apart
struct Rows {
  const void* p;
  size_t rows, bytes, stride;
  size_t span() const { return rows ? (rows - 1) * stride + bytes : 0; }
  // Past 2^62 bytes, where no memory is: below it neither span() nor an offset wraps.
  bool far() const {
    size_t s;
    return p && rows > 1 && (__builtin_mul_overflow(rows - 1, stride, &s) || s >= (size_t)1 << 62);
  }
};

// Could a byte be of both?  Rows of one stride may lie between each other (two slices of a
// wider buffer); of different strides only apart.
bool overlap(const Rows& a, const Rows& b) {
  if (!a.p || !b.p || !a.rows || !b.rows || !a.bytes || !b.bytes) return false;
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (x + a.span() <= y || y + b.span() <= x) return false;
  if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {
    const size_t s = a.stride, d = y >= x ? (y - x) % s : (s - (x - y) % s) % s;
    return d < a.bytes || d + b.bytes > s;
  }
  return true;
}

bool same(const Rows& a, const Rows& b) { return a.p == b.p && (a.rows <= 1 || a.stride == b.stride); }

int check_type(int dtype) {
  return dtype == ORCH_F32 || dtype == ORCH_BF16 ? ORCH_OK : fail("bad dtype");
}

// int8 rows; where their values and scales lie
int check_int8(const orch_int8_rows* r, const char* name, int rows, int cols, Rows* values, Rows* scales, size_t* stride) {
  if (!r || !r->values || !r->scales) return fail("NULL %s", name);
  if (!aligned(r->values, 16) || !aligned(r->scales, 4)) return fail("%s: values must be 16-byte, scales 4-byte aligned", name);
  *stride = rows > 1 ? r->stride : ((size_t)cols + 15) / 16 * 16;
  if (*stride < (size_t)cols || *stride % 16 || *stride >= kMaxInt8Stride)
    return fail("%s: stride must be a multiple of 16, at least the row's bytes and below 2^23", name);
  *values = {r->values, (size_t)rows, (size_t)cols, *stride};
  *scales = {r->scales, 1, (size_t)rows * 4, 0};
  return ORCH_OK;
}

int check_norm(const orch_norm& n, const char* name) {
  if (n.kind != ORCH_NORM_NONE && n.kind != ORCH_NORM_LAYER && n.kind != ORCH_NORM_RMS) return fail("%s: bad kind", name);
  if (n.kind != ORCH_NORM_NONE && !(n.eps > 0.0f && std::isfinite(n.eps))) return fail("%s: eps must be finite and > 0", name);
  if (!aligned(n.weight, 4) || !aligned(n.bias, 4)) return fail("%s: weight and bias must be aligned to their elements", name);
  return ORCH_OK;
}

int check_product(const orch_int8_rows* A, int M, int K, const orch_int8_rows* W, int N, const float* bias, void* workspace,
                  size_t workspace_bytes, int dtype, GemmI8Params* p, Rows (&in)[6], Rows* ws) {
  if (int rc = check_type(dtype)) return rc;
  if (M < 0 || N < 1 || K < 1 || K > kMaxCols) return fail("bad shape: M >= 0, N >= 1, K of 1 .. %d", kMaxCols);
  if (((long long)M / 64 + 1) * ((long long)N / 64 + 1) >= 1ll << 24) return fail("bad shape: M * N too large");
  if (M == 0) return ORCH_OK;
  if (int rc = check_int8(A, "A", M, K, &in[0], &in[1], &p->lda)) return rc;
  if (int rc = check_int8(W, "W", N, K, &in[2], &in[3], &p->ldw)) return rc;
  if (!aligned(bias, 4)) return fail("bias must be aligned to its elements");
  if (workspace && !aligned(workspace, 16)) return fail("workspace must be 16-byte aligned");
  in[4] = {bias, 1, (size_t)N * 4, 0};
  *ws = {workspace, 1, workspace ? workspace_bytes : 0, 0};
  p->A = (const signed char*)A->values; p->W = (const signed char*)W->values;
  p->sa = A->scales; p->sw = W->scales;
  p->M = M; p->N = N; p->K = K; p->bias = bias;
  p->ws = ws->bytes ? (int*)workspace : nullptr;
  p->ws_elems = ws->bytes / 4;
  return ORCH_OK;
}

int check_outputs(const Rows* outs, int n, const Rows (&in)[6], const Rows& ws) {
  for (const Rows& r : in) {
    if (overlap(r, ws)) return fail("workspace overlaps an input");
    for (int i = 0; i < n; ++i)
      if (overlap(r, outs[i])) return fail("out overlaps an input");
  }
  for (int i = 0; i < n; ++i) {
    if (overlap(outs[i], ws)) return fail("out and workspace overlap");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail("the outputs overlap");
  }
  return ORCH_OK;
}

}  // namespace

extern "C" {

int orch_op_block_norms(const orch_block_norms* a, int dtype, void* hip_stream) {
  if (!a) return fail("NULL pointer");
  if (int rc = check_type(dtype)) return rc;
  const size_t es = dtype == ORCH_BF16 ? 2 : 4;
  const int rows = a->rows, H = a->hidden;
  const bool u = a->out || a->out8;
  if (rows < 0 || rows >= kMaxRows || H < 1 || H > kMaxHidden) return fail("bad shape: rows of 0 .. 2^24 - 1, hidden of 1 .. %d", kMaxHidden);
  if (!std::isfinite(a->residual_scale)) return fail("residual_scale must be finite");
  if (a->y)
    if (int rc = check_norm(a->post, "post")) return rc;
  if (u)
    if (int rc = check_norm(a->pre, "pre")) return rc;
  if (rows == 0) return ORCH_OK;
  if (!a->h) return fail("NULL pointer");
  if (!a->h_out && !u) return fail("nothing to write: h_out, out and out8 are NULL");
  if (a->out && a->out8) return fail("out and out8 exclude each other");
  const float* gate = a->y ? a->gate : nullptr;
  const float* shift = u ? a->shift : nullptr;
  const float* scale = u ? a->scale : nullptr;
  int branches = 1;
  if (gate || shift || scale) {
    if (a->rows_per_batch < 1) return fail("gate, shift and scale need rows_per_batch >= 1");
    branches = (rows - 1) / a->rows_per_batch + 1;
    if (branches > 1 && (a->mod_stride < (size_t)H || a->mod_stride >= kFar)) return fail("mod_stride must be at least hidden and below 2^40");
  }
  if (rows > 1)
    for (const auto& s : {a->h_stride, a->y ? a->y_stride : (size_t)H, a->h_out ? a->h_out_stride : (size_t)H,
                          a->out ? a->out_stride : (size_t)H})
      if (s < (size_t)H || s >= kFar) return fail("strides must be at least hidden and below 2^40");
  if (!aligned(a->h, 4) || !aligned(a->h_out, 4) || !aligned(gate, 4) || !aligned(shift, 4) || !aligned(scale, 4) ||
      !aligned(a->y, es) || !aligned(a->out, es))
    return fail("tensors must be aligned to their elements");
  BlockNormsParams p{};
  Rows codes{}, code_scales{};
  if (a->out8) {
    if (int rc = check_int8(a->out8, "out8", rows, H, &codes, &code_scales, &p.codes_stride)) return rc;
    p.codes = (signed char*)a->out8->values;
    p.code_scales = a->out8->scales;
  }
  const size_t n = rows, h4 = (size_t)H * 4, ms = branches > 1 ? a->mod_stride * 4 : 0;
  const Rows h = {a->h, n, h4, a->h_stride * 4}, y = {a->y, n, H * es, a->y_stride * es};
  const Rows h_out = {a->h_out, n, h4, a->h_out_stride * 4}, out = {a->out, n, H * es, a->out_stride * es};
  const Rows outs[] = {h_out, out, codes, code_scales};
  const orch_norm none{};
  const orch_norm &post = a->y ? a->post : none, &pre = u ? a->pre : none;
  for (const Rows& r : {h, y, h_out, out, Rows{gate ? gate : shift ? shift : scale, (size_t)branches, h4, ms}})
    if (r.far()) return fail("strides: rows reach past 64-bit addresses");
  const Rows in[] = {h, y, {gate, (size_t)branches, h4, ms}, {shift, (size_t)branches, h4, ms}, {scale, (size_t)branches, h4, ms},
                     {post.weight, 1, h4, 0}, {post.bias, 1, h4, 0}, {pre.weight, 1, h4, 0}, {pre.bias, 1, h4, 0}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 9; ++j) {
      const bool in_place = (i == 0 && j == 0 && same(outs[i], in[j])) || (i == 1 && j == 1 && same(outs[i], in[j]));
      if (!in_place && overlap(outs[i], in[j])) return fail("an output overlaps an input");
    }
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail("the outputs overlap");
  }
  p.h = a->h; p.y = a->y; p.h_out = a->h_out; p.out = a->out;
  p.gate = gate; p.shift = shift; p.scale = scale;
  // (the stride of a single row is never used)
  p.h_stride = n > 1 ? a->h_stride : 0; p.y_stride = n > 1 && a->y ? a->y_stride : 0;
  p.h_out_stride = n > 1 && a->h_out ? a->h_out_stride : 0; p.out_stride = n > 1 && a->out ? a->out_stride : 0;
  p.mod_stride = branches > 1 ? a->mod_stride : 0;
  p.post = {post.kind, post.eps, post.weight, post.bias};
  p.pre = {pre.kind, pre.eps, pre.weight, pre.bias};
  p.residual_scale = a->residual_scale;
  p.rows = rows; p.hidden = H; p.rows_per_batch = gate || shift || scale ? a->rows_per_batch : rows;
  return launched(launch_block_norms(p, dtype, (hipStream_t)hip_stream), "block norms launch");
}

int orch_op_quantize_rows(const void* x, size_t x_stride, int rows, int cols, const orch_int8_rows* out, int dtype,
                          void* hip_stream) {
  if (int rc = check_type(dtype)) return rc;
  if (rows < 0 || rows >= kMaxRows || cols < 1 || cols > kMaxCols) return fail("bad shape: rows of 0 .. 2^24 - 1, cols of 1 .. %d", kMaxCols);
  if (rows == 0) return ORCH_OK;
  if (!x) return fail("NULL pointer");
  const size_t es = dtype == ORCH_BF16 ? 2 : 4;
  if (rows > 1 && (x_stride < (size_t)cols || x_stride >= kFar)) return fail("x_stride must be at least cols and below 2^40");
  if (!aligned(x, es)) return fail("x must be aligned to its elements");
  QuantizeRowsParams p{};
  Rows values, scales;
  if (int rc = check_int8(out, "out", rows, cols, &values, &scales, &p.codes_stride)) return rc;
  const Rows in = {x, (size_t)rows, cols * es, x_stride * es};
  if (in.far()) return fail("x_stride: rows reach past 64-bit addresses");
  if (overlap(in, values) || overlap(in, scales) || overlap(values, scales)) return fail("x and out overlap");
  p.x = x; p.x_stride = rows > 1 ? x_stride : 0; p.rows = rows; p.cols = cols;
  p.codes = (signed char*)out->values; p.scales = out->scales;
  return launched(launch_quantize_rows(p, dtype, (hipStream_t)hip_stream), "quantise launch");
}

size_t orch_linear_quantized_workspace_bytes(int M, int N, int K) {
  if (M < 1 || N < 1 || K < 1 || K > kMaxCols || ((long long)M / 64 + 1) * ((long long)N / 64 + 1) >= 1ll << 24) return 0;
  return gemm_int8_workspace_bytes(M, N, K);
}

int orch_op_linear_quantized(const orch_int8_rows* A, int M, int K, const orch_int8_rows* W, int N, const float* bias, int epilogue,
                        const float* gate, size_t gate_stride, int rpb, void* out, void* workspace, size_t workspace_bytes,
                        int dtype, void* hip_stream) {
  GemmI8Params p{};
  Rows in[6] = {}, ws{};
  if (epilogue != ORCH_EPI_STORE && epilogue != ORCH_EPI_GELU && epilogue != ORCH_EPI_RESIDUAL) return fail("bad epilogue");
  if (int rc = check_product(A, M, K, W, N, bias, workspace, workspace_bytes, dtype, &p, in, &ws)) return rc;
  if (M == 0) return ORCH_OK;
  if (!out) return fail("NULL pointer");
  const bool res = epilogue == ORCH_EPI_RESIDUAL;
  const size_t es = dtype == ORCH_BF16 && !res ? 2 : 4;
  if (!aligned(out, es)) return fail("out must be aligned to its elements");
  if (res) {
    if (!gate || rpb < 1) return fail("the residual epilogue needs gate and rows_per_batch >= 1");
    const size_t branches = (M - 1) / rpb + 1;
    if (branches > 1 && (gate_stride < (size_t)N || gate_stride >= kFar)) return fail("gate_stride must be at least N and below 2^40");
    if (!aligned(gate, 4)) return fail("gate must be aligned to its elements");
    p.gate = gate; p.gate_stride = branches > 1 ? gate_stride : 0; p.rows_per_batch = rpb;
    in[5] = {gate, branches, (size_t)N * 4, gate_stride * 4};
    if (in[5].far()) return fail("gate_stride: rows reach past 64-bit addresses");
  }
  const Rows o = {out, 1, (size_t)M * N * es, 0};
  if (int rc = check_outputs(&o, 1, in, ws)) return rc;
  p.out = out;
  return launched(launch_gemm_int8(p, epilogue, dtype, (hipStream_t)hip_stream), "int8 product launch");
}

int orch_op_qkv_projection_quantized(const orch_int8_rows* A, int B, int n_tok, int K, const orch_int8_rows* W, const float* bias,
                                int heads, int head_dim, void* q_out, void* kv_out, size_t kv_bs, int kv_tokens,
                                int tok_offset, void* workspace, size_t workspace_bytes, int dtype, void* hip_stream) {
  GemmI8Params p{};
  Rows in[6] = {}, ws{};
  if (!(head_dim == 32 || head_dim == 64 || head_dim == 72 || head_dim == 80 || head_dim == 96 || head_dim == 128))
    return fail("head_dim %d not supported", head_dim);
  if (B < 1 || n_tok < 0 || heads < 1 || (long long)B * n_tok > 0x7fffffffll || (long long)heads * head_dim >= 65536)
    return fail("bad shape: B and heads must be >= 1, heads * head_dim below 65536");
  if (tok_offset < 0 || kv_tokens < 1 || n_tok > kv_tokens - tok_offset)
    return fail("tokens [%d, %d + %d) not within the buffer's %d", tok_offset, tok_offset, n_tok, kv_tokens);
  const int hidden = heads * head_dim;
  if (int rc = check_product(A, B * n_tok, K, W, 3 * hidden, bias, workspace, workspace_bytes, dtype, &p, in, &ws)) return rc;
  if (n_tok == 0) return ORCH_OK;
  if (!q_out || !kv_out) return fail("NULL pointer");
  const size_t es = dtype == ORCH_BF16 ? 2 : 4, branch = 2 * (size_t)kv_tokens * hidden;
  if (B > 1 && (kv_bs < branch || kv_bs >= kFar)) return fail("branch stride too small or past 2^40");
  if (!aligned(q_out, 16) || !aligned(kv_out, 16) || (B > 1 && kv_bs * es % 16)) return fail("q_out, kv_out and its branches must be 16-byte aligned");
  const Rows outs[] = {{q_out, 1, (size_t)B * n_tok * hidden * es, 0}, {kv_out, (size_t)B, branch * es, kv_bs * es}};
  if (outs[1].far()) return fail("branch stride: branches reach past 64-bit addresses");
  if (int rc = check_outputs(outs, 2, in, ws)) return rc;
  p.q = q_out; p.kv = kv_out; p.kv_bs = B > 1 ? kv_bs : 0; p.kv_tokens = kv_tokens; p.tok_offset = tok_offset;
  p.heads = heads; p.hidden = hidden; p.head_dim = head_dim; p.rows_per_batch = n_tok;
  return launched(launch_gemm_int8(p, kEpiQkv, dtype, (hipStream_t)hip_stream), "int8 qkv launch");
}

}  // extern "C"
