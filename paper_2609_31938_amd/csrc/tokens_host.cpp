// C-ABI host layer of the token operators: validation, workspaces, dispatch.
// Everything before a launch is host code; what lies on the device (lengths,
// page tables, positions) is bounds-checked by the kernels that read it.
#include <hip/hip_runtime.h>

#include <cmath>

#include "c3c_ctx.h"
#include "c3c_tokens.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

constexpr int64_t kBig = int64_t(1) << 31;
constexpr int64_t kMaxElems = int64_t(1) << 40;
constexpr int64_t kMaxK = 131071;  // 128 * 128 * K stays below 2^31

int elem_bytes(int dtype) {
  return dtype == C3C_DTYPE_BF16 || dtype == C3C_DTYPE_F16 ? 2 : dtype == C3C_DTYPE_F32 ? 4 : 0;
}

// elements of `rows` rows of `cols`, ld apart; -1 beyond the limit
int64_t extent(int64_t rows, int64_t cols, int64_t ld) {
  if (rows <= 0) return 0;
  if (rows > kMaxElems / ld) return -1;
  return (rows - 1) * ld + cols;
}

int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// One tensor of a call.
struct Span {
  const char* name;
  const void* p;
  int64_t bytes;
  int align;
};

// NULL (though not empty), misaligned: the message, or NULL if all is well.
const char* check_spans(const Span* s, int n) {
  for (int i = 0; i < n; ++i) {
    if (s[i].bytes > 0 && !s[i].p) return "a tensor is NULL";
    if (!aligned(s[i].p, s[i].align)) return "a tensor is not aligned";
  }
  return nullptr;
}

// outputs against inputs and one another, and the workspace against all
const char* check_overlap(const Span* in, int nin, const Span* out, int nout, const void* ws, int64_t wsb) {
  for (int i = 0; i < nout; ++i) {
    for (int j = 0; j < nin; ++j)
      if (overlap(out[i].p, out[i].bytes, in[j].p, in[j].bytes)) return "an output overlaps an input";
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return "two outputs overlap";
    if (overlap(ws, wsb, out[i].p, out[i].bytes)) return "the context's workspace overlaps a tensor";
  }
  for (int j = 0; j < nin; ++j)
    if (overlap(ws, wsb, in[j].p, in[j].bytes)) return "the context's workspace overlaps a tensor";
  return nullptr;
}

int done(c3c_ctx* ctx, hipError_t e) {
  return e == hipSuccess ? C3C_OK : fail(ctx, C3C_E_DEVICE, hipGetErrorString(e));
}

// ---------------------------------------------------------------- linear

const char* check_linear(const c3c_linear_desc* d) {
  if (!d) return "descriptor is NULL";
  if (d->M < 0 || d->N < 1 || d->K < 1) return "M must be >= 0, N and K >= 1";
  if (d->M >= kBig || d->N >= kBig || d->ld_x >= kBig) return "a size exceeds 2^31";
  if (d->K > kMaxK) return "K exceeds 131071: the int32 sum could overflow";
  if (d->ld_x < d->K) return "ld_x is less than K";
  if (d->x_dtype != C3C_DTYPE_I8 && !elem_bytes(d->x_dtype)) return "unknown x_dtype";
  if (!elem_bytes(d->y_dtype)) return "unknown y_dtype";
  if (extent(d->M, d->K, d->ld_x) < 0 || extent(d->M, d->N, d->N) < 0 || extent(d->N, d->K, d->K) < 0)
    return "a tensor exceeds 2^40 elements";
  return nullptr;
}

// Workspace of a call: the quantised rows (each padded to 16 bytes) and their
// scales, which it cannot do without; copies of w and of int8 x in rows of whole
// 16 bytes; the partial sums.
struct LinearSpace {
  int64_t ldq = 0, scale_at = 0, rows_bytes = 0;  // of float x
  int64_t w_at = 0, x_at = 0, pads_end = 0;       // w_at == x_at: no copy of w; x_at == pads_end: none of x
  int64_t part_at = 0;
  LinearPlan plan;
};
LinearSpace linear_space(const c3c_linear_desc& d) {
  LinearSpace s;
  s.plan = plan_linear_i8(d.M, d.N, d.K);
  const bool i8 = d.x_dtype == C3C_DTYPE_I8;
  s.ldq = round_up(d.K, 16);
  if (!i8 && d.M > 0) {
    s.scale_at = round_up(d.M * s.ldq, 256);
    s.rows_bytes = s.scale_at + round_up(d.M * 4, 256);
  }
  s.w_at = s.rows_bytes;
  s.x_at = s.w_at + (linear_pads(d.M, d.K, d.K) ? round_up(d.N * s.ldq, 256) : 0);
  s.pads_end = s.x_at + (i8 && linear_pads(d.M, d.K, d.ld_x) ? round_up(d.M * s.ldq, 256) : 0);
  s.part_at = s.pads_end;
  return s;
}

// ---------------------------------------------------------------- cache

const char* check_cache(const c3c_kv_cache* c, const c3c_kv_batch* b, int dtype, int64_t q_heads, bool need_q) {
  if (!c || !b) return "cache or batch is NULL";
  if (!elem_bytes(dtype)) return "unknown dtype";
  if (c->pages < 0 || c->pages >= kBig || c->heads < 1 || c->heads >= kBig) return "pages must be >= 0, heads >= 1";
  // grids have 65535 places for heads and for sequences
  if (c->heads > 65535 || q_heads > 65535 || b->B > 65535) return "heads, q_heads and B must be at most 65535";
  if (c->page < 16 || c->page % 16 || c->page >= kBig) return "page must be a multiple of 16";
  if (c->dim < 16 || c->dim > 256 || c->dim % 16) return "dim must be a multiple of 16, at most 256";
  if (b->B < 0 || b->B >= kBig || b->T < 0 || b->T >= kBig || b->cols < 0 || b->cols >= kBig)
    return "B, T and cols must be >= 0 and below 2^31";
  if (b->max_new < 0 || b->max_new >= kBig || b->max_len < 0 || b->max_len >= kBig)
    return "max_new and max_len must be >= 0 and below 2^31";
  if (b->T > 0 && b->max_new < 1) return "max_new is 0, but there are new tokens";
  if (b->T > 0 && b->B < 1) return "new tokens of no sequence";
  if (need_q && (q_heads < 1 || q_heads >= kBig)) return "q_heads must be >= 1";
  const int64_t row = c->heads * c->dim;
  if (row >= kBig || q_heads * c->dim >= kBig) return "heads * dim exceeds 2^31";
  if (c->pages > 0 && c->pages > kMaxElems / c->page / row) return "the cache exceeds 2^40 elements";
  if (b->cols > 0 && b->B > kMaxElems / b->cols) return "the page table exceeds 2^40 elements";
  return nullptr;
}

// spans of the cache (4) and of the batch (3)
void cache_spans(const c3c_kv_cache& c, Span* s) {
  const int64_t codes = c.pages * c.heads * c.page * c.dim, scales = c.pages * c.heads * (c.page / 16) * 4;
  s[0] = {"k", c.k, codes, 16};
  s[1] = {"v", c.v, codes, 16};
  s[2] = {"k_scale", c.k_scale, scales, 4};
  s[3] = {"v_scale", c.v_scale, scales, 4};
}
void batch_spans(const c3c_kv_batch& b, Span* s) {
  s[0] = {"table", b.table, b.B * b.cols * 4, 4};
  s[1] = {"cu", b.cu, b.B > 0 ? (b.B + 1) * 4 : 0, 4};
  s[2] = {"len", b.len, b.B * 4, 4};
}

}  // namespace
}  // namespace c3c

using namespace c3c;

extern "C" {

int c3c_quantize_rows(c3c_ctx* ctx, int64_t T, int64_t C, int64_t ld_x, int dtype, const void* x,
                      int8_t* q, float* scale, void* stream) {
  if (!ctx) return C3C_E_INVAL;
  const int es = elem_bytes(dtype);
  if (!es) return fail(ctx, C3C_E_INVAL, "unknown dtype");
  if (T < 0 || C < 1 || ld_x < C || T >= kBig || C >= kBig || ld_x >= kBig)
    return fail(ctx, C3C_E_INVAL, "T must be >= 0, C >= 1, ld_x >= C, all below 2^31");
  if (extent(T, C, ld_x) < 0) return fail(ctx, C3C_E_INVAL, "x exceeds 2^40 elements");
  const Span in[] = {{"x", x, extent(T, C, ld_x) * es, es}};
  const Span out[] = {{"q", q, T * C, 1}, {"scale", scale, T * 4, 4}};
  const char* why = check_spans(in, 1);
  if (!why) why = check_spans(out, 2);
  if (!why) why = check_overlap(in, 1, out, 2, nullptr, 0);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  return done(ctx, launch_quantize_rows(T, C, ld_x, dtype, x, q, C, scale, static_cast<hipStream_t>(stream)));
}

int c3c_linear_i8_workspace_bytes(const c3c_linear_desc* d, size_t* bytes) {
  if (!bytes || check_linear(d)) return C3C_E_INVAL;
  const LinearSpace s = linear_space(*d);
  *bytes = static_cast<size_t>(s.part_at + s.plan.part_bytes);
  return C3C_OK;
}

int c3c_linear_i8(c3c_ctx* ctx, const c3c_linear_desc* d, const void* x, const float* x_scale,
                  const int8_t* w, const float* w_scale, const float* bias, void* y, void* stream) {
  if (!ctx) return C3C_E_INVAL;
  const char* why = check_linear(d);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  const bool i8 = d->x_dtype == C3C_DTYPE_I8;
  const int xs = i8 ? 1 : elem_bytes(d->x_dtype), ys = elem_bytes(d->y_dtype);
  if (i8 ? !x_scale && d->M > 0 : x_scale != nullptr)
    return fail(ctx, C3C_E_INVAL, "x_scale goes with int8 x, and with it alone");
  const Span in[] = {{"x", x, extent(d->M, d->K, d->ld_x) * xs, xs},
                     {"x_scale", x_scale, x_scale ? d->M * 4 : 0, 4},
                     {"w", w, d->N * d->K, 1},
                     {"w_scale", w_scale, d->N * 4, 4},
                     {"bias", bias, bias ? d->N * 4 : 0, 4}};
  const Span out[] = {{"y", y, d->M * d->N * ys, ys}};
  why = check_spans(in, 5);
  if (!why) why = check_spans(out, 1);
  if (!why) why = check_overlap(in, 5, out, 1, ctx->ws, static_cast<int64_t>(ctx->ws_bytes));
  if (why) return fail(ctx, C3C_E_INVAL, why);
  const LinearSpace sp = linear_space(*d);
  const int64_t have = static_cast<int64_t>(ctx->ws_bytes);
  if (sp.rows_bytes > have)
    return fail(ctx, C3C_E_INVAL, "the context's workspace is smaller than the quantised rows need");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!i8 && linear_quantises(d->M, d->K))
    return done(ctx, launch_linear_float(d->M, d->N, d->K, x, d->ld_x, d->x_dtype, w, w_scale, bias, y, d->y_dtype, s));
  unsigned char* ws = static_cast<unsigned char*>(ctx->ws);
  const int8_t* rows = static_cast<const int8_t*>(x);
  int64_t ld = d->ld_x;
  if (!i8 && d->M > 0) {
    int8_t* q = reinterpret_cast<int8_t*>(ws);
    float* scale = reinterpret_cast<float*>(ws + sp.scale_at);
    const hipError_t e = launch_quantize_rows(d->M, d->K, d->ld_x, d->x_dtype, x, q, sp.ldq, scale, s);
    if (e != hipSuccess) return done(ctx, e);
    rows = q;
    x_scale = scale;
    ld = sp.ldq;
  }
  const int8_t* weights = w;
  int64_t K = d->K;
  if (sp.pads_end > sp.w_at && sp.pads_end <= have) {
    // both operands in rows of whole 16 bytes, zero past K
    hipError_t e = hipSuccess;
    if (sp.x_at > sp.w_at) {
      int8_t* to = reinterpret_cast<int8_t*>(ws + sp.w_at);
      e = launch_pad_rows(w, d->N, d->K, d->K, to, sp.ldq, s);
      weights = to;
      K = sp.ldq;
    }
    if (e == hipSuccess && sp.pads_end > sp.x_at) {
      int8_t* to = reinterpret_cast<int8_t*>(ws + sp.x_at);
      e = launch_pad_rows(rows, d->M, d->K, ld, to, sp.ldq, s);
      rows = to;
      ld = sp.ldq;
    }
    if (e != hipSuccess) return done(ctx, e);
  }
  int32_t* part = sp.plan.splits > 1 && sp.part_at + sp.plan.part_bytes <= have
                      ? reinterpret_cast<int32_t*>(ws + sp.part_at)
                      : nullptr;
  return done(ctx, launch_linear_i8(d->M, d->N, K, rows, ld, x_scale, weights, w_scale, bias, y, d->y_dtype,
                                    sp.plan, part, s));
}

int c3c_norm_gate(c3c_ctx* ctx, const c3c_norm_desc* d, const void* h, const void* y,
                  const void* gate, const float* post, const float* pre, void* h_out, void* u,
                  int8_t* u_q, float* u_scale, void* stream) {
  if (!ctx) return C3C_E_INVAL;
  if (!d) return fail(ctx, C3C_E_INVAL, "descriptor is NULL");
  const int es = elem_bytes(d->dtype);
  if (!es) return fail(ctx, C3C_E_INVAL, "unknown dtype");
  if (d->T < 0 || d->C < 1 || d->T >= kBig || d->C >= kBig || extent(d->T, d->C, d->C) < 0)
    return fail(ctx, C3C_E_INVAL, "T must be >= 0, C >= 1, T * C at most 2^40");
  if (gate && d->rows_per_gate < 1) return fail(ctx, C3C_E_INVAL, "rows_per_gate must be >= 1");
  if (!std::isfinite(d->alpha) || !std::isfinite(d->eps) || d->eps < 0.f)
    return fail(ctx, C3C_E_INVAL, "alpha and eps must be finite, eps >= 0");
  if (d->T == 0) return C3C_OK;  // tensors of no elements have no address
  if (!y && (post || gate)) return fail(ctx, C3C_E_INVAL, "post and gate go with y");
  if (pre ? !u && !u_q : u || u_q || u_scale) return fail(ctx, C3C_E_INVAL, "u or u_q goes with pre, and with it alone");
  if (!u_q != !u_scale) return fail(ctx, C3C_E_INVAL, "u_q and u_scale go together");
  if (!h_out && !pre) return fail(ctx, C3C_E_INVAL, "no output is asked for");
  const int64_t n = d->T * d->C, groups = gate && d->T > 0 ? (d->T - 1) / d->rows_per_gate + 1 : 0;
  const Span in[] = {{"h", h == h_out ? nullptr : h, h == h_out ? 0 : n * es, es},
                     {"y", y, y ? n * es : 0, es},
                     {"gate", gate, groups * d->C * es, es},
                     {"post", post, post ? d->C * 4 : 0, 4},
                     {"pre", pre, pre ? d->C * 4 : 0, 4}};
  const Span out[] = {{"h_out", h_out, h_out ? n * es : 0, es},
                      {"u", u, u ? n * es : 0, es},
                      {"u_q", u_q, u_q ? n : 0, 1},
                      {"u_scale", u_scale, u_scale ? d->T * 4 : 0, 4}};
  if (n > 0 && !h) return fail(ctx, C3C_E_INVAL, "h is NULL");
  const char* why = check_spans(in, 5);
  if (!why) why = check_spans(out, 4);
  if (!why) why = check_overlap(in, 5, out, 4, nullptr, 0);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  return done(ctx, launch_norm_gate(*d, h, y, gate, post, pre, h_out, u, u_q, u_scale, static_cast<hipStream_t>(stream)));
}

int c3c_kv_append(c3c_ctx* ctx, const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                  const c3c_rope* rope, int dtype, int64_t q_heads, const void* q, int64_t ld_q,
                  const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* q_out,
                  void* stream) {
  if (!ctx) return C3C_E_INVAL;
  const char* why = check_cache(cache, batch, dtype, q ? q_heads : 0, q != nullptr);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  const int es = elem_bytes(dtype);
  const int64_t T = batch->T, row = cache->heads * cache->dim, qrow = q ? q_heads * cache->dim : 0;
  if (ld_k < row || ld_v < row || ld_k >= kBig || ld_v >= kBig || (q && (ld_q < qrow || ld_q >= kBig)))
    return fail(ctx, C3C_E_INVAL, "a token stride is less than its heads or exceeds 2^31");
  if (!q != !q_out && T > 0) return fail(ctx, C3C_E_INVAL, "q and q_out go together");
  if (q && q == q_out && ld_q != qrow) return fail(ctx, C3C_E_INVAL, "q in place needs contiguous tokens");
  if (extent(T, row, ld_k) < 0 || extent(T, row, ld_v) < 0 || (q && extent(T, qrow, ld_q) < 0))
    return fail(ctx, C3C_E_INVAL, "a tensor exceeds 2^40 elements");
  if (rope) {
    if (rope->rot < 0 || rope->rot % 2 || rope->rot > cache->dim || rope->rows < 0 || rope->rows >= kBig)
      return fail(ctx, C3C_E_INVAL, "rot must be even and at most dim, rows >= 0 and below 2^31");
    if (rope->pairs != 0 && rope->pairs != 1) return fail(ctx, C3C_E_INVAL, "pairs must be 0 or 1");
    if (rope->rot > 0 && rope->rows < 1 && T > 0) return fail(ctx, C3C_E_INVAL, "the angle table is empty");
  }
  const bool turn = rope && rope->rot > 0;
  Span in[9], out[5];
  batch_spans(*batch, in);
  in[3] = {"k", k, extent(T, row, ld_k) * es, es};
  in[4] = {"v", v, extent(T, row, ld_v) * es, es};
  in[5] = {"q", q == q_out ? nullptr : q, q && q != q_out ? extent(T, qrow, ld_q) * es : 0, es};
  in[6] = {"cos", turn ? rope->cos : nullptr, turn ? rope->rows * (rope->rot / 2) * 4 : 0, 4};
  in[7] = {"sin", turn ? rope->sin : nullptr, turn ? rope->rows * (rope->rot / 2) * 4 : 0, 4};
  in[8] = {"pos", turn ? rope->pos : nullptr, turn && rope->pos ? T * 4 : 0, 4};
  cache_spans(*cache, out);
  out[4] = {"q_out", q_out, q ? T * qrow * es : 0, es};
  why = check_spans(in, 9);
  if (!why) why = check_spans(out, 5);
  if (!why) why = check_overlap(in, 9, out, 5, nullptr, 0);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  AppendArgs a{*cache, *batch, turn ? *rope : c3c_rope{}, q, k, v, q_out, q ? q_heads : 0, ld_q, ld_k, ld_v};
  return done(ctx, launch_kv_append(a, dtype, static_cast<hipStream_t>(stream)));
}

int c3c_paged_attention_workspace_bytes(const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                                        int dtype, int64_t q_heads, int causal, int64_t window,
                                        size_t* bytes) {
  if (!bytes || check_cache(cache, batch, dtype, q_heads, true) || q_heads % cache->heads ||
      (causal != 0 && causal != 1) || window < 0 || window >= kBig)
    return C3C_E_INVAL;
  *bytes = static_cast<size_t>(plan_attend(*cache, *batch, dtype, q_heads, causal, window).part_bytes);
  return C3C_OK;
}

int c3c_paged_attention(c3c_ctx* ctx, const c3c_kv_cache* cache, const c3c_kv_batch* batch,
                        int dtype, int64_t q_heads, const void* q, int64_t ld_q, float scale,
                        int causal, int64_t window, void* out, float* lse, void* stream) {
  if (!ctx) return C3C_E_INVAL;
  const char* why = check_cache(cache, batch, dtype, q_heads, true);
  if (why) return fail(ctx, C3C_E_INVAL, why);
  if (q_heads % cache->heads) return fail(ctx, C3C_E_INVAL, "heads must divide q_heads");
  if (batch->T * (q_heads / cache->heads) >= kBig - 2048)
    return fail(ctx, C3C_E_INVAL, "T * q_heads / heads must be below 2^31 - 2048");
  if (!std::isfinite(scale) || scale <= 0.f) return fail(ctx, C3C_E_INVAL, "scale must be finite and positive");
  if (causal != 0 && causal != 1) return fail(ctx, C3C_E_INVAL, "causal must be 0 or 1");
  if (window < 0 || window >= kBig) return fail(ctx, C3C_E_INVAL, "window must be >= 0 and below 2^31");
  const int es = elem_bytes(dtype);
  const int64_t T = batch->T, qrow = q_heads * cache->dim;
  if (ld_q < qrow || ld_q >= kBig) return fail(ctx, C3C_E_INVAL, "ld_q is less than q_heads * dim or exceeds 2^31");
  if (extent(T, qrow, ld_q) < 0) return fail(ctx, C3C_E_INVAL, "q exceeds 2^40 elements");
  Span in[8], o[2];
  batch_spans(*batch, in);
  cache_spans(*cache, in + 3);
  in[7] = {"q", q, extent(T, qrow, ld_q) * es, es};
  o[0] = {"out", out, T * qrow * es, es};
  o[1] = {"lse", lse, lse ? T * q_heads * 4 : 0, 4};
  why = check_spans(in, 8);
  if (!why) why = check_spans(o, 2);
  if (!why) why = check_overlap(in, 8, o, 2, ctx->ws, static_cast<int64_t>(ctx->ws_bytes));
  if (why) return fail(ctx, C3C_E_INVAL, why);
  AttendPlan plan = plan_attend(*cache, *batch, dtype, q_heads, causal, window);
  AttendArgs a{*cache, *batch, q, out, lse, static_cast<float*>(ctx->ws), q_heads, ld_q, window, scale, causal};
  if (plan.part_bytes > static_cast<int64_t>(ctx->ws_bytes)) plan = AttendPlan{};
  return done(ctx, launch_attend(a, dtype, plan, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
