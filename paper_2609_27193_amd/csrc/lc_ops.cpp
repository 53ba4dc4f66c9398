// Entry points of the training operators: embedding, norms, kept activations
// and the linear weight gradient.  Host only: everything is checked before
// anything is enqueued, and the workspace is the caller's, so a call allocates
// nothing and may be captured into a graph.
#include <hip/hip_runtime.h>

#include <cmath>

#include "layercheck.h"
#include "lc_ctx.h"
#include "lc_ops.h"
#include "lc_trace.h"

using namespace lc;

namespace {

constexpr uint64_t kMaxRows = 1ull << 31;
constexpr uint64_t kMaxCols = 1ull << 30;
constexpr uint64_t kMaxSpan = 1ull << 46;  // bytes between the first and the last element
constexpr uint32_t kSpaceAlign = 16;

uint32_t esz_of(int dtype) { return dtype == LC_DT_BF16 ? 2 : 4; }
bool dtype_ok(int dtype) { return dtype == LC_DT_BF16 || dtype == LC_DT_F32; }
uint64_t addr(const void* p) { return reinterpret_cast<uint64_t>(p); }

lc_status check_matrix(const char* name, const lc_matrix* m) {
  if (!m) return fail(LC_ERR_INVALID_ARG, "%s is NULL", name);
  if (!dtype_ok(m->dtype)) return fail(LC_ERR_INVALID_ARG, "%s: unknown dtype %d", name, m->dtype);
  if (m->reserved != 0) return fail(LC_ERR_INVALID_ARG, "%s: reserved field must be 0", name);
  if (m->cols == 0 || m->cols > kMaxCols)
    return fail(LC_ERR_INVALID_ARG, "%s: %llu columns", name, static_cast<unsigned long long>(m->cols));
  if (m->rows > kMaxRows)
    return fail(LC_ERR_INVALID_ARG, "%s: %llu rows", name, static_cast<unsigned long long>(m->rows));
  if (m->rows > 1 && (m->stride < m->cols || m->stride > kMaxSpan / (4 * m->rows)))
    return fail(LC_ERR_INVALID_ARG, "%s: stride %llu", name, static_cast<unsigned long long>(m->stride));
  if (m->rows == 0) return LC_OK;  // holds nothing: data may be NULL
  if (!m->data) return fail(LC_ERR_INVALID_ARG, "%s: data is NULL", name);
  if (addr(m->data) % esz_of(m->dtype)) return fail(LC_ERR_INVALID_ARG, "%s: data is misaligned", name);
  return LC_OK;
}

lc_status check_saved(const char* name, const lc_saved_act* s) {
  if (!s) return fail(LC_ERR_INVALID_ARG, "%s is NULL", name);
  if (s->cols == 0 || s->cols > kMaxCols)
    return fail(LC_ERR_INVALID_ARG, "%s: %llu columns", name, static_cast<unsigned long long>(s->cols));
  if (s->rows > kMaxRows)
    return fail(LC_ERR_INVALID_ARG, "%s: %llu rows", name, static_cast<unsigned long long>(s->rows));
  const uint64_t blocks = (s->cols + kActBlock - 1) / kActBlock;
  if (s->rows > 1 && (s->code_stride < s->cols || s->code_stride > kMaxSpan / s->rows))
    return fail(LC_ERR_INVALID_ARG, "%s: code_stride %llu", name, static_cast<unsigned long long>(s->code_stride));
  if (s->rows > 1 && (s->scale_stride < blocks || s->scale_stride > kMaxSpan / s->rows))
    return fail(LC_ERR_INVALID_ARG, "%s: scale_stride %llu", name, static_cast<unsigned long long>(s->scale_stride));
  if (s->rows > 0 && (!s->codes || !s->scales)) return fail(LC_ERR_INVALID_ARG, "%s: codes or scales is NULL", name);
  return LC_OK;
}

lc_status check_shape(const char* name, uint64_t rows, uint64_t cols, uint64_t want_rows, uint64_t want_cols) {
  if (rows == want_rows && cols == want_cols) return LC_OK;
  return fail(LC_ERR_INVALID_ARG, "%s is %llu x %llu, not %llu x %llu", name, static_cast<unsigned long long>(rows),
              static_cast<unsigned long long>(cols), static_cast<unsigned long long>(want_rows),
              static_cast<unsigned long long>(want_cols));
}

// Rows of bytes in memory, for the check that what a call writes shares no
// byte with anything else that it touches.
struct Area {
  const char* name;
  uint64_t base, rows, width, pitch;  // bytes; rows 0: nothing
};
Area area_of(const char* name, const lc_matrix* m) {
  if (!m) return {name, 0, 0, 0, 0};
  const uint64_t e = esz_of(m->dtype);
  return {name, addr(m->data), m->rows, m->cols * e, m->stride * e};
}
Area codes_of(const lc_saved_act* s) {
  if (!s) return {"codes", 0, 0, 0, 0};
  return {"codes", addr(s->codes), s->rows, s->cols, s->code_stride};
}
Area scales_of(const lc_saved_act* s) {
  if (!s) return {"scales", 0, 0, 0, 0};
  return {"scales", addr(s->scales), s->rows, (s->cols + kActBlock - 1) / kActBlock, s->scale_stride};
}
Area flat(const char* name, const void* p, uint64_t bytes) { return {name, addr(p), p && bytes ? 1u : 0u, bytes, bytes}; }

bool overlap(const Area& a, const Area& b) {
  if (!a.rows || !b.rows) return false;
  const uint64_t a_end = a.base + (a.rows - 1) * a.pitch + a.width, b_end = b.base + (b.rows - 1) * b.pitch + b.width;
  if (a_end <= b.base || b_end <= a.base) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  // columns beside each other in one buffer; a single row or a vector has the pitch of the rows beside it
  const uint64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
  if (b.rows > 1 && b.pitch != pitch) return true;
  const uint64_t off = b.base >= a.base ? (b.base - a.base) % pitch : (pitch - (a.base - b.base) % pitch) % pitch;
  return off < a.width || off + b.width > pitch;
}

// The first n_out areas are written.
template <size_t N>
lc_status check_apart(const Area (&areas)[N], size_t n_out) {
  for (size_t i = 0; i < n_out; ++i)
    for (size_t j = i + 1; j < N; ++j)
      if (overlap(areas[i], areas[j]))
        return fail(LC_ERR_INVALID_ARG, "%s and %s overlap in memory", areas[i].name, areas[j].name);
  return LC_OK;
}

lc_status check_tokens(const void* tokens, int32_t dtype, uint64_t n) {
  if (dtype != LC_IT_I32 && dtype != LC_IT_I64) return fail(LC_ERR_INVALID_ARG, "unknown token dtype %d", dtype);
  if (n > kMaxRows) return fail(LC_ERR_INVALID_ARG, "%llu tokens", static_cast<unsigned long long>(n));
  if (n && !tokens) return fail(LC_ERR_INVALID_ARG, "tokens is NULL");
  if (addr(tokens) % (dtype == LC_IT_I64 ? 8 : 4)) return fail(LC_ERR_INVALID_ARG, "tokens is misaligned");
  return LC_OK;
}

lc_status check_flag(const char* name, int32_t v) {
  return v == 0 || v == 1 ? LC_OK : fail(LC_ERR_INVALID_ARG, "%s must be 0 or 1", name);
}

lc_status check_vector(const char* name, const void* p, uint32_t align) {
  return addr(p) % align ? fail(LC_ERR_INVALID_ARG, "%s is misaligned", name) : LC_OK;
}

lc_status check_space(const void* workspace, uint64_t bytes, uint64_t need) {
  if (need == 0) return LC_OK;
  if (!workspace) return fail(LC_ERR_INVALID_ARG, "workspace is NULL");
  if (addr(workspace) % kSpaceAlign) return fail(LC_ERR_INVALID_ARG, "workspace is not %u-byte aligned", kSpaceAlign);
  if (bytes < need)
    return fail(LC_ERR_CAPACITY, "workspace of %llu bytes, %llu are needed", static_cast<unsigned long long>(bytes),
                static_cast<unsigned long long>(need));
  return LC_OK;
}

// The kernels go to the stream's device, which has to be the current one.
lc_status check_stream(void* stream) {
  if (!stream) return LC_OK;
  int dev = -1, sdev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return fail(LC_ERR_HIP, "no HIP device");
  }
  if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &sdev) != hipSuccess) {
    (void)hipGetLastError();
    return fail(LC_ERR_INVALID_ARG, "stream is not a HIP stream");
  }
  if (sdev != dev) return fail(LC_ERR_INVALID_ARG, "the stream belongs to device %d, not the current %d", sdev, dev);
  return LC_OK;
}

lc_status launched(const char* func, hipError_t e) {
  return e == hipSuccess ? LC_OK : fail(LC_ERR_HIP, "%s: %s", func, hipGetErrorString(e));
}

// A single row's strides are the caller's to leave unset; the kernels reckon
// with those of rows that follow it closely.
Rows rows_of(const lc_matrix* m) { return m ? Rows{addr(m->data), m->rows > 1 ? m->stride : m->cols} : Rows{0, 0}; }
Kept kept_of(const lc_saved_act* s) {
  if (!s) return Kept{0, 0, 0, 0};
  const bool many = s->rows > 1;
  return Kept{addr(s->codes), addr(s->scales), many ? s->code_stride : s->cols,
              many ? s->scale_stride : (s->cols + kActBlock - 1) / kActBlock};
}

lc_status check_norm(const lc_norm_params* p) {
  if (!p) return fail(LC_ERR_INVALID_ARG, "params is NULL");
  if (p->kind != LC_NORM_LAYER && p->kind != LC_NORM_RMS) return fail(LC_ERR_INVALID_ARG, "unknown norm kind %d", p->kind);
  if (!dtype_ok(p->param_dtype)) return fail(LC_ERR_INVALID_ARG, "unknown param dtype %d", p->param_dtype);
  if (p->bias && p->kind == LC_NORM_RMS) return fail(LC_ERR_INVALID_ARG, "LC_NORM_RMS has no bias");
  if (!(p->eps >= 0.0) || !std::isfinite(p->eps)) return fail(LC_ERR_INVALID_ARG, "eps must be finite and >= 0");
  lc_status st = check_vector("weight", p->weight, esz_of(p->param_dtype));
  return st != LC_OK ? st : check_vector("bias", p->bias, esz_of(p->param_dtype));
}

}  // namespace

#define LC_CHECK(call)                         \
  do {                                         \
    const lc_status st_ = (call);              \
    if (st_ != LC_OK) return st_;              \
  } while (0)

extern "C" lc_status lc_embedding_forward(const lc_matrix* weight, const void* tokens, int32_t token_dtype,
                                          uint64_t n_tokens, int64_t first_token, double scale, const lc_matrix* out,
                                          void* stream) {
  lc::TraceRange trace_("lc_embedding_forward");
  LC_CHECK(check_matrix("weight", weight));
  LC_CHECK(check_matrix("out", out));
  LC_CHECK(check_tokens(tokens, token_dtype, n_tokens));
  LC_CHECK(check_shape("out", out->rows, out->cols, n_tokens, weight->cols));
  const Area areas[] = {area_of("out", out), area_of("weight", weight),
                        flat("tokens", tokens, n_tokens * (token_dtype == LC_IT_I64 ? 8 : 4))};
  LC_CHECK(check_apart(areas, 1));
  LC_CHECK(check_stream(stream));
  if (n_tokens == 0) return LC_OK;
  EmbedFwd a{};
  a.w = rows_of(weight);
  a.out = rows_of(out);
  a.tokens = addr(tokens);
  a.n = n_tokens;
  a.first = first_token;
  a.vocab = weight->rows;
  a.dim = static_cast<uint32_t>(weight->cols);
  a.scale = static_cast<float>(scale);
  a.w_dtype = weight->dtype;
  a.out_dtype = out->dtype;
  a.token64 = token_dtype == LC_IT_I64;
  return launched("lc_embedding_forward", launch_embed_fwd(a, static_cast<hipStream_t>(stream)));
}

extern "C" uint64_t lc_embedding_backward_workspace(uint64_t n_tokens, uint64_t cols) {
  return n_tokens > kMaxRows || cols == 0 || cols > kMaxCols ? 0 : embed_bwd_workspace(n_tokens, cols);
}

extern "C" lc_status lc_embedding_backward(const lc_matrix* dout, const void* tokens, int32_t token_dtype,
                                           uint64_t n_tokens, int64_t first_token, double scale, int32_t accumulate,
                                           const lc_matrix* dweight, void* workspace, uint64_t workspace_bytes,
                                           void* stream) {
  lc::TraceRange trace_("lc_embedding_backward");
  LC_CHECK(check_matrix("dout", dout));
  LC_CHECK(check_matrix("dweight", dweight));
  LC_CHECK(check_tokens(tokens, token_dtype, n_tokens));
  LC_CHECK(check_flag("accumulate", accumulate));
  LC_CHECK(check_shape("dout", dout->rows, dout->cols, n_tokens, dweight->cols));
  const uint64_t need = embed_bwd_workspace(n_tokens, dweight->cols);
  LC_CHECK(check_space(workspace, workspace_bytes, need));
  const Area areas[] = {area_of("dweight", dweight), flat("workspace", workspace, need), area_of("dout", dout),
                        flat("tokens", tokens, n_tokens * (token_dtype == LC_IT_I64 ? 8 : 4))};
  LC_CHECK(check_apart(areas, 2));
  LC_CHECK(check_stream(stream));
  if (dweight->rows == 0) return LC_OK;
  EmbedBwd a{};
  a.dout = rows_of(dout);
  a.dw = rows_of(dweight);
  a.tokens = addr(tokens);
  a.n = n_tokens;
  a.first = first_token;
  a.vocab = dweight->rows;
  a.dim = static_cast<uint32_t>(dweight->cols);
  a.scale = static_cast<float>(scale);
  a.dout_dtype = dout->dtype;
  a.dw_dtype = dweight->dtype;
  a.token64 = token_dtype == LC_IT_I64;
  a.accumulate = accumulate;
  a.ws = static_cast<uint8_t*>(workspace);
  return launched("lc_embedding_backward", launch_embed_bwd(a, static_cast<hipStream_t>(stream)));
}

extern "C" lc_status lc_norm_forward(const lc_norm_params* params, const lc_matrix* x, const lc_matrix* y, float* mean,
                                     float* rstd, const lc_saved_act* saved, void* stream) {
  lc::TraceRange trace_("lc_norm_forward");
  LC_CHECK(check_norm(params));
  LC_CHECK(check_matrix("x", x));
  LC_CHECK(check_matrix("y", y));
  LC_CHECK(check_shape("y", y->rows, y->cols, x->rows, x->cols));
  if (y->dtype != x->dtype) return fail(LC_ERR_INVALID_ARG, "y has another dtype than x");
  if (mean && params->kind == LC_NORM_RMS) return fail(LC_ERR_INVALID_ARG, "LC_NORM_RMS has no mean");
  LC_CHECK(check_vector("mean", mean, 4));
  LC_CHECK(check_vector("rstd", rstd, 4));
  if (saved) {
    LC_CHECK(check_saved("saved", saved));
    LC_CHECK(check_shape("saved", saved->rows, saved->cols, x->rows, x->cols));
  }
  const uint64_t param_bytes = x->cols * esz_of(params->param_dtype);
  const Area areas[] = {area_of("y", y), flat("mean", mean, x->rows * 4), flat("rstd", rstd, x->rows * 4),
                        codes_of(saved), scales_of(saved), area_of("x", x), flat("weight", params->weight, param_bytes),
                        flat("bias", params->bias, param_bytes)};
  LC_CHECK(check_apart(areas, 5));
  LC_CHECK(check_stream(stream));
  NormFwd a{};
  a.x = rows_of(x);
  a.y = rows_of(y);
  a.kept = kept_of(saved);
  a.weight = addr(params->weight);
  a.bias = addr(params->bias);
  a.mean = mean;
  a.rstd = rstd;
  a.rows = x->rows;
  a.dim = static_cast<uint32_t>(x->cols);
  a.eps = static_cast<float>(params->eps);
  a.dtype = x->dtype;
  a.param_dtype = params->param_dtype;
  a.layer = params->kind == LC_NORM_LAYER;
  return launched("lc_norm_forward", launch_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

extern "C" uint64_t lc_norm_backward_workspace(uint64_t rows, uint64_t cols) {
  return rows > kMaxRows || cols > kMaxCols ? 0 : norm_bwd_workspace(rows, cols);
}

extern "C" lc_status lc_norm_backward(const lc_norm_params* params, const lc_matrix* dy, const lc_matrix* x,
                                      const float* mean, const float* rstd, const lc_saved_act* saved,
                                      const lc_matrix* dx, void* dweight, void* dbias, int32_t grad_dtype,
                                      int32_t accumulate, void* workspace, uint64_t workspace_bytes, void* stream) {
  lc::TraceRange trace_("lc_norm_backward");
  LC_CHECK(check_norm(params));
  LC_CHECK(check_matrix("dy", dy));
  if ((x != nullptr) == (saved != nullptr)) return fail(LC_ERR_INVALID_ARG, "exactly one of x and saved must be given");
  if (x) {
    LC_CHECK(check_matrix("x", x));
    LC_CHECK(check_shape("x", x->rows, x->cols, dy->rows, dy->cols));
    if (x->dtype != dy->dtype) return fail(LC_ERR_INVALID_ARG, "x has another dtype than dy");
  } else {
    LC_CHECK(check_saved("saved", saved));
    LC_CHECK(check_shape("saved", saved->rows, saved->cols, dy->rows, dy->cols));
  }
  const bool wants_mean = x && params->kind == LC_NORM_LAYER;
  if (!wants_mean && mean) return fail(LC_ERR_INVALID_ARG, "mean goes with x and LC_NORM_LAYER only");
  if (dy->rows && ((wants_mean && !mean) || !rstd)) return fail(LC_ERR_INVALID_ARG, "mean or rstd is NULL");
  LC_CHECK(check_vector("mean", mean, 4));
  LC_CHECK(check_vector("rstd", rstd, 4));
  if (dx) {
    LC_CHECK(check_matrix("dx", dx));
    LC_CHECK(check_shape("dx", dx->rows, dx->cols, dy->rows, dy->cols));
    if (dx->dtype != dy->dtype) return fail(LC_ERR_INVALID_ARG, "dx has another dtype than dy");
  }
  if (dbias && params->kind == LC_NORM_RMS) return fail(LC_ERR_INVALID_ARG, "LC_NORM_RMS has no bias");
  LC_CHECK(check_flag("accumulate", accumulate));
  const bool grads = dweight || dbias;
  if (grads) {
    if (!dtype_ok(grad_dtype)) return fail(LC_ERR_INVALID_ARG, "unknown gradient dtype %d", grad_dtype);
    LC_CHECK(check_vector("dweight", dweight, esz_of(grad_dtype)));
    LC_CHECK(check_vector("dbias", dbias, esz_of(grad_dtype)));
  }
  const uint64_t need = grads ? norm_bwd_workspace(dy->rows, dy->cols) : 0;
  LC_CHECK(check_space(workspace, workspace_bytes, need));
  const uint64_t param_bytes = dy->cols * esz_of(params->param_dtype);
  const uint64_t grad_bytes = grads ? dy->cols * esz_of(grad_dtype) : 0;
  const Area areas[] = {area_of("dx", dx), flat("dweight", dweight, grad_bytes), flat("dbias", dbias, grad_bytes),
                        flat("workspace", workspace, need), area_of("dy", dy), area_of("x", x), codes_of(saved),
                        scales_of(saved), flat("mean", mean, dy->rows * 4), flat("rstd", rstd, dy->rows * 4),
                        flat("weight", params->weight, param_bytes)};
  LC_CHECK(check_apart(areas, 4));
  LC_CHECK(check_stream(stream));
  NormBwd a{};
  a.dy = rows_of(dy);
  a.x = rows_of(x);
  a.dx = rows_of(dx);
  a.kept = kept_of(saved);
  a.weight = addr(params->weight);
  a.mean = mean;
  a.rstd = rstd;
  a.part = grads ? static_cast<float*>(workspace) : nullptr;
  a.rows = dy->rows;
  a.dim = static_cast<uint32_t>(dy->cols);
  a.dtype = dy->dtype;
  a.param_dtype = params->param_dtype;
  a.layer = params->kind == LC_NORM_LAYER;
  a.dweight = addr(dweight);
  a.dbias = addr(dbias);
  a.grad_dtype = grad_dtype;
  a.accumulate = accumulate;
  return launched("lc_norm_backward", launch_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

extern "C" lc_status lc_act_save(const lc_matrix* x, const lc_saved_act* saved, void* stream) {
  lc::TraceRange trace_("lc_act_save");
  LC_CHECK(check_matrix("x", x));
  LC_CHECK(check_saved("saved", saved));
  LC_CHECK(check_shape("saved", saved->rows, saved->cols, x->rows, x->cols));
  const Area areas[] = {codes_of(saved), scales_of(saved), area_of("x", x)};
  LC_CHECK(check_apart(areas, 2));
  LC_CHECK(check_stream(stream));
  const ActCopy a{rows_of(x), kept_of(saved), x->rows, static_cast<uint32_t>(x->cols), x->dtype};
  return launched("lc_act_save", launch_act_save(a, static_cast<hipStream_t>(stream)));
}

extern "C" lc_status lc_act_load(const lc_saved_act* saved, const lc_matrix* out, void* stream) {
  lc::TraceRange trace_("lc_act_load");
  LC_CHECK(check_saved("saved", saved));
  LC_CHECK(check_matrix("out", out));
  LC_CHECK(check_shape("out", out->rows, out->cols, saved->rows, saved->cols));
  const Area areas[] = {area_of("out", out), codes_of(saved), scales_of(saved)};
  LC_CHECK(check_apart(areas, 1));
  LC_CHECK(check_stream(stream));
  const ActCopy a{rows_of(out), kept_of(saved), out->rows, static_cast<uint32_t>(out->cols), out->dtype};
  return launched("lc_act_load", launch_act_load(a, static_cast<hipStream_t>(stream)));
}

extern "C" uint64_t lc_linear_wgrad_workspace(uint64_t rows, uint64_t n, uint64_t k) {
  if (rows > kMaxRows || n == 0 || k == 0 || n > kMaxCols || k > kMaxCols || n > kMaxSpan / 4 / k) return 0;
  return wgrad_workspace(rows, n, k);
}

extern "C" lc_status lc_linear_wgrad(const lc_matrix* dy, const lc_saved_act* saved, const void* col_scale,
                                     const void* col_shift, int32_t param_dtype, const lc_matrix* dweight, void* dbias,
                                     int32_t accumulate, void* workspace, uint64_t workspace_bytes, void* stream) {
  lc::TraceRange trace_("lc_linear_wgrad");
  LC_CHECK(check_matrix("dy", dy));
  LC_CHECK(check_saved("saved", saved));
  LC_CHECK(check_matrix("dweight", dweight));
  if (saved->rows != dy->rows) LC_CHECK(check_shape("saved", saved->rows, saved->cols, dy->rows, saved->cols));
  LC_CHECK(check_shape("dweight", dweight->rows, dweight->cols, dy->cols, saved->cols));
  if (dweight->rows > kMaxSpan / 4 / dweight->cols) return fail(LC_ERR_INVALID_ARG, "dweight is too large");
  LC_CHECK(check_flag("accumulate", accumulate));
  if ((col_scale || col_shift) && !dtype_ok(param_dtype))
    return fail(LC_ERR_INVALID_ARG, "unknown param dtype %d", param_dtype);
  LC_CHECK(check_vector("col_scale", col_scale, col_scale ? esz_of(param_dtype) : 1));
  LC_CHECK(check_vector("col_shift", col_shift, col_shift ? esz_of(param_dtype) : 1));
  LC_CHECK(check_vector("dbias", dbias, esz_of(dweight->dtype)));
  const uint64_t need = wgrad_workspace(dy->rows, dy->cols, saved->cols);
  LC_CHECK(check_space(workspace, workspace_bytes, need));
  const uint64_t param_bytes = saved->cols * esz_of(param_dtype);
  const Area areas[] = {area_of("dweight", dweight), flat("dbias", dbias, dy->cols * esz_of(dweight->dtype)),
                        flat("workspace", workspace, need), area_of("dy", dy), codes_of(saved), scales_of(saved),
                        flat("col_scale", col_scale, param_bytes), flat("col_shift", col_shift, param_bytes)};
  LC_CHECK(check_apart(areas, 3));
  LC_CHECK(check_stream(stream));
  Wgrad a{};
  a.dy = rows_of(dy);
  a.dw = rows_of(dweight);
  a.x = kept_of(saved);
  a.col_scale = addr(col_scale);
  a.col_shift = addr(col_shift);
  a.dbias = addr(dbias);
  a.rows = dy->rows;
  a.n = static_cast<uint32_t>(dy->cols);
  a.k = static_cast<uint32_t>(saved->cols);
  a.dtype = dy->dtype;
  a.param_dtype = param_dtype;
  a.dw_dtype = dweight->dtype;
  a.accumulate = accumulate;
  a.ws = static_cast<uint8_t*>(workspace);
  return launched("lc_linear_wgrad", launch_wgrad(a, static_cast<hipStream_t>(stream)));
}
