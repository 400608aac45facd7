// The vocabulary's operators (embedding, log probabilities from hidden rows,
// distillation): argument validation, workspaces and the dispatch to the kernels.
// See include/nsp.h for the contract.  Nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "nsp.h"
#include "row_checks.hpp"
#include "vocab_internal.hpp"

namespace {

using nsp::set_error;
using namespace nsp::checks;

// An output and another argument share nothing.
nsp_status check_apart(const nsp_rows *a, const char *a_name, int64_t a_rows, int64_t a_es, const nsp_rows *b, const char *b_name,
                       int64_t b_rows, int64_t b_es, int64_t n) {
  if (!a || !b || a_rows == 0 || b_rows == 0) return NSP_OK;
  const auto bytes = [&](const nsp_rows *r, int64_t rows, int64_t es) { return (uintptr_t)(((rows - 1) * r->token_stride + n) * es); };
  const uintptr_t x = reinterpret_cast<uintptr_t>(a->data), y = reinterpret_cast<uintptr_t>(b->data);
  if (x < y + bytes(b, b_rows, b_es) && y < x + bytes(a, a_rows, a_es)) return set_error(NSP_EINVAL, "%s overlaps %s", a_name, b_name);
  return NSP_OK;
}

nsp_status check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (need == 0) return NSP_OK;
  if (!workspace) return set_error(NSP_EWORKSPACE, "workspace is NULL (%zu bytes are needed)", need);
  NSP_TRY(check_array(workspace, 256, true, "workspace"));
  if (bytes < need) return set_error(NSP_EWORKSPACE, "workspace of %zu bytes: %zu are needed", bytes, need);
  return NSP_OK;
}

nsp_status check_vocab(int32_t vocab, int32_t most) {
  if (vocab < 1) return set_error(NSP_EINVAL, "vocab = %d < 1", vocab);
  if (vocab > most) return set_error(NSP_EUNSUPPORTED, "vocab = %d > %d", vocab, most);
  return NSP_OK;
}

// An inverse temperature.
nsp_status check_inverse(float scale) {
  if (!(scale >= 0x1p-64f && scale <= 0x1p64f))
    return set_error(NSP_EINVAL, "scale = %g not in 2^-64 .. 2^64", (double)scale);
  return NSP_OK;
}

// ----------------------------------- log probabilities from hidden rows --

nsp_status check_linear_sizes(int64_t n_tokens, int32_t dim, int32_t vocab) {
  NSP_TRY(check_tokens(n_tokens, 1));
  if (n_tokens > nsp::plan::kLinearMaxTokens)
    return set_error(NSP_EUNSUPPORTED, "n_tokens = %lld > 2^22", (long long)n_tokens);
  if (dim < 1) return set_error(NSP_EINVAL, "dim = %d < 1", dim);
  if (dim % 8 != 0 || dim > nsp::plan::kLinearMaxDim)
    return set_error(NSP_EUNSUPPORTED, "dim = %d is not a multiple of 8 up to %d", dim, nsp::plan::kLinearMaxDim);
  return check_vocab(vocab, nsp::plan::kLinearMaxVocab);
}

// Rows of whole 16 bytes, as the direct loads take them.
nsp_status check_whole_rows(const nsp_rows *r, int64_t rows, int64_t dim, int64_t es, bool output, const char *name) {
  NSP_TRY(check_rows(r, rows, 1, dim, es, output, name));
  if (rows == 0) return NSP_OK;
  NSP_TRY(check_array(r->data, 16, true, name));
  if (rows > 1 && (r->token_stride * es) % 16 != 0)
    return set_error(NSP_EINVAL, "%s: a stride of %lld elements is no multiple of 16 bytes", name, (long long)r->token_stride);
  if (rows > 1 && !output && r->token_stride > nsp::plan::kLinearMaxStride)
    return set_error(NSP_EUNSUPPORTED, "%s: a stride of %lld elements > 2^20", name, (long long)r->token_stride);
  return NSP_OK;
}

int64_t stride_of(const nsp_rows *r, int64_t rows, int64_t dim) { return rows > 1 ? r->token_stride : dim; }

nsp_status linear_inputs(int64_t n_tokens, int32_t dim, int32_t vocab, const nsp_rows *x, const nsp_rows *w, const int64_t *targets,
                         float scale, nsp::LinearArgs *a) {
  NSP_TRY(check_linear_sizes(n_tokens, dim, vocab));
  NSP_TRY(check_inverse(scale));
  NSP_TRY(check_whole_rows(x, n_tokens, dim, 2, false, "x"));
  NSP_TRY(check_whole_rows(w, n_tokens > 0 ? vocab : 0, dim, 2, false, "w"));
  a->x = static_cast<const char *>(x->data);
  a->x_stride = stride_of(x, n_tokens, dim);
  a->w = static_cast<const char *>(w->data);
  a->w_stride = stride_of(w, vocab, dim);
  a->targets = targets;
  a->n_tokens = n_tokens;
  a->dim = dim;
  a->vocab = vocab;
  a->scale = scale;
  return NSP_OK;
}

// ------------------------------------------------------------ distillation --

nsp_status check_distill(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, const nsp_rows *rows, int32_t top, const int64_t *index,
                         const float *teacher, nsp_distill_kind kind, float scale) {
  NSP_TRY(check_dtype(dtype, "dtype"));
  NSP_TRY(check_vocab(vocab, nsp::kLogpMaxVocab));
  NSP_TRY(check_tokens(n_tokens, 1));
  NSP_TRY(check_inverse(scale));
  NSP_TRY(check_rows(rows, n_tokens, 1, vocab, elem_bytes(dtype), false, "logits"));
  if (top < 1) return set_error(NSP_EINVAL, "top = %d < 1", top);
  if (top > NSP_DISTILL_MAX_TOP) return set_error(NSP_EUNSUPPORTED, "top = %d > %d", top, NSP_DISTILL_MAX_TOP);
  if (kind != NSP_DISTILL_GIVEN && kind != NSP_DISTILL_NORMALIZED) return set_error(NSP_EINVAL, "unknown distillation kind %d", (int)kind);
  NSP_TRY(check_array(index, 8, n_tokens > 0, "index"));
  return check_array(teacher, 4, n_tokens > 0, "teacher_logp");
}

void distill_inputs(int64_t n_tokens, int32_t vocab, const nsp_rows &rows, int32_t top, const int64_t *index, const float *teacher,
                    nsp_distill_kind kind, float scale, nsp::DistillArgs *a) {
  a->logits = static_cast<const char *>(rows.data);
  a->row_stride = rows.token_stride;
  a->index = index;
  a->teacher = teacher;
  a->n_tokens = (int32_t)n_tokens;
  a->vocab = vocab;
  a->top = top;
  a->normalized = kind == NSP_DISTILL_NORMALIZED;
  a->scale = scale;
}

size_t distill_ws(int64_t n_tokens, int32_t vocab) {
  const int parts = nsp::plan::logp_parts(n_tokens, vocab);
  return parts > 1 ? align256((size_t)n_tokens * parts * sizeof(float4)) : 0;
}

// --------------------------------------------------------------- embedding --

nsp_status check_embedding(nsp_dtype w_dtype, nsp_dtype dtype, int64_t n_tokens, int32_t dim, int32_t vocab, float scale) {
  NSP_TRY(check_dtype(w_dtype, "w_dtype"));
  NSP_TRY(check_dtype(dtype, "dtype"));
  NSP_TRY(check_tokens(n_tokens, 1));
  if (n_tokens > nsp::plan::kEmbedMaxTokens) return set_error(NSP_EUNSUPPORTED, "n_tokens = %lld > 2^26", (long long)n_tokens);
  if (dim < 1) return set_error(NSP_EINVAL, "dim = %d < 1", dim);
  if (dim > nsp::plan::kEmbedMaxDim) return set_error(NSP_EUNSUPPORTED, "dim = %d > 2^20", dim);
  if (!std::isfinite(scale)) return set_error(NSP_EINVAL, "scale is not finite");
  return check_vocab(vocab, nsp::plan::kEmbedMaxVocab);
}

}  // namespace

static_assert(NSP_DISTILL_MAX_TOP == nsp::kDistillMaxTop, "one limit");

extern "C" {

size_t nsp_linear_logp_fwd_workspace(int64_t n_tokens, int32_t dim, int32_t vocab) {
  if (check_linear_sizes(n_tokens, dim, vocab) != NSP_OK || n_tokens == 0) return 0;
  set_error(NSP_OK, nullptr);
  return nsp::plan::linear_fwd(n_tokens, dim, vocab).bytes;
}

nsp_status nsp_linear_logp_fwd(int64_t n_tokens, int32_t dim, int32_t vocab, const nsp_rows *x, const nsp_rows *w,
                               const int64_t *targets, float scale, float *logp, float *lse, float *entropy, void *workspace,
                               size_t ws_bytes, hipStream_t stream) {
  nsp::LinearArgs a{};
  NSP_TRY(linear_inputs(n_tokens, dim, vocab, x, w, targets, scale, &a));
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(logp, 4, false, "logp"));
  NSP_TRY(check_array(targets, 8, some && logp, "targets"));
  NSP_TRY(check_array(entropy, 4, false, "entropy"));
  if (!some) return set_error(NSP_OK, nullptr);
  NSP_TRY(check_workspace(workspace, ws_bytes, nsp::plan::linear_fwd(n_tokens, dim, vocab).bytes));
  a.logp = logp;
  a.lse = lse;
  a.entropy = entropy;
  a.ws = static_cast<char *>(workspace);
  return hip_status(nsp::timed_launch(nsp::K_LINEAR_FWD, stream, [&] { return nsp::launch_linear_logp_fwd(a, stream); }),
                    "log probability launch");
}

size_t nsp_linear_logp_bwd_workspace(int64_t n_tokens, int32_t dim, int32_t vocab) {
  if (check_linear_sizes(n_tokens, dim, vocab) != NSP_OK || n_tokens == 0) return 0;
  set_error(NSP_OK, nullptr);
  return nsp::plan::linear_bwd_bytes(n_tokens, dim, vocab);
}

nsp_status nsp_linear_logp_bwd(nsp_dtype grad_dtype, int64_t n_tokens, int32_t dim, int32_t vocab, const nsp_rows *x,
                               const nsp_rows *w, const int64_t *targets, float scale, const float *lse, const float *entropy,
                               const float *g_logp, const float *g_lse, const float *g_entropy, const nsp_rows *dx,
                               const nsp_rows *dw, void *workspace, size_t ws_bytes, hipStream_t stream) {
  nsp::LinearArgs a{};
  NSP_TRY(check_dtype(grad_dtype, "grad_dtype"));
  NSP_TRY(linear_inputs(n_tokens, dim, vocab, x, w, targets, scale, &a));
  const int64_t es = elem_bytes(grad_dtype);
  if (dx) NSP_TRY(check_whole_rows(dx, n_tokens, dim, es, true, "dx"));
  if (dw) NSP_TRY(check_whole_rows(dw, vocab, dim, es, true, "dw"));
  NSP_TRY(check_apart(dx, "dx", n_tokens, es, x, "x", n_tokens, 2, dim));
  NSP_TRY(check_apart(dw, "dw", vocab, es, x, "x", n_tokens, 2, dim));
  if (n_tokens > 0) {
    NSP_TRY(check_apart(dx, "dx", n_tokens, es, w, "w", vocab, 2, dim));
    NSP_TRY(check_apart(dw, "dw", vocab, es, w, "w", vocab, 2, dim));
  }
  NSP_TRY(check_apart(dw, "dw", vocab, es, dx, "dx", n_tokens, es, dim));
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(g_logp, 4, false, "g_logp"));
  NSP_TRY(check_array(g_lse, 4, false, "g_lse"));
  NSP_TRY(check_array(g_entropy, 4, false, "g_entropy"));
  NSP_TRY(check_array(targets, 8, some && g_logp, "targets"));
  NSP_TRY(check_array(entropy, 4, some && g_entropy, "entropy"));
  if (!dx && !dw) return set_error(NSP_OK, nullptr);
  if (some) NSP_TRY(check_workspace(workspace, ws_bytes, nsp::plan::linear_bwd_bytes(n_tokens, dim, vocab)));
  a.lse_in = lse;
  a.entropy_in = entropy;
  a.g_logp = g_logp;
  a.g_lse = g_lse;
  a.g_entropy = g_entropy;
  a.g_f32 = grad_dtype == NSP_F32;
  if (dx) {
    a.dx = static_cast<char *>(dx->data);
    a.dx_stride = stride_of(dx, n_tokens, dim);
  }
  if (dw) {
    a.dw = static_cast<char *>(dw->data);
    a.dw_stride = stride_of(dw, vocab, dim);
  }
  a.ws = static_cast<char *>(workspace);
  return hip_status(nsp::timed_launch(nsp::K_LINEAR_BWD, stream, [&] { return nsp::launch_linear_logp_bwd(a, stream); }),
                    "log probability backward launch");
}

size_t nsp_distill_fwd_workspace(int64_t n_tokens, int32_t vocab) {
  if (n_tokens < 0 || n_tokens > kMaxRows || vocab < 1 || vocab > nsp::kLogpMaxVocab) return 0;
  return distill_ws(n_tokens, vocab);
}

nsp_status nsp_distill_fwd(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, const void *logits, int64_t row_stride, int32_t top,
                           const int64_t *index, const float *teacher_logp, nsp_distill_kind kind, float scale, float *loss,
                           float *lse, void *workspace, size_t ws_bytes, hipStream_t stream) {
  const nsp_rows rows = {const_cast<void *>(logits), row_stride, 0};
  NSP_TRY(check_distill(dtype, n_tokens, vocab, &rows, top, index, teacher_logp, kind, scale));
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(loss, 4, false, "loss"));
  if (!some) return set_error(NSP_OK, nullptr);
  NSP_TRY(check_workspace(workspace, ws_bytes, distill_ws(n_tokens, vocab)));
  nsp::DistillArgs a{};
  distill_inputs(n_tokens, vocab, rows, top, index, teacher_logp, kind, scale, &a);
  a.loss = loss;
  a.lse = lse;
  a.parts = nsp::plan::logp_parts(n_tokens, vocab);
  a.part_sums = a.parts > 1 ? static_cast<float4 *>(workspace) : nullptr;
  return hip_status(nsp::timed_launch(nsp::K_DISTILL_FWD, stream, [&] { return nsp::launch_distill_fwd(dtype == NSP_F32, a, stream); }),
                    "distillation launch");
}

nsp_status nsp_distill_bwd(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, const void *logits, int64_t row_stride, int32_t top,
                           const int64_t *index, const float *teacher_logp, nsp_distill_kind kind, float scale, const float *lse,
                           const float *g_loss, void *dlogits, int64_t d_row_stride, hipStream_t stream) {
  const nsp_rows rows = {const_cast<void *>(logits), row_stride, 0}, out = {dlogits, d_row_stride, 0};
  NSP_TRY(check_distill(dtype, n_tokens, vocab, &rows, top, index, teacher_logp, kind, scale));
  const int64_t es = elem_bytes(dtype);
  NSP_TRY(check_rows(&out, n_tokens, 1, vocab, es, true, "dlogits"));
  NSP_TRY(check_overlap(&rows, "logits", &out, "dlogits", n_tokens, 1, vocab, es));
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(g_loss, 4, some, "g_loss"));
  if (!some) return set_error(NSP_OK, nullptr);
  nsp::DistillArgs a{};
  distill_inputs(n_tokens, vocab, rows, top, index, teacher_logp, kind, scale, &a);
  a.lse_in = lse;
  a.g_loss = g_loss;
  a.dlogits = static_cast<char *>(dlogits);
  a.d_row_stride = d_row_stride;
  return hip_status(nsp::timed_launch(nsp::K_DISTILL_BWD, stream, [&] { return nsp::launch_distill_bwd(dtype == NSP_F32, a, stream); }),
                    "distillation backward launch");
}

nsp_status nsp_embedding_fwd(nsp_dtype w_dtype, nsp_dtype dtype, int64_t n_tokens, int32_t dim, int32_t vocab, const int64_t *tokens,
                             const nsp_rows *w, float scale, const nsp_rows *y, hipStream_t stream) {
  NSP_TRY(check_embedding(w_dtype, dtype, n_tokens, dim, vocab, scale));
  const int64_t es = elem_bytes(dtype), ews = elem_bytes(w_dtype);
  const bool some = n_tokens > 0;
  NSP_TRY(check_rows(w, some ? vocab : 0, 1, dim, ews, false, "w"));
  NSP_TRY(check_rows(y, n_tokens, 1, dim, es, true, "y"));
  NSP_TRY(check_array(tokens, 8, some, "tokens"));
  if (!some) return set_error(NSP_OK, nullptr);
  NSP_TRY(check_apart(y, "y", n_tokens, es, w, "w", vocab, ews, dim));
  nsp::EmbedArgs a{};
  a.tokens = tokens;
  a.n_tokens = (int32_t)n_tokens;
  a.vocab = vocab;
  a.dim = dim;
  a.scale = scale;
  a.w = view(w);
  a.y = view(y);
  return hip_status(nsp::timed_launch(nsp::K_EMBED_FWD, stream,
                                      [&] { return nsp::launch_embedding_fwd(w_dtype == NSP_F32, dtype == NSP_F32, a, stream); }),
                    "embedding launch");
}

size_t nsp_embedding_bwd_workspace(int64_t n_tokens, int32_t dim, int32_t vocab) {
  if (check_embedding(NSP_BF16, NSP_BF16, n_tokens, dim, vocab, 1.f) != NSP_OK) return 0;
  set_error(NSP_OK, nullptr);
  return nsp::plan::embed_bwd(n_tokens, dim, vocab).bytes;
}

nsp_status nsp_embedding_bwd(nsp_dtype w_dtype, nsp_dtype dtype, int64_t n_tokens, int32_t dim, int32_t vocab, const int64_t *tokens,
                             const nsp_rows *dy, float scale, const nsp_rows *dw, void *workspace, size_t ws_bytes,
                             hipStream_t stream) {
  NSP_TRY(check_embedding(w_dtype, dtype, n_tokens, dim, vocab, scale));
  const int64_t es = elem_bytes(dtype), ews = elem_bytes(w_dtype);
  NSP_TRY(check_rows(dy, n_tokens, 1, dim, es, false, "dy"));
  NSP_TRY(check_rows(dw, vocab, 1, dim, ews, true, "dw"));
  NSP_TRY(check_array(tokens, 8, n_tokens > 0, "tokens"));
  NSP_TRY(check_apart(dw, "dw", vocab, ews, dy, "dy", n_tokens, es, dim));
  nsp::EmbedArgs a{};
  a.f = nsp::plan::embed_bwd(n_tokens, dim, vocab);
  NSP_TRY(check_workspace(workspace, ws_bytes, a.f.bytes));
  a.tokens = tokens;
  a.n_tokens = (int32_t)n_tokens;
  a.vocab = vocab;
  a.dim = dim;
  a.scale = scale;
  a.w = view(dw);
  a.y = view(dy);
  a.ws = static_cast<char *>(workspace);
  return hip_status(nsp::timed_launch(nsp::K_EMBED_BWD, stream,
                                      [&] { return nsp::launch_embedding_bwd(w_dtype == NSP_F32, dtype == NSP_F32, a, stream); }),
                    "embedding backward launch");
}

}  // extern "C"
