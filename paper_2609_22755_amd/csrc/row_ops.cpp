// Row operators (rotary positions, norms, token log probabilities): argument
// validation, the scaled rotary frequencies and the dispatch to the kernels.
// See include/nsp.h for the contract.  Nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "nsp.h"
#include "nsp_internal.hpp"
#include "row_checks.hpp"

namespace {

using nsp::set_error;
using namespace nsp::checks;

nsp_status rotary(bool bwd, nsp_rotary_layout layout, nsp_dtype dtype, int64_t n_tokens, int32_t head_dim,
                  int32_t rot_dim, const double *freqs, float scale, const int64_t *positions, int32_t q_heads,
                  const nsp_rows *q, const nsp_rows *q_out, int32_t k_heads, const nsp_rows *k,
                  const nsp_rows *k_out, hipStream_t stream) {
  if (layout != NSP_ROTARY_HALF && layout != NSP_ROTARY_PAIRS)
    return set_error(NSP_EINVAL, "unknown rotary layout %d", (int)layout);
  NSP_TRY(check_dtype(dtype, "dtype"));
  if (head_dim < 1) return set_error(NSP_EINVAL, "head_dim = %d < 1", head_dim);
  if (head_dim > nsp::kRotaryMaxDim)
    return set_error(NSP_EUNSUPPORTED, "head_dim = %d > %d", head_dim, nsp::kRotaryMaxDim);
  if (rot_dim < 2 || rot_dim > head_dim || rot_dim % 2 != 0)
    return set_error(NSP_EINVAL, "rot_dim = %d is not even and in 2 .. head_dim = %d", rot_dim, head_dim);
  if (!std::isfinite(scale)) return set_error(NSP_EINVAL, "scale is not finite");
  if (q_heads < 1 || q_heads > 65536) return set_error(NSP_EINVAL, "q_heads = %d not in 1 .. 65536", q_heads);
  if (k_heads < 0 || k_heads > 65536) return set_error(NSP_EINVAL, "k_heads = %d not in 0 .. 65536", k_heads);
  NSP_TRY(check_tokens(n_tokens, q_heads + k_heads));
  const int64_t es = elem_bytes(dtype);
  const char *const names[2][4] = {{"q", "q_out", "k", "k_out"}, {"dq_out", "dq", "dk_out", "dk"}};
  const char *const *nm = names[bwd ? 1 : 0];
  NSP_TRY(check_rows(q, n_tokens, q_heads, head_dim, es, false, nm[0]));
  NSP_TRY(check_rows(q_out, n_tokens, q_heads, head_dim, es, true, nm[1]));
  NSP_TRY(check_overlap(q, nm[0], q_out, nm[1], n_tokens, q_heads, head_dim, es));
  if (k_heads > 0) {
    NSP_TRY(check_rows(k, n_tokens, k_heads, head_dim, es, false, nm[2]));
    NSP_TRY(check_rows(k_out, n_tokens, k_heads, head_dim, es, true, nm[3]));
    NSP_TRY(check_overlap(k, nm[2], k_out, nm[3], n_tokens, k_heads, head_dim, es));
  } else if (k || k_out) {
    return set_error(NSP_EINVAL, "%s and %s must be NULL without key heads", nm[2], nm[3]);
  }
  if (n_tokens == 0) return set_error(NSP_OK, nullptr);
  NSP_TRY(check_array(freqs, 8, true, "freqs"));
  NSP_TRY(check_array(positions, 8, true, "positions"));
  nsp::RotaryArgs a{};
  a.x[0] = view(q);
  a.y[0] = view(q_out);
  a.heads[0] = q_heads;
  a.copy[0] = rot_dim < head_dim && !same_view(q, q_out, n_tokens, q_heads);
  if (k_heads > 0) {
    a.x[1] = view(k);
    a.y[1] = view(k_out);
    a.copy[1] = rot_dim < head_dim && !same_view(k, k_out, n_tokens, k_heads);
  }
  a.heads[1] = k_heads;
  a.n_tokens = n_tokens;
  a.freqs = freqs;
  a.positions = positions;
  a.scale = scale;
  a.sign = bwd ? -1.f : 1.f;
  a.head_dim = head_dim;
  a.half = rot_dim / 2;
  return hip_status(nsp::timed_launch(nsp::K_ROTARY, stream,
                                      [&] { return nsp::launch_rotary(layout == NSP_ROTARY_PAIRS, dtype == NSP_F32, a, stream); }),
                    "rotary launch");
}

nsp_status check_norm(nsp_norm_kind kind, nsp_dtype dtype, nsp_dtype w_dtype, int64_t n_tokens, int32_t n_heads,
                      int32_t n) {
  if (kind != NSP_NORM_LAYER && kind != NSP_NORM_RMS) return set_error(NSP_EINVAL, "unknown norm kind %d", (int)kind);
  NSP_TRY(check_dtype(dtype, "dtype"));
  NSP_TRY(check_dtype(w_dtype, "w_dtype"));
  if (n < 1) return set_error(NSP_EINVAL, "n = %d < 1", n);
  if (n > nsp::kNormMaxN) return set_error(NSP_EUNSUPPORTED, "n = %d > %d", n, nsp::kNormMaxN);
  if (n_heads < 1) return set_error(NSP_EINVAL, "n_heads = %d < 1", n_heads);
  return check_tokens(n_tokens, n_heads);
}

size_t norm_ws(int64_t rows, int32_t n) {   // the larger of the two types' needs
  const int a = nsp::norm_bwd_parts(rows, n, false), b = nsp::norm_bwd_parts(rows, n, true);
  return align256((size_t)(a > b ? a : b) * 2 * (size_t)n * sizeof(float));
}

nsp_status check_logp(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, float scale, const nsp_rows *rows) {
  NSP_TRY(check_dtype(dtype, "dtype"));
  if (vocab < 1) return set_error(NSP_EINVAL, "vocab = %d < 1", vocab);
  if (vocab > nsp::kLogpMaxVocab) return set_error(NSP_EUNSUPPORTED, "vocab = %d > 2^30", vocab);
  NSP_TRY(check_tokens(n_tokens, 1));
  if (!(scale >= 0x1p-64f && scale <= 0x1p64f))
    return set_error(NSP_EINVAL, "scale = %g not in 2^-64 .. 2^64", (double)scale);
  return check_rows(rows, n_tokens, 1, vocab, elem_bytes(dtype), false, "logits");
}

struct LogpWs {
  size_t top_off, bytes;
  int parts;
};

LogpWs logp_ws(int64_t n_tokens, int32_t vocab, int32_t top) {
  LogpWs w{0, 0, nsp::token_logp_parts(n_tokens, vocab)};
  if (w.parts > 1) {
    w.top_off = align256((size_t)n_tokens * w.parts * sizeof(float4));
    w.bytes = w.top_off + align256((size_t)n_tokens * w.parts * top * sizeof(uint64_t));
  }
  return w;
}

}  // namespace

extern "C" {

nsp_status nsp_rotary_fwd(nsp_rotary_layout layout, nsp_dtype dtype, int64_t n_tokens, int32_t head_dim,
                          int32_t rot_dim, const double *freqs, float scale, const int64_t *positions,
                          int32_t q_heads, const nsp_rows *q, const nsp_rows *q_out, int32_t k_heads,
                          const nsp_rows *k, const nsp_rows *k_out, hipStream_t stream) {
  return rotary(false, layout, dtype, n_tokens, head_dim, rot_dim, freqs, scale, positions, q_heads, q, q_out, k_heads,
                k, k_out, stream);
}

nsp_status nsp_rotary_bwd(nsp_rotary_layout layout, nsp_dtype dtype, int64_t n_tokens, int32_t head_dim,
                          int32_t rot_dim, const double *freqs, float scale, const int64_t *positions,
                          int32_t q_heads, const nsp_rows *dq_out, const nsp_rows *dq, int32_t k_heads,
                          const nsp_rows *dk_out, const nsp_rows *dk, hipStream_t stream) {
  return rotary(true, layout, dtype, n_tokens, head_dim, rot_dim, freqs, scale, positions, q_heads, dq_out, dq,
                k_heads, dk_out, dk, stream);
}

nsp_status nsp_rotary_frequencies(int32_t rot_dim, double base, nsp_rotary_scaling scaling, double factor,
                                  double context, double low, double high, double *freqs, float *scale) {
  if (rot_dim < 2 || rot_dim > 1024 || rot_dim % 2 != 0)
    return set_error(NSP_EINVAL, "rot_dim = %d is not even and in 2 .. 1024", rot_dim);
  if (!std::isfinite(base) || !(base > 0)) return set_error(NSP_EINVAL, "base must be finite and positive (got %g)", base);
  if (scaling < NSP_ROTARY_PLAIN || scaling > NSP_ROTARY_PARTS)
    return set_error(NSP_EINVAL, "unknown rotary scaling %d", (int)scaling);
  if (scaling != NSP_ROTARY_PLAIN && !(std::isfinite(factor) && factor >= 1))
    return set_error(NSP_EINVAL, "factor must be finite and at least 1 (got %g)", factor);
  if (scaling == NSP_ROTARY_BASE && rot_dim < 4)
    return set_error(NSP_EINVAL, "rot_dim = %d: a scaled base needs at least 4", rot_dim);
  if (scaling == NSP_ROTARY_PARTS) {
    if (!std::isfinite(context) || !(context > 0))
      return set_error(NSP_EINVAL, "context must be finite and positive (got %g)", context);
    if (!(low >= 0) || !(high > low) || !std::isfinite(high))
      return set_error(NSP_EINVAL, "0 <= low < high is needed (got low %g, high %g)", low, high);
  }
  if (!freqs) return set_error(NSP_EINVAL, "freqs is NULL");
  if (scaling == NSP_ROTARY_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == NSP_ROTARY_LINEAR) f /= factor;
    if (scaling == NSP_ROTARY_PARTS) {
      const double turns = context * f / 6.283185307179586476925286766559;
      const double g = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
      f = f * (g + (1.0 - g) / factor);
    }
    freqs[i] = f;
  }
  if (scale) *scale = scaling == NSP_ROTARY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return set_error(NSP_OK, nullptr);
}

nsp_status nsp_norm_fwd(nsp_norm_kind kind, nsp_dtype dtype, nsp_dtype w_dtype, int64_t n_tokens, int32_t n_heads,
                        int32_t n, const nsp_rows *x, const void *w, const void *b, float eps, const nsp_rows *y,
                        float *mean, float *rstd, hipStream_t stream) {
  NSP_TRY(check_norm(kind, dtype, w_dtype, n_tokens, n_heads, n));
  if (!std::isfinite(eps) || !(eps >= 0.f)) return set_error(NSP_EINVAL, "eps must be finite and >= 0 (got %g)", (double)eps);
  const int64_t es = elem_bytes(dtype);
  NSP_TRY(check_rows(x, n_tokens, n_heads, n, es, false, "x"));
  NSP_TRY(check_rows(y, n_tokens, n_heads, n, es, true, "y"));
  NSP_TRY(check_overlap(x, "x", y, "y", n_tokens, n_heads, n, es));
  NSP_TRY(check_array(w, (size_t)elem_bytes(w_dtype), false, "w"));
  NSP_TRY(check_array(b, (size_t)elem_bytes(w_dtype), false, "b"));
  NSP_TRY(check_array(mean, 4, false, "mean"));
  NSP_TRY(check_array(rstd, 4, false, "rstd"));
  if (n_tokens == 0) return set_error(NSP_OK, nullptr);
  nsp::NormArgs a{};
  a.x = view(x);
  a.y = view(y);
  a.w = w;
  a.b = b;
  a.w_f32 = w_dtype == NSP_F32;
  a.rms = kind == NSP_NORM_RMS;
  a.rows = (int32_t)(n_tokens * n_heads);
  a.n = n;
  a.heads = nsp::FastDiv((uint32_t)n_heads);
  a.eps = eps;
  a.mean = a.rms ? nullptr : mean;
  a.rstd = rstd;
  return hip_status(nsp::timed_launch(nsp::K_NORM_FWD, stream, [&] { return nsp::launch_norm_fwd(dtype == NSP_F32, a, stream); }),
                    "norm launch");
}

size_t nsp_norm_bwd_workspace(int64_t n_tokens, int32_t n_heads, int32_t n) {
  if (check_norm(NSP_NORM_RMS, NSP_BF16, NSP_BF16, n_tokens, n_heads, n) != NSP_OK) return 0;
  set_error(NSP_OK, nullptr);
  return norm_ws(n_tokens * n_heads, n);
}

nsp_status nsp_norm_bwd(nsp_norm_kind kind, nsp_dtype dtype, nsp_dtype w_dtype, int64_t n_tokens, int32_t n_heads,
                        int32_t n, const nsp_rows *x, const void *w, const nsp_rows *dy, const float *mean,
                        const float *rstd, const nsp_rows *dx, void *dw, void *db, void *workspace, size_t ws_bytes,
                        hipStream_t stream) {
  NSP_TRY(check_norm(kind, dtype, w_dtype, n_tokens, n_heads, n));
  const int64_t es = elem_bytes(dtype);
  const size_t ews = (size_t)elem_bytes(w_dtype);
  NSP_TRY(check_rows(x, n_tokens, n_heads, n, es, false, "x"));
  NSP_TRY(check_rows(dy, n_tokens, n_heads, n, es, false, "dy"));
  NSP_TRY(check_rows(dx, n_tokens, n_heads, n, es, true, "dx"));
  NSP_TRY(check_overlap(x, "x", dx, "dx", n_tokens, n_heads, n, es));
  NSP_TRY(check_overlap(dy, "dy", dx, "dx", n_tokens, n_heads, n, es));
  NSP_TRY(check_array(w, ews, false, "w"));
  NSP_TRY(check_array(mean, 4, kind == NSP_NORM_LAYER && n_tokens > 0, "mean"));
  NSP_TRY(check_array(rstd, 4, n_tokens > 0, "rstd"));
  NSP_TRY(check_array(dw, ews, false, "dw"));
  NSP_TRY(check_array(db, ews, false, "db"));
  const int64_t rows = n_tokens * n_heads;
  if (dw || db) {
    const size_t need = norm_ws(rows, n);
    if (need > 0) {
      if (!workspace) return set_error(NSP_EWORKSPACE, "workspace is NULL (%zu bytes are needed)", need);
      NSP_TRY(check_array(workspace, 256, true, "workspace"));
      if (ws_bytes < need)
        return set_error(NSP_EWORKSPACE, "workspace of %zu bytes: %zu are needed", ws_bytes, need);
    }
  } else if (rows == 0) {
    return set_error(NSP_OK, nullptr);
  }
  nsp::NormArgs a{};
  a.x = view(x);
  a.dy = view(dy);
  a.y = view(dx);
  a.w = w;
  a.w_f32 = w_dtype == NSP_F32;
  a.rms = kind == NSP_NORM_RMS;
  a.rows = (int32_t)rows;
  a.n = n;
  a.heads = nsp::FastDiv((uint32_t)n_heads);
  a.mean_in = mean;
  a.rstd_in = rstd;
  a.dw = dw;
  a.db = db;
  a.part = (dw || db) ? static_cast<float *>(workspace) : nullptr;
  return hip_status(nsp::timed_launch(nsp::K_NORM_BWD, stream, [&] { return nsp::launch_norm_bwd(dtype == NSP_F32, a, stream); }),
                    "norm backward launch");
}

size_t nsp_token_logp_workspace(int64_t n_tokens, int32_t vocab, int32_t top) {
  if (n_tokens < 0 || n_tokens > kMaxRows || vocab < 1 || vocab > nsp::kLogpMaxVocab || top < 0 || top > NSP_TOKEN_LOGP_MAX_TOP) return 0;
  return logp_ws(n_tokens, vocab, top).bytes;
}

nsp_status nsp_token_logp_fwd(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, const void *logits,
                              int64_t row_stride, const int64_t *targets, float scale, float *logp, float *lse,
                              float *entropy, int32_t top, float *top_logp, int64_t *top_index, void *workspace,
                              size_t ws_bytes, hipStream_t stream) {
  const nsp_rows rows = {const_cast<void *>(logits), row_stride, 0};
  NSP_TRY(check_logp(dtype, n_tokens, vocab, scale, &rows));
  if (top < 0) return set_error(NSP_EINVAL, "top = %d < 0", top);
  if (top > NSP_TOKEN_LOGP_MAX_TOP)
    return set_error(NSP_EUNSUPPORTED, "top = %d > %d", top, NSP_TOKEN_LOGP_MAX_TOP);
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(logp, 4, false, "logp"));
  NSP_TRY(check_array(targets, 8, some && logp, "targets"));
  NSP_TRY(check_array(entropy, 4, false, "entropy"));
  NSP_TRY(check_array(top_logp, 4, some && top > 0, "top_logp"));
  NSP_TRY(check_array(top_index, 8, some && top > 0, "top_index"));
  if (!some) return set_error(NSP_OK, nullptr);
  const LogpWs w = logp_ws(n_tokens, vocab, top);
  if (w.bytes > 0) {
    if (!workspace) return set_error(NSP_EWORKSPACE, "workspace is NULL (%zu bytes are needed)", w.bytes);
    NSP_TRY(check_array(workspace, 256, true, "workspace"));
    if (ws_bytes < w.bytes)
      return set_error(NSP_EWORKSPACE, "workspace of %zu bytes: %zu are needed", ws_bytes, w.bytes);
  }
  nsp::LogpArgs a{};
  a.logits = static_cast<const char *>(logits);
  a.row_stride = row_stride;
  a.targets = targets;
  a.scale = scale;
  a.n_tokens = (int32_t)n_tokens;
  a.vocab = vocab;
  a.top = top;
  a.logp = logp;
  a.lse = lse;
  a.entropy = entropy;
  a.top_logp = top_logp;
  a.top_index = top_index;
  a.parts = w.parts;
  if (w.parts > 1) {
    a.part_sums = static_cast<float4 *>(workspace);
    a.part_top = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + w.top_off);
  }
  return hip_status(nsp::timed_launch(nsp::K_LOGP_FWD, stream,
                                      [&] { return nsp::launch_token_logp_fwd(dtype == NSP_F32, a, stream); }),
                    "token log probability launch");
}

nsp_status nsp_token_logp_bwd(nsp_dtype dtype, int64_t n_tokens, int32_t vocab, const void *logits,
                              int64_t row_stride, const int64_t *targets, float scale, const float *lse,
                              const float *entropy, const float *g_logp, const float *g_lse, const float *g_entropy,
                              void *dlogits, int64_t d_row_stride, hipStream_t stream) {
  const nsp_rows rows = {const_cast<void *>(logits), row_stride, 0}, out = {dlogits, d_row_stride, 0};
  NSP_TRY(check_logp(dtype, n_tokens, vocab, scale, &rows));
  const int64_t es = elem_bytes(dtype);
  NSP_TRY(check_rows(&out, n_tokens, 1, vocab, es, true, "dlogits"));
  NSP_TRY(check_overlap(&rows, "logits", &out, "dlogits", n_tokens, 1, vocab, es));
  const bool some = n_tokens > 0;
  NSP_TRY(check_array(lse, 4, some, "lse"));
  NSP_TRY(check_array(g_logp, 4, false, "g_logp"));
  NSP_TRY(check_array(g_lse, 4, false, "g_lse"));
  NSP_TRY(check_array(g_entropy, 4, false, "g_entropy"));
  NSP_TRY(check_array(targets, 8, some && g_logp, "targets"));
  NSP_TRY(check_array(entropy, 4, some && g_entropy, "entropy"));
  if (!some) return set_error(NSP_OK, nullptr);
  nsp::LogpBwdArgs a{};
  a.logits = static_cast<const char *>(logits);
  a.dlogits = static_cast<char *>(dlogits);
  a.row_stride = row_stride;
  a.d_row_stride = d_row_stride;
  a.targets = targets;
  a.scale = scale;
  a.n_tokens = (int32_t)n_tokens;
  a.vocab = vocab;
  a.lse = lse;
  a.entropy = entropy;
  a.g_logp = g_logp;
  a.g_lse = g_lse;
  a.g_entropy = g_entropy;
  return hip_status(nsp::timed_launch(nsp::K_LOGP_BWD, stream,
                                      [&] { return nsp::launch_token_logp_bwd(dtype == NSP_F32, a, stream); }),
                    "token log probability backward launch");
}

}  // extern "C"
