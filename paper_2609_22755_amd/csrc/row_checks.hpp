// Argument checks that the calls on rows share.  Host code; nothing here allocates
// or throws.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nsp.h"
#include "nsp_internal.hpp"

#define NSP_TRY(expr)                 \
  do {                                \
    nsp_status _st = (expr);          \
    if (_st != NSP_OK) return _st;    \
  } while (0)

namespace nsp {
namespace checks {

constexpr int64_t kMaxRows = INT32_MAX;
constexpr int64_t kMaxStride = int64_t(1) << 40;

inline nsp_status check_dtype(nsp_dtype t, const char *name) {
  if (t != NSP_BF16 && t != NSP_F32) return set_error(NSP_EINVAL, "unknown %s %d", name, (int)t);
  return NSP_OK;
}

inline int64_t elem_bytes(nsp_dtype t) { return t == NSP_F32 ? 4 : 2; }

inline nsp_status check_tokens(int64_t n_tokens, int64_t n_heads) {
  if (n_tokens < 0 || n_tokens > kMaxRows)
    return set_error(NSP_EINVAL, "n_tokens = %lld not in 0 .. 2^31 - 1", (long long)n_tokens);
  if (n_tokens * n_heads > kMaxRows)
    return set_error(NSP_EINVAL, "%lld tokens of %lld heads: more than 2^31 - 1 rows", (long long)n_tokens,
                     (long long)n_heads);
  return NSP_OK;
}

inline nsp_status check_array(const void *p, size_t align, bool needed, const char *name) {
  if (!p) return needed ? set_error(NSP_EINVAL, "%s is NULL", name) : NSP_OK;
  if (reinterpret_cast<uintptr_t>(p) % align != 0)
    return set_error(NSP_EINVAL, "%s is not %zu-byte aligned", name, align);
  return NSP_OK;
}

// Rows of n elements of es bytes.  Those of an output lie apart.
inline nsp_status check_rows(const nsp_rows *r, int64_t tokens, int64_t heads, int64_t n, int64_t es, bool output,
                      const char *name) {
  if (!r) return set_error(NSP_EINVAL, "%s is NULL", name);
  if (tokens == 0) return NSP_OK;
  NSP_TRY(check_array(r->data, (size_t)es, true, name));
  const int64_t ts = r->token_stride, hs = r->head_stride;
  if (ts < 0 || hs < 0 || ts > kMaxStride || hs > kMaxStride)
    return set_error(NSP_EINVAL, "%s: strides %lld, %lld not in 0 .. 2^40", name, (long long)ts, (long long)hs);
  // (every byte offset then stays below 2^63)
  const __int128 last = (__int128)(tokens - 1) * ts + (__int128)(heads - 1) * hs + n;
  if (last > ((__int128)1 << 60)) return set_error(NSP_EINVAL, "%s: the rows span more than 2^60 elements", name);
  if (output) {
    // one of the two axes steps over whole rows, the other over whole runs of the first
    int64_t cnt_a = heads, s_a = hs, cnt_b = tokens, s_b = ts;
    if (cnt_b > 1 && (cnt_a == 1 || s_b < s_a)) {
      cnt_a = tokens, s_a = ts, cnt_b = heads, s_b = hs;
    }
    const __int128 run = cnt_a > 1 ? (__int128)(cnt_a - 1) * s_a + n : (__int128)n;
    if ((cnt_a > 1 && s_a < n) || (cnt_b > 1 && s_b < run))
      return set_error(NSP_EINVAL, "%s: rows of an output overlap (strides %lld, %lld; %lld elements a row)", name,
                       (long long)ts, (long long)hs, (long long)n);
  }
  return NSP_OK;
}

inline bool same_view(const nsp_rows *a, const nsp_rows *b, int64_t tokens, int64_t heads) {
  return a->data == b->data && (tokens <= 1 || a->token_stride == b->token_stride) &&
         (heads <= 1 || a->head_stride == b->head_stride);
}

// In place, or apart.
inline nsp_status check_overlap(const nsp_rows *in, const char *in_name, const nsp_rows *out, const char *out_name,
                         int64_t tokens, int64_t heads, int64_t n, int64_t es) {
  if (tokens == 0 || same_view(in, out, tokens, heads)) return NSP_OK;
  const auto bytes = [&](const nsp_rows *r) {
    return (uintptr_t)(((tokens - 1) * r->token_stride + (heads - 1) * r->head_stride + n) * es);
  };
  const uintptr_t a = reinterpret_cast<uintptr_t>(in->data), b = reinterpret_cast<uintptr_t>(out->data);
  if (a < b + bytes(out) && b < a + bytes(in))
    return set_error(NSP_EINVAL, "%s overlaps %s without being the same view", out_name, in_name);
  return NSP_OK;
}

inline RowView view(const nsp_rows *r) {
  return RowView{static_cast<char *>(r->data), r->token_stride, r->head_stride};
}

inline nsp_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return set_error(NSP_OK, nullptr);
  return set_error(NSP_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace checks
}  // namespace nsp
