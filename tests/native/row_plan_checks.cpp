// The rules by which the row operators divide their work (row_plans.hpp), as the
// library compiles them, and the workspaces that row_ops.cpp derives from them:
// every shape taken by some row, no row left out, workspaces within the stated
// sizes, sums no longer than the header says.
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "nsp.h"
#include "nsp_internal.hpp"

namespace nsp {
int32_t set_error(int32_t status, const char *, ...) { return status; }
hipError_t timed_call(KernelId, hipStream_t, hipError_t (*)(void *), void *) { abort(); }
hipError_t launch_rotary(bool, bool, const RotaryArgs &, hipStream_t) { abort(); }
hipError_t launch_norm_fwd(bool, const NormArgs &, hipStream_t) { abort(); }
hipError_t launch_norm_bwd(bool, const NormArgs &, hipStream_t) { abort(); }
hipError_t launch_token_logp_fwd(bool, const LogpArgs &, hipStream_t) { abort(); }
hipError_t launch_token_logp_bwd(bool, const LogpBwdArgs &, hipStream_t) { abort(); }
int norm_bwd_parts(int64_t rows, int n, bool f32) { return plan::norm_parts(rows, n, f32); }
int token_logp_parts(int64_t n, int vocab) { return plan::logp_parts(n, vocab); }
}  // namespace nsp

#define CHECK(x)                                                \
  do {                                                          \
    if (!(x)) {                                                 \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #x);      \
      std::exit(1);                                             \
    }                                                           \
  } while (0)

using namespace nsp::plan;

template <int N, class Rule>
static void shapes(const NormShape (&list)[N], int v, Rule rule) {
  int taken[N] = {};
  for (int n = 1; n <= 65536; ++n) {
    const NormShape s = rule(n);
    CHECK((s.lpr == 0) == (n < v || n > 16384));
    if (s.lpr == 0) continue;
    CHECK(s.lpr * s.ch * v >= n && s.lpr * s.rows() <= 1024 && s.lpr * s.rows() % 64 == 0);
    int i = 0;
    while (i < N && (list[i].lpr != s.lpr || list[i].ch != s.ch)) ++i;
    CHECK(i < N);
    ++taken[i];
  }
  for (int i = 0; i < N; ++i) CHECK(taken[i] > 0);
}

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int main() {
  shapes(kNormFwdBf16, 8, [](int n) { return norm_fwd_shape(n, false); });
  shapes(kNormFwdF32, 4, [](int n) { return norm_fwd_shape(n, true); });
  shapes(kNormBwdBf16, 8, [](int n) { return norm_bwd_shape(n, false); });
  shapes(kNormBwdF32, 4, [](int n) { return norm_bwd_shape(n, true); });

  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  for (int i = 0; i < 400000; ++i) {
    int64_t rows = pick(1, INT32_MAX) >> pick(0, 30);
    if (rows < 1) rows = 1;
    int n = (int)(pick(1, 65536) >> pick(0, 16));
    if (n < 1) n = 1;
    const bool f32 = rng() & 1;
    const NormShape f = norm_fwd_shape(n, f32), b = norm_bwd_shape(n, f32);
    const int fg = norm_fwd_grid(rows, f), parts = norm_parts(rows, n, f32), bg = norm_bwd_grid(rows, b, parts);
    CHECK(fg >= 1 && fg <= kFwdMost && fg <= row_groups(rows, f) && bg >= 1 && bg <= row_groups(rows, b) && parts >= 0 && parts <= 1024);
    CHECK((int64_t)bg <= (b.lpr > 0 && parts > 0 ? parts : kBwdMost));
    // terms of dw and db one after another: a lane's or strand's rows, the groups of a
    // workgroup (or its waves), the parts' strands, their waves
    int64_t longest;
    if (b.lpr > 0 && parts > 0) longest = up(row_groups(rows, b), bg) + b.rows();
    else if (b.lpr > 0) longest = up(rows, 64) + 16;
    else longest = up(parts > 0 ? up(rows, parts) : rows, 128) + 16;
    if (parts > 0) longest += up(parts, 128) + 16;
    CHECK(longest <= 128 + rows / 256);
    const size_t ws = nsp_norm_bwd_workspace(rows, 1, n);
    CHECK(ws <= (size_t)8192 * n + 1024 && ws >= (size_t)parts * 2 * n * 4 && ws % 256 == 0);

    const int64_t tokens = rows;
    const int vocab = (int)(pick(1, 1 << 30) >> pick(0, 29)) + 1, top = (int)pick(0, 64);
    const int lp = logp_parts(tokens, vocab);
    CHECK(lp >= 1 && lp <= kLogpMaxParts && (lp == 1 || tokens < 512));
    for (const int v : {4, 8}) {
      const int len = logp_part_len(vocab, lp, v);
      CHECK(len % v == 0 && (int64_t)len * lp >= vocab && (int64_t)len * (lp - 1) < vocab);
    }
    const size_t lw = nsp_token_logp_workspace(tokens, vocab, top);
    CHECK(lw <= (4u << 20) && lw % 256 == 0 && (lp > 1) == (lw > 0));
    if (lp > 1) CHECK(lw >= (size_t)tokens * lp * (16 + 8 * (size_t)top));
  }
  std::puts("row plan checks ok");
  return 0;
}
