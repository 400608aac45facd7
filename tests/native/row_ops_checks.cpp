// The row operators' host code on the CPU, for sanitizers: argument checks,
// overlap rules against brute force, workspace sizes, FastDiv, the rotary
// frequencies.  The launchers are stand-ins that record what they were given.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <string>

#include "nsp.h"
#include "nsp_internal.hpp"

static std::string g_error;
static int g_launches = 0;
static nsp::RotaryArgs g_rotary;
static nsp::NormArgs g_norm;
static nsp::LogpArgs g_logp;
static nsp::LogpBwdArgs g_logp_bwd;

namespace nsp {
int32_t set_error(int32_t status, const char *fmt, ...) {
  char buf[512];
  buf[0] = 0;
  if (fmt) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
  }
  g_error = buf;
  return status;
}
hipError_t timed_call(KernelId id, hipStream_t, hipError_t (*launch)(void *), void *ctx) {
  if (id < 0 || id >= kNumKernels) abort();
  return launch(ctx);
}
hipError_t launch_rotary(bool, bool, const RotaryArgs &a, hipStream_t) { ++g_launches; g_rotary = a; return hipSuccess; }
hipError_t launch_norm_fwd(bool, const NormArgs &a, hipStream_t) { ++g_launches; g_norm = a; return hipSuccess; }
hipError_t launch_norm_bwd(bool, const NormArgs &a, hipStream_t) { ++g_launches; g_norm = a; return hipSuccess; }
hipError_t launch_token_logp_fwd(bool, const LogpArgs &a, hipStream_t) { ++g_launches; g_logp = a; return hipSuccess; }
hipError_t launch_token_logp_bwd(bool, const LogpBwdArgs &a, hipStream_t) { ++g_launches; g_logp_bwd = a; return hipSuccess; }
int norm_bwd_parts(int64_t rows, int n, bool) { return rows <= 200 || rows * 8 <= n ? 0 : (int)(rows < 768 ? rows : 768); }
int token_logp_parts(int64_t n, int vocab) { return n > 0 && n < 64 && vocab > 4096 ? 8 : 1; }
}  // namespace nsp

#define CHECK(x)                                                          \
  do {                                                                    \
    if (!(x)) {                                                           \
      std::fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #x, g_error.c_str()); \
      std::exit(1);                                                       \
    }                                                                     \
  } while (0)

static char *const kBase = reinterpret_cast<char *>(uintptr_t(1) << 40);   // never dereferenced

// The bytes of a view's elements, and whether two rows share one.
static bool bytes_of(const nsp_rows &r, int64_t T, int64_t H, int n, int es, std::set<int64_t> *out) {
  bool twice = false;
  for (int64_t t = 0; t < T; ++t)
    for (int64_t h = 0; h < H; ++h)
      for (int e = 0; e < n; ++e)
        twice |= !out->insert((static_cast<char *>(r.data) - kBase) + (t * r.token_stride + h * r.head_stride + e) * es).second;
  return twice;
}

int main() {
  std::mt19937_64 rng(5);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };

  for (int i = 0; i < 200000; ++i) {   // FastDiv: any divisor and dividend below 2^31
    const uint32_t d = (uint32_t)(i < 2000 ? i + 1 : (pick(1, INT32_MAX) >> pick(0, 30)) + 1), x = (uint32_t)pick(0, INT32_MAX);
    if (d > INT32_MAX) continue;
    const nsp::FastDiv f(d);
    CHECK(f.quot(x) == x / d && f.quot(INT32_MAX) == INT32_MAX / d && f.quot(0) == 0 && f.quot(d - 1) == 0 && f.quot(d) == 1);
  }

  int accepted = 0, refused = 0;
  for (int i = 0; i < 60000; ++i) {    // views: what is taken never overlaps itself or, but in place, its input
    const int64_t T = pick(0, 3);
    const int H = (int)pick(1, 3), n = (int)pick(1, 6), es = pick(0, 1) ? 2 : 4;
    auto view = [&] { return nsp_rows{kBase + pick(0, 30) * es, pick(0, 20), pick(0, 20)}; };
    nsp_rows x = view(), y = pick(0, 3) ? view() : x;
    const int before = g_launches;
    const nsp_status st = nsp_norm_fwd(NSP_NORM_RMS, es == 2 ? NSP_BF16 : NSP_F32, NSP_F32, T, H, n, &x, nullptr, nullptr, 1e-6f, &y, nullptr,
                                       nullptr, nullptr);
    std::set<int64_t> in, out;
    bytes_of(x, T, H, n, es, &in);
    const bool twice = bytes_of(y, T, H, n, es, &out);
    bool meet = false;
    for (int64_t b : out) meet |= in.count(b) != 0;
    const bool same = x.data == y.data && (T <= 1 || x.token_stride == y.token_stride) && (H <= 1 || x.head_stride == y.head_stride);
    if (st == NSP_OK) {
      ++accepted;
      CHECK(!twice && (!meet || same) && g_launches == before + (T > 0));
      if (T > 0) CHECK(g_norm.rows == T * H && g_norm.n == n && g_norm.rms && (int)g_norm.heads.d == H);
    } else {
      ++refused;
      CHECK(st == NSP_EINVAL && g_launches == before && !g_error.empty() && T > 0);
    }
  }
  CHECK(accepted > 5000 && refused > 5000);

  for (int i = 0; i < 20000; ++i) {    // sizes at and past the limits: refused or launched, never out of range
    const int64_t T = pick(0, 1) ? pick(-2, 4) : pick(INT32_MAX - 2LL, INT32_MAX + 2LL);
    const int H = (int)(pick(0, 1) ? pick(-1, 3) : pick(65535, 65537)), D = (int)pick(-1, 260), r = (int)pick(-1, 260);
    nsp_rows q{kBase, pick(0, 3) ? (int64_t)H * D : (int64_t)1 << pick(30, 62), D}, k = q;
    const int before = g_launches;
    const nsp_status st = nsp_rotary_fwd(NSP_ROTARY_HALF, NSP_BF16, T, D, r, reinterpret_cast<double *>(kBase), 1.f,
                                         reinterpret_cast<int64_t *>(kBase), H, &q, &q, 1, &k, &k, nullptr);
    CHECK(st == NSP_OK || g_launches == before);
    if (st == NSP_OK && T > 0)
      CHECK(g_rotary.half * 2 == r && r <= D && D <= 256 && !g_rotary.copy[0] && T * (H + 1) <= INT32_MAX && g_rotary.sign == 1.f);
    const int V = (int)(pick(0, 1) ? pick(-1, 9000) : pick((1 << 30) - 1, (1 << 30) + 1)), top = (int)pick(-1, 66);
    const size_t ws = nsp_token_logp_workspace(T, V, top);
    CHECK(ws <= (4u << 20) && nsp_norm_bwd_workspace(T, H, D) <= (size_t)8192 * 65536 + 1024);
    const nsp_status s2 = nsp_token_logp_fwd(NSP_F32, T, V, kBase, V, reinterpret_cast<int64_t *>(kBase), 1.f, reinterpret_cast<float *>(kBase),
                                             reinterpret_cast<float *>(kBase), nullptr, top, reinterpret_cast<float *>(kBase),
                                             reinterpret_cast<int64_t *>(kBase), kBase, ws, nullptr);
    if (s2 == NSP_OK && T > 0) {
      CHECK(g_logp.parts >= 1 && g_logp.parts <= nsp::kLogpMaxParts && g_logp.vocab == V);
      if (g_logp.parts > 1)
        CHECK((char *)(g_logp.part_sums + T * g_logp.parts) <= (char *)g_logp.part_top &&
              (char *)(g_logp.part_top + T * g_logp.parts * top) <= kBase + ws);
    }
  }

  double f[512];
  float scale = 0.f;
  for (int i = 0; i < 5000; ++i) {
    const int r = (int)pick(-2, 1030);
    const nsp_status st = nsp_rotary_frequencies(r, std::pow(10.0, (double)pick(-2, 8)), (nsp_rotary_scaling)pick(-1, 4), (double)pick(0, 40),
                                                 (double)pick(-1, 100000), (double)pick(-1, 3), (double)pick(0, 64), f, &scale);
    CHECK(st == NSP_OK || st == NSP_EINVAL);
    if (st == NSP_OK)
      for (int k = 0; k < r / 2; ++k) CHECK(std::isfinite(f[k]) && f[k] > 0);
  }
  std::puts("row checks ok");
  return 0;
}
