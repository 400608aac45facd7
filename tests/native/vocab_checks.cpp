// The vocabulary's operators on the CPU, for sanitizers: their plans over seeded
// random sizes, and their host code with launchers that record what they were given.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>

#include "nsp.h"
#include "vocab_internal.hpp"

static std::string g_error;
static int g_launches = 0;
static nsp::LinearArgs g_linear;
static nsp::DistillArgs g_distill;
static nsp::EmbedArgs g_embed;

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
hipError_t launch_linear_logp_fwd(const LinearArgs &a, hipStream_t) { ++g_launches; g_linear = a; return hipSuccess; }
hipError_t launch_linear_logp_bwd(const LinearArgs &a, hipStream_t) { ++g_launches; g_linear = a; return hipSuccess; }
hipError_t launch_distill_fwd(bool, const DistillArgs &a, hipStream_t) { ++g_launches; g_distill = a; return hipSuccess; }
hipError_t launch_distill_bwd(bool, const DistillArgs &a, hipStream_t) { ++g_launches; g_distill = a; return hipSuccess; }
hipError_t launch_embedding_fwd(bool, bool, const EmbedArgs &a, hipStream_t) { ++g_launches; g_embed = a; return hipSuccess; }
hipError_t launch_embedding_bwd(bool, bool, const EmbedArgs &a, hipStream_t) { ++g_launches; g_embed = a; return hipSuccess; }
}  // namespace nsp

#define CHECK(x)                                                                   \
  do {                                                                             \
    if (!(x)) {                                                                    \
      std::fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #x, g_error.c_str());   \
      std::exit(1);                                                                \
    }                                                                              \
  } while (0)

namespace plan = nsp::plan;
static std::mt19937_64 g_rng(7);
static int64_t spread(int64_t lo, int64_t hi) {
  const double u = std::uniform_real_distribution<double>(std::log((double)lo), std::log((double)hi))(g_rng);
  const int64_t v = (int64_t)std::llround(std::exp(u));
  return v < lo ? lo : v > hi ? hi : v;
}
static int64_t pick(int64_t n) { return (int64_t)(g_rng() % (uint64_t)n); }

static void linear_plans(int64_t T, int dim, int V) {
  const plan::LinearFwd f = plan::linear_fwd(T, dim, V);
  CHECK(f.tile == 32 || f.tile == 64 || f.tile == 128 || f.tile == 256);
  CHECK(f.panel >= T || f.panel == plan::linear_panel(f.tiles_p));
  CHECK(f.panel % f.tile == 0 && f.tiles_p * plan::kTileP >= V);
  CHECK((f.tiles_p * (f.panel / f.tile) + 8) * 512 < int64_t(1) << 32);   // threads of a launch
  CHECK(f.target_off >= (size_t)(f.tiles_p * f.panel * 16) && f.z_off >= f.target_off + (size_t)f.panel * 4);
  CHECK(f.split >= 1 && (f.split == 1 || (T <= f.panel && dim / f.split >= 512)));
  CHECK(f.bytes >= f.z_off + (f.split > 1 ? (size_t)f.split * f.panel * f.tiles_p * plan::kTileP * 4 : 0));
  CHECK(f.split * f.tiles_p * (f.panel / f.tile) <= (f.split > 1 ? plan::kUnits : INT32_MAX - 8));
  const plan::LinearBwd b = plan::linear_bwd(T, dim, V);
  CHECK(b.rows >= T && b.rows % b.tile == 0 && b.rows < T + b.tile);
  CHECK(b.piece % plan::kTileP == 0 && b.pieces >= 1);
  CHECK((int64_t)b.piece * b.pieces >= V && (int64_t)b.piece * (b.pieces - 1) < V);
  CHECK(b.dim >= dim && b.dim % 64 == 0);
  CHECK(b.split_x >= 1 && b.split_x <= 64 && b.split_w >= 1 && b.split_w <= 64);
  CHECK(b.split_z == 1 || (b.pieces == 1 && dim / b.split_z >= 512));
  CHECK(b.z_off >= b.dl_off + (size_t)b.copies * b.rows * b.piece * 2 && b.bytes >= b.z_off + (b.split_z > 1 ? (size_t)b.split_z * b.rows * b.piece * 4 : 0));
  // a part of 256 k at least
  CHECK(b.split_x == 1 || b.piece / b.split_x >= 256);
  CHECK(b.split_w == 1 || T / b.split_w >= 256);
  const int64_t cols = plan::ceil_div(dim, plan::kTileP);
  CHECK((b.piece / plan::kTileP * (b.rows / b.tile) + 8) * 512 < int64_t(1) << 32);
  CHECK(cols * plan::ceil_div(b.copies * b.rows, b.tile_x) * b.split_x + cols * (b.piece / plan::kTileP) * b.split_w < INT32_MAX - 16);
  const int64_t n_x = cols * plan::ceil_div(b.copies * T, b.tile_x);
  if (n_x * b.split_x <= plan::kUnits) {
    const int beside = plan::linear_split_beside(b.split_x, n_x, b.piece, cols * (b.piece / plan::kTileP) * b.split_w, plan::ceil_div(T, b.split_w));
    CHECK(beside >= 1 && beside <= b.split_x);
  }
  // one after another, none over the next
  const size_t off[] = {b.count_off, b.order_off, b.place_off, b.coef_off, b.target_off, b.x_off, b.dl_off, b.sum_x_off, b.sum_w_off, b.bytes};
  const size_t need[] = {4, (size_t)b.rows * 4, (size_t)T * 4, (size_t)b.rows * 16, (size_t)b.rows * 4, (size_t)b.copies * T * b.dim * 2,
                         (size_t)b.copies * b.rows * b.piece * 2, b.pieces > 1 || b.split_x > 1 || b.copies > 1 ? (size_t)b.split_x * b.copies * b.rows * dim * 4 : 0,
                         b.split_w > 1 ? (size_t)b.split_w * (V < b.piece ? V : b.piece) * dim * 4 : 0};
  for (int i = 0; i < 9; ++i) CHECK(off[i] % 256 == 0 && off[i] + need[i] <= off[i + 1]);
}

static void embed_plans(int64_t T, int dim, int V) {
  const plan::EmbedBwd f = plan::embed_bwd(T, dim, V);
  CHECK(f.chunk % 8 == 0 && f.chunk <= 128 && (int64_t)f.chunk * f.chunks >= T && (int64_t)f.chunk * (f.chunks - 1) < T);
  CHECK(f.bits >= 1 && f.bits <= plan::kSortBits && f.passes * f.bits >= 1 && ((int64_t)V >> (f.passes * f.bits)) == 0);   // the key V too
  CHECK((f.blocks == 0) == (T <= plan::kSortWhole) && (f.blocks == 0 || (int64_t)f.blocks * plan::kSortBlock >= T));
  const size_t list = (size_t)T * 4, hist = f.blocks ? ((size_t)(f.blocks + 1) << f.bits) * 4 : 0;
  CHECK(f.token_off[0] >= f.key_off[0] + list);
  if (f.blocks) {
    CHECK(f.key_off[1] >= f.token_off[0] + list && f.token_off[1] >= f.key_off[1] + list && f.hist_off >= f.token_off[1] + list);
    CHECK(f.flag_off >= f.hist_off + hist && f.part_off >= f.flag_off + (size_t)V);
  } else {
    CHECK(f.part_off >= f.token_off[0] + list);
  }
  CHECK(f.bytes >= f.part_off + (f.chunks > 1 ? (size_t)f.chunks * 2 * dim * 4 : 0));
  if (plan::embed_few(T, dim, 4)) CHECK(T <= plan::kEmbedFew);


}

static nsp_rows rows_at(uintptr_t at, int64_t stride) { return nsp_rows{reinterpret_cast<void *>(at), stride, 0}; }

// Whether extents [a, a + n) and [b, b + m) meet.
static bool meet(uintptr_t a, uintptr_t n, uintptr_t b, uintptr_t m) { return a < b + m && b < a + n; }

static void calls() {
  const uintptr_t base = uintptr_t(1) << 40;
  int64_t targets[1];
  float v[1];
  for (int i = 0; i < 20000; ++i) {
    const int64_t T = pick(6), dim = 8 * (1 + pick(4)), V = 1 + pick(9);
    const auto place = [&](int64_t n) { return rows_at(base + 16 * (uintptr_t)pick(300), n + 8 * pick(3)); };
    const nsp_rows x = place(dim), w = place(dim), dx = place(dim), dw = place(dim);
    const nsp_dtype g = pick(2) ? NSP_F32 : NSP_BF16;
    const uintptr_t es = g == NSP_F32 ? 4 : 2;
    const bool has_dx = pick(4) > 0, has_dw = pick(4) > 0;
    const auto extent = [&](const nsp_rows &r, int64_t n, uintptr_t e) { return n > 0 ? (uintptr_t)((n - 1) * r.token_stride + dim) * e : 0; };
    const auto at = [](const nsp_rows &r) { return reinterpret_cast<uintptr_t>(r.data); };
    const auto over = [&](const nsp_rows &a, int64_t na, uintptr_t ea, const nsp_rows &b, int64_t nb, uintptr_t eb) {
      return na > 0 && nb > 0 && meet(at(a), extent(a, na, ea), at(b), extent(b, nb, eb));
    };
    bool bad = false;
    if (has_dx) bad |= over(dx, T, es, x, T, 2) || (T > 0 && over(dx, T, es, w, V, 2));
    if (has_dw) bad |= over(dw, V, es, x, T, 2) || (T > 0 && over(dw, V, es, w, V, 2));
    if (has_dx && has_dw) bad |= over(dw, V, es, dx, T, es);
    const int before = g_launches;
    const nsp_status st = nsp_linear_logp_bwd(g, T, (int32_t)dim, (int32_t)V, &x, &w, targets, 1.f, v, v, v, v, v, has_dx ? &dx : nullptr,
                                              has_dw ? &dw : nullptr, reinterpret_cast<void *>(base << 1), size_t(1) << 40, nullptr);
    CHECK((st == NSP_OK) == !bad);
    CHECK(g_launches == before + (!bad && (has_dx || has_dw) ? 1 : 0));
    if (st == NSP_OK && (has_dx || has_dw)) CHECK(g_linear.n_tokens == T && g_linear.dim == dim && g_linear.vocab == V && !g_linear.dx == !has_dx);
    // the embedding's table and rows
    const nsp_status se = nsp_embedding_bwd(g, NSP_BF16, T, (int32_t)dim, (int32_t)V, targets, &x, 1.f, &dw, reinterpret_cast<void *>(base << 1),
                                            size_t(1) << 40, nullptr);
    CHECK((se == NSP_OK) == !over(dw, V, es, x, T, 2));
    const nsp_status sf = nsp_embedding_fwd(g, NSP_BF16, T, (int32_t)dim, (int32_t)V, targets, &w, 1.f, &dx, nullptr);
    CHECK((sf == NSP_OK) == !over(dx, T, 2, w, V, es));
    // workspaces: a byte less is refused
    const size_t need = nsp_linear_logp_fwd_workspace(T, (int32_t)dim, (int32_t)V);
    CHECK((need == 0) == (T == 0));
    if (need) {
      void *const ws = reinterpret_cast<void *>(base << 1);
      CHECK(nsp_linear_logp_fwd(T, (int32_t)dim, (int32_t)V, &x, &w, targets, 1.f, v, v, v, ws, need, nullptr) == NSP_OK);
      CHECK(nsp_linear_logp_fwd(T, (int32_t)dim, (int32_t)V, &x, &w, targets, 1.f, v, v, v, ws, need - 1, nullptr) == NSP_EWORKSPACE);
    }
  }
}

int main() {
  for (int i = 0; i < 20000; ++i) {
    const int V = (int)spread(1, plan::kLinearMaxVocab), dim = (int)(8 * spread(1, plan::kLinearMaxDim / 8));
    linear_plans(spread(1, plan::kLinearMaxTokens), dim, V);
    linear_plans(spread(1, 4096), (int)(8 * spread(1, 1024)), (int)spread(1, 200000));
    embed_plans(spread(1, plan::kEmbedMaxTokens), (int)spread(1, plan::kEmbedMaxDim), (int)spread(1, plan::kEmbedMaxVocab));
    embed_plans(spread(1, 40000), (int)spread(1, 8192), (int)spread(1, 200000));
  }
  for (const int V : {1, 2, 255, 256, 257, 511, 512, 513, (1 << 18) - 1, 1 << 18, (1 << 27) - 1, 1 << 30}) embed_plans(20000, 64, V);
  calls();
  std::printf("vocabulary checks ok\n");
  return 0;
}
