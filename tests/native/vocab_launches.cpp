// The launches of the vocabulary's operators on the CPU, for sanitizers: what the launchers
// take from the plans over seeded random sizes, and the zeros of few tokens byte by byte.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "vocab_plans.hpp"

namespace plan = nsp::plan;

#define CHECK(x)                                                      \
  do {                                                                \
    if (!(x)) {                                                       \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #x);            \
      std::exit(1);                                                   \
    }                                                                 \
  } while (0)

static std::mt19937_64 g_rng(11);
static int64_t spread(int64_t lo, int64_t hi) {
  const double u = std::uniform_real_distribution<double>(std::log((double)lo), std::log((double)hi))(g_rng);
  const int64_t v = (int64_t)std::llround(std::exp(u));
  return v < lo ? lo : v > hi ? hi : v;
}
static int64_t pick(int64_t n) { return (int64_t)(g_rng() % (uint64_t)n); }

// Stages of 64 k until the units are through with n_x * s tiles of dx and n_w of dw.
static int64_t turns(int s, int64_t n_x, int64_t k_x, int64_t n_w, int64_t k_w) {
  const int64_t x = plan::ceil_div(plan::ceil_div(k_x, s), 64) + 4, w = plan::ceil_div(k_w, 64) + 4;
  std::vector<int64_t> free_at(plan::kUnits, 0);
  for (int64_t i = 0; i < n_x * s; ++i) free_at[i] += x;
  int64_t left = n_w;                            // as many as the idle units end while dx's run
  for (int64_t i = n_x * s; i < plan::kUnits; ++i) left -= x / w;
  return x + (left > 0 ? plan::ceil_div(left, plan::kUnits) * w : 0);
}

static void linear_calls(int64_t T, int dim, int V) {
  for (const bool f32 : {false, true}) {
    const plan::LinearBwd b = plan::linear_bwd(T, dim, V, f32);
    const int64_t cols = plan::ceil_div(dim, plan::kTileP);
    // numbers of an element: two for float32 gradients and few tokens
    CHECK(b.copies == (T <= plan::kLinearTwice ? 2 : 1) && b.numbers == (f32 || b.copies > 1 ? 2 : 1));
    CHECK(b.numbers == b.copies || b.tile_x == 256);
    CHECK(b.piece % plan::kTileP == 0 && (int64_t)b.piece * b.pieces >= V && (int64_t)b.piece * (b.pieces - 1) < V);
    CHECK(plan::linear_bwd_bytes(T, dim, V) >= b.bytes);
    // what is kept of the logits' gradient: 512 MB (few tokens, twice: 1 GB), or 8192 bytes a token, and what whole tiles add
    const size_t dl = (size_t)b.numbers * b.rows * b.piece * 2, all = (size_t)b.numbers * b.rows * plan::round_up(V, plan::kTileP) * 2;
    CHECK(dl <= all && (dl <= (size_t)b.copies * ((size_t(1) << 29) + (size_t)b.numbers * b.rows * 512) || dl <= 8192 * (size_t)b.rows + (size_t)b.rows * 512 * b.numbers));
    // one after another, none over the next; the logits' parts from sum_x on
    const size_t off[] = {b.count_off, b.order_off, b.place_off, b.coef_off, b.target_off, b.x_off, b.dl_off, b.sum_x_off, b.sum_w_off, b.bytes};
    const bool sums_x = b.pieces > 1 || b.split_x > 1 || b.copies > 1;
    const size_t need[] = {4, (size_t)b.rows * 4, (size_t)T * 4, (size_t)b.rows * 16, (size_t)b.rows * 4, (size_t)b.copies * T * b.dim * 2, dl,
                           sums_x ? (size_t)b.split_x * b.copies * b.rows * dim * 4 : 0,
                           b.split_w > 1 ? (size_t)b.split_w * (V < b.piece ? V : b.piece) * dim * 4 : 0};
    for (int i = 0; i < 9; ++i) CHECK(off[i] % 256 == 0 && off[i] + need[i] <= off[i + 1]);
    CHECK(b.split_z == 1 || (b.pieces == 1 && b.z_off + (size_t)b.split_z * b.rows * b.piece * 4 <= b.bytes));
    for (int k = 0; k < 4; ++k) {
      const bool dx = k & 1, dw = k & 2;
      const plan::LinearBwd c = plan::linear_bwd_call(T, dim, V, f32, dx, dw);
      // (the workspace is the plan's)
      CHECK(c.bytes == b.bytes && c.split_x >= 1 && c.split_x <= b.split_x && c.split_w == b.split_w && c.piece == b.piece);
      CHECK(c.split_x == b.split_x || (dx && dw));
      const int64_t n_x = cols * plan::ceil_div(b.copies * T, b.tile_x), n_w = cols * (b.piece / plan::kTileP) * b.split_w;
      if (dx && dw && n_x * b.split_x <= plan::kUnits) {
        const int64_t k_x = b.numbers / b.copies * (int64_t)b.piece, k_w = plan::ceil_div(b.numbers * T, b.split_w);
        CHECK(turns(c.split_x, n_x, k_x, n_w, k_w) <= turns(b.split_x, n_x, k_x, n_w, k_w));
      }
      CHECK((plan::round_up(cols * plan::ceil_div(b.copies * b.rows, b.tile_x) * c.split_x, 8) + plan::round_up(n_w, 8)) * 512 < int64_t(1) << 32 ||
            b.rows * (int64_t)dim > int64_t(1) << 36);
    }
  }
}

// The kernel of zeros, as its threads go: every byte of every row once or more, none beside.
static void fill(int vocab, int64_t bytes, int64_t row_bytes, int64_t skew) {
  const plan::EmbedFill f = plan::embed_fill(vocab, bytes, row_bytes);
  CHECK(f.grid >= 1 && f.grid <= plan::kFillGrid && (int64_t)f.grid * plan::kFillThreads < int64_t(1) << 32);
  CHECK(f.lanes >= 1 && plan::kFillThreads % f.lanes == 0);
  const int64_t extent = (vocab - 1) * row_bytes + bytes;
  std::vector<uint8_t> hit(extent, 0);
  const auto zero = [&](int64_t from, int64_t to) {
    CHECK(from >= 0 && to <= extent);
    for (int64_t i = from; i < to; ++i) hit[i] = 1;
  };
  const int per = plan::kFillThreads / f.lanes;
  const int64_t units = f.rows == 1 ? f.strips : plan::ceil_div(f.rows, per) * f.strips;
  CHECK(f.grid == units || f.grid == plan::kFillGrid);
  for (int64_t unit = 0; unit < units; ++unit)
    for (int t = 0; t < plan::kFillThreads; ++t) {
      if (f.rows == 1) {
        const int64_t at = unit * plan::kFillBytes - skew + 16 * t, lo = at > 0 ? at : 0, hi = at + 16 < f.bytes ? at + 16 : f.bytes;
        if (lo < hi) zero(lo, hi);
      } else {
        const int64_t group = unit / f.strips, v = group * per + t / f.lanes, c = (unit - group * f.strips) * plan::kFillBytes + 16 * (t % f.lanes);
        if (v >= f.rows || c >= f.bytes) continue;
        const int64_t from = f.bytes >= 16 ? (c < f.bytes - 16 ? c : f.bytes - 16) : 0;
        zero(v * row_bytes + from, v * row_bytes + (f.bytes >= 16 ? from + 16 : f.bytes));
      }
    }
  for (int64_t i = 0; i < extent; ++i) CHECK(hit[i] == (i % row_bytes < bytes || vocab == 1));
}

static void few_tokens(int64_t T, int dim, int V) {
  for (const int es : {2, 4}) {
    if (!plan::embed_few(T, dim, es)) continue;
    // a workgroup of 256 a token and strip of 64 vectors
    CHECK(T * plan::ceil_div(dim, 64 * (16 / es)) * 256 < int64_t(1) << 32);
    CHECK(T <= 2048 && T * dim * es <= 4 << 20);
    for (const int ews : {2, 4}) {
      const plan::EmbedFill f = plan::embed_fill(V, (int64_t)dim * ews, (int64_t)dim * ews);
      CHECK((int64_t)f.grid * plan::kFillThreads < int64_t(1) << 32 && f.strips * plan::kFillBytes >= f.bytes + 127);
    }
  }
}

int main() {
  for (int i = 0; i < 20000; ++i) {
    linear_calls(spread(1, plan::kLinearMaxTokens), (int)(8 * spread(1, plan::kLinearMaxDim / 8)), (int)spread(1, plan::kLinearMaxVocab));
    linear_calls(spread(1, 4096), (int)(8 * spread(1, 1024)), (int)spread(1, 200000));
    few_tokens(spread(1, 4096), (int)spread(1, plan::kEmbedMaxDim), (int)spread(1, plan::kEmbedMaxVocab));
  }
  for (const int64_t T : {1, 64, 65, 127, 128, 129, 256, 65536, 65537}) linear_calls(T, 4096, 131072);
  for (int i = 0; i < 600; ++i) {
    const int64_t bytes = 2 * spread(1, 6000), vocab = spread(1, 60);
    fill((int)vocab, bytes, bytes, 2 * pick(64));
    fill((int)vocab, bytes, bytes + 2 * (1 + pick(30)), 2 * pick(64));
  }
  std::printf("vocabulary launches ok\n");
  return 0;
}
