// How the vocabulary's operators divide their work: tiles, pieces and parts.
// Rules of the host, without HIP, on sizes and types alone.
#pragma once

#include <cstddef>
#include <cstdint>

namespace nsp {
namespace plan {

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
constexpr size_t pad256(size_t x) { return (x + 255) & ~size_t(255); }

// ----------------------------------- log probabilities from hidden rows --

constexpr int64_t kLinearMaxTokens = 1 << 22;
constexpr int kLinearMaxDim = 1 << 16, kLinearMaxVocab = 1 << 24;
constexpr int64_t kLinearMaxStride = 1 << 20;   // offsets within a tile stay below 2^31 bytes
constexpr int kTileP = 256;                     // vocabulary rows, or columns of a gradient, of a tile

// Compute units that a product's tiles should keep busy.
constexpr int kUnits = 256;

// Tokens of a tile of logits.  Past 128 tokens, 128 or 256: the tiles of 128 take some
// 0.56 of the time, and leave fewer compute units idle in their last turn.
constexpr int linear_tile(int64_t n_tokens, int vocab) {
  if (n_tokens <= 128) return n_tokens <= 32 ? 32 : n_tokens <= 64 ? 64 : 128;
  const int64_t p = ceil_div(vocab, kTileP), half = ceil_div(p * ceil_div(n_tokens, 128), kUnits), whole = ceil_div(p * ceil_div(n_tokens, 256), kUnits);
  return 56 * half < 100 * whole ? 128 : 256;
}

// Tokens of the forward that are worked on together, at most: 16 bytes are kept of each
// and tile of the vocabulary (256 MB at 131072 rows).  Fewer of large vocabularies: 1 GB,
// but 4096 tokens at least.
constexpr int64_t kLinearPanel = 32768;
constexpr int64_t linear_panel(int64_t tiles_p) {
  int64_t n = kLinearPanel;
  while (n > 4096 && n * tiles_p > (int64_t(1) << 26)) n /= 2;
  return n;
}

// Parts of the logits' sums over dim, where their tiles are too few: of 512 k at least,
// and three at least, since they are written and read once more.  (us whole and in parts,
// forward: 8 x 4400 of 9040 rows 48 and 24, 1 x 4096 of 4000 29 and 15, 600 x 8192 of 2000 73
// and 36, 1486 x 2176 of 1285 29 and 28; backward: 4 x 4616 of 2740 72 and 39, 16 x 4472 of
// 14375 118 and 94.  In two parts: 1000 x 2048 of 4000 forward 28 and 34, 2000 x 1024 of 1000
// backward 59 and 63)
constexpr int linear_logit_split(int64_t tiles, int dim) {
  int64_t s = kUnits / tiles;
  const int64_t most = dim / 512;
  s = s < most ? s : most;
  return (int)(s < 3 ? 1 : s > 16 ? 16 : s);
}

struct LinearFwd {
  int tile;
  int split;                   // parts of the logits' sums
  int64_t panel;               // tokens, a multiple of the tile or all of them
  int64_t tiles_p;
  size_t part_off, target_off, z_off, bytes;
};
constexpr LinearFwd linear_fwd(int64_t n_tokens, int dim, int vocab) {
  LinearFwd f{};
  f.tile = linear_tile(n_tokens, vocab);
  f.tiles_p = ceil_div(vocab, kTileP);
  f.panel = linear_panel(f.tiles_p);
  if (n_tokens < f.panel) f.panel = round_up(n_tokens, f.tile);
  f.part_off = 0;
  f.target_off = pad256((size_t)f.tiles_p * f.panel * 16);
  f.z_off = f.target_off + pad256((size_t)f.panel * 4);
  // (more than one part: one panel)
  f.split = n_tokens > 0 ? linear_logit_split(f.tiles_p * ceil_div(n_tokens, f.tile), dim) : 1;
  f.bytes = f.z_off + (f.split > 1 ? (size_t)f.split * f.panel * f.tiles_p * kTileP * 4 : 0);
  return f;
}

// Parts of a product's sums over k, where its tiles are too few: of 256 k at least.
constexpr int linear_split(int64_t tiles, int64_t n_k) {
  int64_t s = tiles > 0 ? kUnits / tiles : 1;
  const int64_t most = n_k / 256;
  s = s < most ? s : most;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}
// Parts of dx's sums where its tiles (n_x a part) run before n_w tiles of dw in one launch:
// those up to `most` that let the compute units end soonest.  A tile takes its
// stages of 64 k and some 4 to store.  (Calls with `most` and with these, us: 777 x 1000 x
// 50021, where 16 parts leave a fourth turn of 16 tiles of dw, 295 and 291; 64 x 1024 x
// 32000 56 and 49; 300 x 2048 x 4000 58 and 52; 300 x 1024 x 50000 152 and 153.)
constexpr int linear_split_beside(int most, int64_t n_x, int64_t k_x, int64_t n_w, int64_t k_w) {
  int best = most;
  int64_t least = INT64_MAX;
  for (int s = most; s >= 1 && 2 * s >= most; --s) {
    const int64_t x = ceil_div(ceil_div(k_x, s), 64) + 4, w = ceil_div(k_w, 64) + 4, idle = kUnits - n_x * s;
    const int64_t beside = idle * (x / w), left = n_w > beside ? n_w - beside : 0, end = x + ceil_div(left, kUnits) * w;
    if (end < least) {
      least = end;
      best = s;
    }
  }
  return best;
}
// Tokens that one workgroup finds the rows of, which then every workgroup of the
// gathering does for itself.
constexpr int kLinearFew = 1024;

// The gradient of the logits goes into the products as bf16, rounded once, or as two bf16
// numbers, itself and what its rounding leaves (2^-16).  One rounding leaves some 0.0017 of a
// gradient's 2-norm: a token's dx and a rare id's dw are a few terms, and there it does not
// average.  Two numbers where the caller takes float32 gradients, of any number of tokens;
// they are twice the products of dx and dw.  bf16 gradients, whose own rounding is 0.0017
// too, take them up to so many tokens, where the weight's bytes are most of the time and the
// second number is cheap (0.0017 instead of 0.0022 to 0.0026 in all; us with one number and two: 4 x
// 4616 x 2740 39 and 42, 25 x 384 x 29140 33 and 40, 64 x 1024 x 32000 50 and 64, 100 x 704 x
// 12000 42 and 52).  In such calls the second numbers are rows of their own beside the first,
// one more tile's work at most; past them they go through the same tiles after the first
// (along k), so that neither x nor dx's sums are there twice.
constexpr int kLinearTwice = 128;

struct LinearBwd {
  int copies;                  // rows of a token
  int numbers;                 // bf16 numbers of an element of the logits' gradient
  int tile;                    // tokens of a tile of logits
  int tile_x;                  // tokens of a tile of dx
  int64_t rows;                // tokens, in whole tiles
  int piece;                   // vocabulary rows of a piece, in whole tiles
  int pieces;
  int dim;                     // elements between gathered rows: whole 128-byte lines
  int split_z, split_x, split_w;   // parts of the logits', dx's and dw's sums
  size_t count_off, order_off, place_off, coef_off, target_off, x_off, dl_off, z_off, sum_x_off, sum_w_off, bytes;
};
// The gradient of the logits is kept for one piece of the vocabulary at a time,
// some 2^28 numbers of it (512 MB): large enough that adding dx's float32 sums
// of one piece to the next costs little (a read and a write of T dim against
// 6 T dim piece operations: 2% at pieces of 32768).  From 65536 tokens on pieces stay at 4096
// rows, so that the memory grows with the tokens only; the sums are 8% there (4096 x 131072 of
// 8192 tokens 1330 TFLOP/s, of 65536 1244, of 262144 1225).  Two numbers an element: half
// the piece.
constexpr LinearBwd linear_bwd(int64_t n_tokens, int dim, int vocab, bool f32 = false) {
  LinearBwd f{};
  f.copies = n_tokens <= kLinearTwice ? 2 : 1;
  f.numbers = f32 ? 2 : f.copies;
  const int along = f.numbers / f.copies;        // times that a product goes over k
  f.tile = linear_tile(n_tokens, vocab);
  f.rows = round_up(n_tokens, f.tile);
  f.dim = (int)round_up(dim, 64);
  const int64_t all = round_up(vocab, kTileP);
  int64_t piece = (int64_t(1) << 28) / (f.rows > 0 ? along * f.rows : 1) / kTileP * kTileP;
  piece = piece < 4096 / along ? 4096 / along : piece;
  f.pieces = (int)(piece >= all ? 1 : ceil_div(all, piece));
  f.piece = (int)round_up(ceil_div(all, f.pieces), kTileP);
  f.pieces = (int)ceil_div(all, f.piece);
  const int64_t cols = ceil_div(dim, kTileP);
  f.tile_x = n_tokens <= 64 ? 64 : 256;
  f.split_x = linear_split(cols * ceil_div(f.copies * n_tokens, f.tile_x), f.piece);
  f.split_w = linear_split(cols * (f.piece / kTileP), n_tokens);
  size_t at = 0;
  f.count_off = at, at += 256;
  f.order_off = at, at += pad256((size_t)f.rows * 4);
  f.place_off = at, at += pad256((size_t)f.rows * 4);
  f.coef_off = at, at += pad256((size_t)f.rows * 16);
  f.target_off = at, at += pad256((size_t)f.rows * 4);
  f.x_off = at, at += pad256((size_t)f.copies * f.rows * f.dim * 2);
  f.dl_off = at, at += pad256((size_t)f.numbers * f.rows * f.piece * 2);
  f.sum_x_off = at;
  if (f.pieces > 1 || f.split_x > 1 || f.copies > 1) at += pad256((size_t)f.split_x * f.copies * f.rows * dim * 4);
  f.sum_w_off = at;
  if (f.split_w > 1) at += pad256((size_t)f.split_w * f.piece * dim * 4);
  // the logits' parts are read before those sums begin (more than one part: one piece)
  f.z_off = f.sum_x_off;
  f.split_z = n_tokens > 0 ? linear_logit_split(f.rows / f.tile * (f.piece / kTileP), dim) : 1;
  const size_t z_end = f.z_off + (f.split_z > 1 ? (size_t)f.split_z * f.rows * f.piece * 4 : 0);
  at = at > z_end ? at : z_end;
  f.bytes = n_tokens > 0 ? at : 0;
  return f;
}
// As a call runs it: dx's parts fewer where its tiles run beside dw's.
constexpr LinearBwd linear_bwd_call(int64_t n_tokens, int dim, int vocab, bool f32, bool dx, bool dw) {
  LinearBwd f = linear_bwd(n_tokens, dim, vocab, f32);
  const int64_t cols = ceil_div(dim, kTileP), x = cols * ceil_div(f.copies * n_tokens, f.tile_x);
  if (dx && dw && x * f.split_x <= kUnits)
    f.split_x = linear_split_beside(f.split_x, x, f.numbers / f.copies * (int64_t)f.piece, cols * (f.piece / kTileP) * f.split_w,
                                    ceil_div(f.numbers * n_tokens, f.split_w));
  return f;
}
// Of gradients of either type.
constexpr size_t linear_bwd_bytes(int64_t n_tokens, int dim, int vocab) {
  const size_t a = linear_bwd(n_tokens, dim, vocab, false).bytes, b = linear_bwd(n_tokens, dim, vocab, true).bytes;
  return a > b ? a : b;
}

// --------------------------------------------------------------- embedding --

constexpr int64_t kEmbedMaxTokens = 1 << 26;
constexpr int kEmbedMaxVocab = 1 << 30, kEmbedMaxDim = 1 << 20;
constexpr int kSortBlock = 4096;                // tokens that a workgroup of a pass takes
constexpr int kSortWhole = 16384;               // tokens that one workgroup sorts by itself
constexpr int kSortBits = 9;                    // most of a digit

// Few tokens, of at most so many bytes of dy: a kernel of zeros and one that finds each
// id's tokens itself.  (us with a sort and without, three tables in turn, ids spread over the
// logarithm of the vocabulary.  Taken without: 24 x 4096 of 131072 rows 197 and 160, the zeros
// 159; 70 x 1393 float32 of 69335 75 and 61; 400 x 512 of 3000 15.0 and 7.0; 1000 x 512 of 3000
// 16.3 and 9.1; 2000 x 512 of 3000 18.6 and 13.5, of 32000 21.1 and 20.9; 1000 x 1024 float32 of
// 32000 32.7 and 30.2; 1000 x 2048 bf16 of 3000 17.7 and 11.4, of 131072 102 and 91, and between
// them, of 32000, where the sort hides beside the zeros, even: 33.5 and 33.8; 24 x 65536 of 5000 130
// and 103.  Taken with: 1500 x 1024 bf16 of 32000 20.7 and 21.5; 2000 x 1024 21.9 and 25.3; 2000 x 512
// float32 21.4 and 19.3.)  Where most tokens have one id the workgroup of that id adds them
// all: 2000 x 512 of 3000 rows, half of them one id's 63 us, all of them 174.
constexpr int kEmbedFew = 2048;
constexpr bool embed_few(int64_t n_tokens, int dim, int es) {
  return n_tokens <= kEmbedFew && n_tokens * dim * es <= (n_tokens <= 1024 ? 4 << 20 : 2 << 20);
}

struct EmbedBwd {
  int chunk, chunks;           // sorted tokens of a chunk
  int passes, bits;            // of the sort: digits of so many bits (a token id, or vocab for none)
  int blocks;                  // workgroups of a pass; 0: one workgroup sorts
  size_t key_off[2], token_off[2], hist_off, flag_off, part_off, bytes;
};
// A chunk's sorted tokens are summed by one wave a strip of columns; what a
// token's rows come to in a chunk they do not end in is kept in float32.  Longer
// chunks keep less (two rows each) and leave the joining wave of a frequent id fewer
// (of an id with a twelfth of the tokens, which is what the most frequent ones have:
// 100, of narrow rows 500); shorter ones leave more waves, and one chunk needs no
// second kernel.
constexpr EmbedBwd embed_bwd(int64_t n_tokens, int dim, int vocab) {
  EmbedBwd f{};
  if (n_tokens <= 0) return f;
  f.chunk = n_tokens <= 32 ? 32 : 8;
  while (f.chunk < 128 && n_tokens > (dim < 512 ? 6250 : 1250) * (int64_t)f.chunk) f.chunk *= 2;
  f.chunks = (int)ceil_div(n_tokens, f.chunk);
  int width = 1;
  while (width < 31 && (int64_t(1) << width) <= vocab) ++width;
  f.passes = (width + kSortBits - 1) / kSortBits;
  f.bits = (width + f.passes - 1) / f.passes;
  f.blocks = n_tokens <= kSortWhole ? 0 : (int)ceil_div(n_tokens, kSortBlock);
  size_t at = 0;
  for (int i = 0; i < (f.blocks ? 2 : 1); ++i) {
    f.key_off[i] = at, at += pad256((size_t)n_tokens * 4);
    f.token_off[i] = at, at += pad256((size_t)n_tokens * 4);
  }
  f.hist_off = at;
  if (f.blocks) at += pad256(((size_t)(f.blocks + 1) << f.bits) * 4);
  f.flag_off = at;
  if (f.blocks) at += pad256((size_t)vocab);
  f.part_off = at;
  if (f.chunks > 1) at += pad256((size_t)f.chunks * 2 * dim * 4);
  f.bytes = at;
  return f;
}

// Zeros in the rows of a table, a vector of 16 bytes a thread: rows side by side as one
// row, cut at lines of 128 bytes; others `lanes` threads a row.
constexpr int kFillThreads = 256, kFillBytes = 16 * kFillThreads;
constexpr int64_t kFillGrid = 1 << 23;          // (a launch holds less than 2^32 threads)
struct EmbedFill {
  int64_t rows, bytes, strips; // of a row
  int lanes;
  int grid;
};
constexpr EmbedFill embed_fill(int vocab, int64_t bytes, int64_t row_bytes) {
  EmbedFill f{};
  const bool whole = vocab == 1 || row_bytes == bytes;
  f.rows = whole ? 1 : vocab;
  f.bytes = whole ? vocab * bytes : bytes;
  f.strips = ceil_div(f.bytes + (whole ? 127 : 0), kFillBytes);
  f.lanes = 1;
  while (f.lanes < kFillThreads && 16 * f.lanes < bytes) f.lanes *= 2;
  const int64_t grid = ceil_div(f.rows, kFillThreads / f.lanes) * f.strips;
  f.grid = (int)(grid < kFillGrid ? grid : kFillGrid);
  return f;
}

}  // namespace plan
}  // namespace nsp
