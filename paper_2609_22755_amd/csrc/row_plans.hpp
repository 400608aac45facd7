// How the row operators divide their work: lanes and vectors of a row, workgroups,
// parts.  Rules of the host, without HIP, on sizes and types alone.
#pragma once

#include <cstddef>
#include <cstdint>

namespace nsp {
namespace plan {

// ------------------------------------------------------------------- norms --

// Lanes of a row, and its vectors (of 16 bytes) a lane; 0 lanes: the wide kernels.
struct NormShape {
  int lpr, ch;
  constexpr int rows() const { return lpr > 0 && lpr < 256 ? 256 / lpr : 1; }   // of a workgroup
};

// The first of a list that holds the row is taken.  A wave holds a row as long
// as its lanes do (up to 32 elements each: sums without a barrier; float32 rows
// of 1111 in 5 vectors a lane 5.6 TB/s backward, in 4 of 128 lanes 5.0), then few
// wide groups; three vectors a lane where four would leave many empty (10000 bf16
// forward 5.3 TB/s in 3 of 512 lanes, 4.1 in 2 of 1024).
inline constexpr NormShape kNormFwdBf16[] = {{16, 1},  {16, 2},  {64, 1},  {64, 2},  {64, 3},  {64, 4},
                                             {128, 3}, {128, 4}, {256, 3}, {512, 2}, {512, 3}, {1024, 2}};
inline constexpr NormShape kNormFwdF32[] = {{16, 1},  {16, 2},  {64, 1},  {64, 2},  {64, 3},   {64, 4},  {128, 3},
                                            {128, 4}, {256, 3}, {512, 2}, {512, 3}, {1024, 2}, {1024, 4}};
inline constexpr NormShape kNormBwdBf16[] = {{16, 1}, {16, 2},  {64, 1},  {64, 2},  {64, 3}, {64, 4},
                                             {128, 3}, {128, 4}, {512, 2}, {512, 3}, {512, 4}};
inline constexpr NormShape kNormBwdF32[] = {{16, 1}, {16, 2}, {64, 1},  {64, 2},  {64, 3},  {64, 4},  {64, 5},
                                            {64, 6}, {64, 8}, {512, 2}, {512, 3}, {512, 4}, {1024, 4}};

// Every shape holds more than the one before it (or no row would take it), in 32
// elements a lane, 16 where 1024 lanes leave 128 registers each.
template <int N>
constexpr bool sound(const NormShape (&shapes)[N], int v) {
  for (int i = 0; i < N; ++i)
    if ((i > 0 && shapes[i].lpr * shapes[i].ch <= shapes[i - 1].lpr * shapes[i - 1].ch) || shapes[i].ch * v > (shapes[i].lpr < 1024 ? 32 : 16))
      return false;
  return true;
}
static_assert(sound(kNormFwdBf16, 8) && sound(kNormFwdF32, 4) && sound(kNormBwdBf16, 8) && sound(kNormBwdF32, 4), "a shape no row takes, or one too large");

template <int N>
constexpr NormShape shape_of(const NormShape (&shapes)[N], int v, int n) {
  const int vecs = (n + v - 1) / v;
  if (n < v) return {0, 0};
  for (const NormShape s : shapes)
    if (s.lpr * s.ch >= vecs) return s;
  return {0, 0};
}
constexpr NormShape norm_fwd_shape(int n, bool f32) { return f32 ? shape_of(kNormFwdF32, 4, n) : shape_of(kNormFwdBf16, 8, n); }
constexpr NormShape norm_bwd_shape(int n, bool f32) { return f32 ? shape_of(kNormBwdF32, 4, n) : shape_of(kNormBwdBf16, 8, n); }

constexpr int64_t row_groups(int64_t rows, NormShape sh) { return (rows + sh.rows() - 1) / sh.rows(); }

// The forward's workgroups take four row groups in turn, where there are so
// many (fewer reload the weights more often, more leave the last ones alone: rows
// of 8192 bf16 6.1 TB/s, with two 5.7, with eight 5.9).
constexpr int kFwdTurns = 4, kFwdLeast = 2048, kFwdMost = 1 << 21;
constexpr int norm_fwd_grid(int64_t rows, NormShape sh) {
  const int64_t groups = row_groups(rows, sh);
  const int64_t grid = groups / kFwdTurns > kFwdLeast ? groups / kFwdTurns : groups < kFwdLeast ? groups : kFwdLeast;
  return (int)(grid < kFwdMost ? grid : kFwdMost);
}

// Parts of dw and db, 1024 at most; 0: formed without any.
//
// As many workgroups as keep some 32 KB a compute unit on the way (a lane has
// its next row's vectors of x and dy in flight): more of them get in each
// other's way in memory (2 M rows of 128 bf16: three a compute unit 264 us, two
// 277, four 306), and each leaves a part; fewer leave it idle (120 K rows of 1111
// bf16, three vectors a lane: two 182 us, one 207).
constexpr int norm_parts(int64_t rows, int n, bool f32) {
  const NormShape sh = norm_bwd_shape(n, f32);
  // Few rows: without parts 24 x 4096 bf16 5.4 us, with them 11.3; 200 x 1000 6.8
  // and 9.1; 500 x 128 float32 8.3 and 7.1.  Wide ones longer: 600 x 8192 19.0 and
  // 24.9; 500 x 4096 24.8 and 18.3.
  if (rows <= 200 || (rows <= 640 && rows * 12 <= n)) return 0;
  // The widths of the wide kernels: parts of 4096 rows, 32 a strand one after another.
  if (sh.lpr == 0) return rows <= 4096 ? 0 : rows <= 1023 * 4096 ? (int)((rows + 4095) / 4096) : 1024;
  const int64_t groups = row_groups(rows, sh);
  int per_cu = sh.lpr > 256 || sh.ch > 3 ? 1 : sh.ch > 1 ? 2 : 3;
  while (per_cu > 1 && groups < 4 * 256 * per_cu) --per_cu;
  return (int)(groups < 256 * per_cu ? groups : 256 * per_cu);
}

// Workgroups of the backward's dx: one a part, where it leaves them.
constexpr int kBwdMost = 1024;
constexpr int norm_bwd_grid(int64_t rows, NormShape sh, int parts) {
  const int64_t groups = row_groups(rows, sh);
  return parts > 0 && sh.lpr > 0 ? parts : (int)(groups < kBwdMost ? groups : kBwdMost);
}

// ------------------------------------------------- token log probabilities --

// Most parts that a row of logits is split in.
constexpr int kLogpMaxParts = 64;

// Two workgroups a compute unit, each with 2048 elements at least.  (32 rows of
// 131072 with one alternative: 11.4 us, with four a compute unit 13.8, with eight
// 17.9; 1000 rows of 32000 with five, one part a row, 19.4, two 28.6.)
constexpr int logp_parts(int64_t n_tokens, int vocab) {
  if (n_tokens <= 0) return 1;
  const int64_t wanted = (512 + n_tokens - 1) / n_tokens, most = ((int64_t)vocab + 2047) / 2048;
  const int64_t p = wanted < most ? wanted : most;
  return (int)(p < kLogpMaxParts ? p : kLogpMaxParts);
}
// Elements of a part, in vectors of v.
constexpr int logp_part_len(int vocab, int parts, int v) { return (int)((((int64_t)vocab + parts - 1) / parts + v - 1) / v * v); }

}  // namespace plan
}  // namespace nsp
