// Log probabilities of given tokens straight from hidden rows and the
// vocabulary's weight, and their gradients, for gfx950: the logits
// a[t][v] = <x[t], w[v]> exist a tile at a time.
//
// Bound by the matrix cores: 2 T dim V operations forward, three times that
// backward (the logits are made again, dx and dw are a product each).  4096 x 4096 x
// 151643 forward 3.74 ms (1361 TFLOP/s); 8192 x 4096 x 131072, a tenth of the tokens
// ignored, backward 18.0 to 18.6 ms (1318 to 1280), with float32 gradients 31.5; a library's product of these sizes, its result stored
// to memory, 1366 to 1486 (NT).  The clock under this load is 1.6 to 1.7 GHz: power bounds
// both.  24 rows of 131072 x 4096, a read of the weight: 177 us (6.1 TB/s).
//
// Forward: a tile of 256 vocabulary rows and up to 256 tokens.  A lane holds one
// token of it, so the tile's maximum, sum and weighted sum of a token are made
// in registers and leave as 16 bytes a token and tile; a second kernel joins a
// token's tiles.
//
// Backward: the tokens whose gradient is not zero (ignored targets drop out) are
// gathered into rows side by side; then, piece by piece of the vocabulary,
//     dl = scale (k0 p + k1 p ln p + 1[target]) of the piece's logits, bf16
//     dw[piece] = dl^T x,   dx += dl w[piece]
// dl is rounded to bf16 (half a step, 2^-8 of each term at most), which the matrix
// instructions take; for float32 gradients, and of up to 128 tokens, what that rounding
// leaves goes in as a second number (2^-16; vocab_plans.hpp has what either costs).  Sums are
// float32, over pieces too.
#include "gemm_tile.hpp"
#include "row_common.hpp"
#include "vocab_internal.hpp"

namespace nsp {
namespace {

using tile::kAcross;
using tile::kAlong;
using tile::Product;

constexpr float kNegInf = -__builtin_inff();
constexpr float kNan = __builtin_nanf("");
constexpr float kLowest = -3.402823466e38f;
constexpr int kGroup = 4;      // neighbouring tiles of p that share q's in an L2

// A tile of logits: 256 vocabulary rows, NQ tokens.
template <int NQ>
struct LogitTile;
template <>
struct LogitTile<256> { typedef Product<kAlong, kAlong, 256, 256, 2, 4> P; };
template <>
struct LogitTile<128> { typedef Product<kAlong, kAlong, 256, 128, 2, 4> P; };
template <>
struct LogitTile<64> { typedef Product<kAlong, kAlong, 256, 64, 4, 2> P; };
template <>
struct LogitTile<32> { typedef Product<kAlong, kAlong, 256, 32, 8, 1> P; };

// The p of element i of a block, from the block's first.
__device__ __forceinline__ int p_of(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// 32 q's (one a lane pair) of 32 * NB p's, of a wave's sums, as rows of p: through
// LDS (32 * 32 * NB elements of the wave's own), 16 bytes a lane.  put(row, byte,
// 16 bytes) for rows below `rows`, elements below `cols`.
template <int NB, bool F32, class Put>
__device__ __forceinline__ void put_rows(const f32x16 *acc, char *lds, int rows, int cols, int lane_, Put put) {
  const int lane = hidden(lane_);
  constexpr int CH = NB * (F32 ? 8 : 4), PER = F32 ? 4 : 8;
  const int l32 = lane & 31, h = lane >> 5;
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
#pragma unroll
    for (int gq = 0; gq < 4; ++gq) {
      const f32x4 v = {acc[mb][4 * gq], acc[mb][4 * gq + 1], acc[mb][4 * gq + 2], acc[mb][4 * gq + 3]};
      const int c = F32 ? 8 * mb + 2 * gq + h : 4 * mb + gq;
      char *p = lds + 16 * (l32 * CH + (c ^ (l32 & (CH - 1))));
      if constexpr (F32) *(f32x4 *)p = v;
      else *(bf16x4 *)(p + 8 * h) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    }
#pragma unroll
  for (int j = 0; j < CH / 2; ++j) {
    const int row = (64 * j + lane) / CH, c = (64 * j + lane) % CH;
    const f32x4 v = *(const f32x4 *)(lds + 16 * (row * CH + (c ^ (row & (CH - 1)))));
    if (row < rows && c * PER < cols) put(row, 16 * c, v);
  }
}

// What is read back from the workspace as a number of rows or a row stays among the n
// there are, also where something else writes the workspace meanwhile.
__device__ __forceinline__ int rows_of(const int *count, int64_t n) { return (int)min((uint32_t)*count, (uint32_t)n); }
__device__ __forceinline__ int64_t row_of(const int *order, int64_t at, int64_t n) { return min((uint32_t)order[at], (uint32_t)n - 1); }

// ------------------------------------------------- logits of few tiles --

// Sums of a part of dim, in float32: [part][rows][cols], for calls whose tiles are fewer than
// the compute units.  Such a call is bound by what a unit has on its way from memory; the
// parts bring more units to bear (8 x 4400 of 9040 rows: 36 tiles 48 us, 7 parts each 24).
struct LogitParts {
  const char *w, *x;
  int64_t w_stride, x_stride;
  const int *count;            // rows of the n, null: all
  int n, vocab, dim;
  int split, tiles_p;
  int64_t rows, cols;          // whole tiles
  float *sums;

  // Columns c .. c + 3 of a row, the parts in order.
  __device__ __forceinline__ f32x4 at(int64_t row, int64_t c) const {
    const float *from = sums + row * cols + c;
    f32x4 z = *(const f32x4 *)from;
    for (int p0 = 1; p0 < split; p0 += 5) {
      f32x4 v[5];
#pragma unroll
      for (int j = 0; j < 5; ++j) v[j] = p0 + j < split ? *(const f32x4 *)(from + (p0 + j) * rows * cols) : f32x4{};
#pragma unroll
      for (int j = 0; j < 5; ++j) z += v[j];
    }
    return z;
  }
};

template <int NQ>
__global__ __launch_bounds__(512, 2) void linear_parts_kernel(LogitParts f) {
  typedef typename LogitTile<NQ>::P P;
  static_assert(P::kLds >= P::NW * 4096 * P::BP, "room for the rows that are stored");
  __shared__ __attribute__((aligned(1024))) char smem[P::kLds];
  const int n = f.count ? rows_of(f.count, f.n) : f.n;
  tile::Place at;
  if (!at.find(blockIdx.x, f.tiles_p, (n + NQ - 1) / NQ, f.split, kGroup)) return;
  P x;
  const int v0 = at.p * P::NP, q0 = at.q * NQ;
  const int len = (int)plan::round_up(plan::ceil_div(f.dim, f.split), tile::kStep);
  const int k0 = at.part * len, n_k = max(0, min(f.dim - k0, len));
  x.run(smem, typename P::LoadP(f.w, f.w_stride, v0, f.vocab, k0, n_k, x.wave, x.lane),
        typename P::LoadQ(f.x, f.x_stride, q0, n, k0, n_k, x.wave, x.lane), n_k);
#pragma unroll
  for (int q = 0; q < P::BQ; ++q) {
    float *out = f.sums + (at.part * f.rows + q0 + x.q0() + 32 * q) * f.cols + v0 + x.p0();
    put_rows<P::BP, true>(x.acc[q], smem + x.wave * (4096 * P::BP), 32, 32 * P::BP, x.lane,
                          [&](int row, int byte, f32x4 v) { *(f32x4 *)((char *)(out + row * f.cols) + byte) = v; });
  }
}

// Workgroups of `tiles` tiles: as many for each XCD.
int grid_of(int64_t tiles) { return (int)plan::round_up(tiles, kXcdQueues); }

hipError_t logit_parts(const LogitParts &f, int tile, hipStream_t s) {
  const int grid = grid_of(f.tiles_p * (f.rows / tile) * f.split);
  if (tile == 32) linear_parts_kernel<32><<<grid, 512, 0, s>>>(f);
  else if (tile == 64) linear_parts_kernel<64><<<grid, 512, 0, s>>>(f);
  else if (tile == 128) linear_parts_kernel<128><<<grid, 512, 0, s>>>(f);
  else linear_parts_kernel<256><<<grid, 512, 0, s>>>(f);
  return hipGetLastError();
}

// ----------------------------------------------------------------- forward --

struct FwdTiles {
  LinearArgs a;
  int64_t t0;                  // first token of the panel
  int64_t panel;
  int n;                       // its tokens
  int tiles_p, tiles_q;
  float4 *part;                // [tile of p][panel]: largest, sum, weighted sum
  float *at_target;            // [panel]
};

template <int NQ>
__global__ __launch_bounds__(512, 2) void linear_logp_tiles_kernel(FwdTiles f) {
  typedef typename LogitTile<NQ>::P P;
  __shared__ __attribute__((aligned(1024))) char smem[P::kLds];
  tile::Place at;
  if (!at.find(blockIdx.x, f.tiles_p, f.tiles_q, 1, kGroup)) return;
  P x;
  const int v0 = at.p * P::NP, q0 = at.q * NQ;
  const LinearArgs &a = f.a;
  x.run(smem, typename P::LoadP(a.w, a.w_stride, v0, a.vocab, 0, a.dim, x.wave, x.lane),
        typename P::LoadQ(a.x, a.x_stride, f.t0 + q0, f.t0 + f.n, 0, a.dim, x.wave, x.lane), a.dim);
  const int l32 = x.lane & 31, h = x.lane >> 5;
  const float c = a.scale * kLog2e;
  float4 *stat = (float4 *)smem;                 // [WP][NQ]
  const int vw = v0 + x.p0();
#pragma unroll
  for (int q = 0; q < P::BQ; ++q) {
    const int tok = q0 + x.q0() + 32 * q + l32;
    if (v0 + P::NP > a.vocab) {
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (vw + 32 * p + p_of(i, h) >= a.vocab) x.acc[q][p][i] = kNegInf;
    }
    const int64_t y = a.logp && tok < f.n ? a.targets[f.t0 + tok] : -1;
    const bool mine = y >= vw && y < vw + 32 * P::BP && y < a.vocab;
    if (__any(mine)) {
      const int e = mine ? (int)(y - vw) : -1;
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (e == 32 * p + p_of(i, h)) f.at_target[tok] = x.acc[q][p][i];
    }
    float m = kLowest;
#pragma unroll
    for (int p = 0; p < P::BP; ++p)
#pragma unroll
      for (int i = 0; i < 16; i += 2) m = fmaxf(fmaxf(m, x.acc[q][p][i]), x.acc[q][p][i + 1]);
    m = wave_max_halves(m);
    float s = 0.f, u = 0.f;
    const auto sums = [&](auto least) {
      s = u = 0.f;
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float d = (x.acc[q][p][i] - m) * c, e = fast_exp2(d);
          s += e;
          u = fmaf(e, least(d), u);
        }
    };
    sums([](float d) { return d; });
    // 0 times infinity: logits of -inf count for nothing (a NaN stays one in s)
    if (__any(u != u)) sums([](float d) { return fmaxf(d, -200.f); });
    s = wave_sum_halves(s);
    u = wave_sum_halves(u);
    if (h == 0) stat[x.wp * NQ + x.q0() + 32 * q + l32] = make_float4(m, s, u, 0.f);
  }
  __syncthreads();
  const int tok = (int)threadIdx.x;
  if (tok < NQ && q0 + tok < f.n) {
    float4 r = stat[tok];
#pragma unroll
    for (int w = 1; w < P::WP; ++w) {
      const float4 o = stat[w * NQ + tok];
      const float m = fmaxf(r.x, o.x), dr = fmaxf((r.x - m) * c, -1e4f), dd = fmaxf((o.x - m) * c, -1e4f);
      const float er = fast_exp2(dr), eo = fast_exp2(dd);
      r.z = er * (r.z + dr * r.y) + eo * (o.z + dd * o.y);
      r.y = er * r.y + eo * o.y;
      r.x = m;
    }
    f.part[at.p * f.panel + q0 + tok] = r;
  }
}

// The same of logits in parts: a wave a token and tile, a lane four of its logits.
__global__ __launch_bounds__(256) void linear_logp_stats_kernel(FwdTiles f, LogitParts z) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tok = (int)(unit / f.tiles_p), tile = (int)(unit - (int64_t)tok * f.tiles_p);
  if (tok >= f.n) return;
  const int v = tile * plan::kTileP + 4 * lane;
  const f32x4 raw = z.at(tok, v);
  const float c = f.a.scale * kLog2e;
  const int64_t y = f.a.logp ? f.a.targets[tok] : -1;
  float a[4], m = kLowest, s = 0.f, u = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = v + i < f.a.vocab ? raw[i] : kNegInf;
    if (v + i == y && y < f.a.vocab) f.at_target[tok] = a[i];
    m = fmaxf(m, a[i]);
  }
  m = wave_max(m);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float d = (a[i] - m) * c, e = fast_exp2(d);
    s += e;
    u = fmaf(e, fmaxf(d, -200.f), u);              // (0 times infinity: 0; a NaN stays one in s)
  }
  s = group_sum<64>(s);
  u = group_sum<64>(u);
  if (lane == 0) f.part[tile * f.panel + tok] = make_float4(m, s, u, 0.f);
}

// The tiles of 16 tokens a workgroup: 64 strands of tiles, joined over the four of a
// wave, then over the waves.
constexpr int kJoinTokens = 16, kJoinStrands = 64;
__global__ __launch_bounds__(kJoinTokens * kJoinStrands) void linear_logp_join_kernel(FwdTiles f) {
  constexpr int kWaves = kJoinTokens * kJoinStrands / 64;
  __shared__ float4 sh[kWaves][kJoinTokens];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mine = lane % kJoinTokens;
  const int tok = (int)blockIdx.x * kJoinTokens + mine, strand = threadIdx.x / kJoinTokens;
  const float c = f.a.scale * kLog2e;
  float m = kLowest, s = 0.f, u = 0.f;
  const auto add = [&](float om, float os, float ou) {
    const float to = fmaxf(m, om), d = fmaxf((m - to) * c, -1e4f), e = fmaxf((om - to) * c, -1e4f);
    const float fd = fast_exp2(d), fe = fast_exp2(e);
    u = fd * (u + d * s) + fe * (ou + e * os);
    s = fd * s + fe * os;
    m = to;
  };
  const auto across = [&](int lanes) {             // (both sides add the same two, the lower lanes' first)
    const float om = __shfl_xor(m, lanes), os = __shfl_xor(s, lanes), ou = __shfl_xor(u, lanes);
    if (lane & lanes) {
      const float tm = m, ts = s, tu = u;
      m = om, s = os, u = ou;
      add(tm, ts, tu);
    } else {
      add(om, os, ou);
    }
  };
  if (tok < f.n) {
    const float4 *part = f.part + tok;
    for (int t = strand; t < f.tiles_p; t += 8 * kJoinStrands) {
      float4 o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = t + i * kJoinStrands < f.tiles_p ? part[(t + i * kJoinStrands) * f.panel] : make_float4(kLowest, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) add(o[i].x, o[i].y, o[i].z);
    }
  }
  across(16);
  across(32);
  if (lane < kJoinTokens) sh[wave][lane] = make_float4(m, s, u, 0.f);
  __syncthreads();
  if (wave != 0) return;
  {
    const float4 o = sh[lane / kJoinTokens * (kWaves / 4)][mine];
    m = o.x, s = o.y, u = o.z;
  }
#pragma unroll
  for (int w = 1; w < kWaves / 4; ++w) {
    const float4 o = sh[lane / kJoinTokens * (kWaves / 4) + w][mine];
    add(o.x, o.y, o.z);
  }
  across(16);
  across(32);
  if (lane >= kJoinTokens || tok >= f.n) return;
  const int64_t t = f.t0 + tok;
  const bool none = s == 0.f;                    // logits of -inf alone
  const float log_s = log2f(s) * kLn2, top = m * f.a.scale;
  float lse = none ? kNegInf : top + log_s;
  const bool lost = !none && !(fabsf(lse) < -kNegInf);
  if (lost) lse = kNan;
  f.a.lse[t] = lse;
  if (f.a.entropy) f.a.entropy[t] = none ? 0.f : lost ? kNan : log_s - u / s * kLn2;
  if (f.a.logp) {
    const int64_t y = f.a.targets[t];
    float r = 0.f;
    if (y >= 0 && y < f.a.vocab) {
      const float z = f.at_target[tok];
      r = none ? kNegInf : lost ? kNan : (z - m) * f.a.scale - log_s;
    }
    f.a.logp[t] = r;
  }
}

// ---------------------------------------------------------------- backward --

struct BwdTiles {
  LinearArgs a;
  plan::LinearBwd f;
  int *count;                  // rows gathered
  int *order;                  // [rows]: their tokens
  int *place;                  // [tokens]: a token's row, -1: it has no gradient
  float4 *coef;                // [rows]: lse, k0, k1, the target's
  int *target;                 // [rows], -1: none
  char *x;                     // gathered rows [copies][rows][f.dim]; second copies follow the last first
  char *dl;                    // [numbers][rows][piece]; copies likewise, second numbers of one copy from `rows` on
  float *sum_x, *sum_w;        // [split][copies][rows][dim], [split][piece][dim]
  __device__ __forceinline__ int rows() const { return rows_of(count, a.n_tokens); }
  __device__ __forceinline__ int64_t token(int r) const { return row_of(order, r, a.n_tokens); }
  int v0, n_v;                 // the piece
  bool first, last;            // of the pieces
  bool sums_x;                 // dx goes by float32 sums
  int tiles_dim;               // tiles of columns
  int grid_x, grid_w;          // workgroups of dx and dw, multiples of kXcdQueues
};

// A token's coefficients; whether it has a gradient.
struct Coefficients {
  bool some = false;
  float lse = 0.f, k0 = 0.f, k1 = 0.f, at = 0.f;
  int y = -1;
  __device__ __forceinline__ Coefficients(const LinearArgs &a, int64_t t) {
    if (t >= a.n_tokens) return;
    const int64_t target = a.g_logp ? a.targets[t] : -1;
    const bool given = target >= 0 && target < a.vocab;
    const float gl = given ? a.g_logp[t] : 0.f, gs = a.g_lse ? a.g_lse[t] : 0.f, ge = a.g_entropy ? a.g_entropy[t] : 0.f;
    lse = a.lse_in[t];
    some = !(lse == kNegInf || (gl == 0.f && gs == 0.f && ge == 0.f));
    k0 = a.scale * (gs - gl - (ge != 0.f ? ge * a.entropy_in[t] : 0.f)) + (lse < -kNegInf ? 0.f : kNan);
    k1 = -a.scale * ge * kLn2;
    at = a.scale * gl;
    y = given ? (int)target : -1;
  }
  __device__ __forceinline__ void store(const BwdTiles &b, int64_t t, int row) const {
    b.place[t] = some ? row : -1;
    if (!some) return;
    b.order[row] = (int)t;
    b.coef[row] = make_float4(lse, k0, k1, at);
    b.target[row] = y;
  }
};

// Threads of a workgroup of 1024 before this one that have `some`; n: of all.
__device__ __forceinline__ int count_before(bool some, int (&sums)[16], int &n) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t in = __ballot(some);
  if (lane == 0) sums[wave] = __popcll(in);
  __syncthreads();
  int before = __popcll(in & ((uint64_t(1) << lane) - 1));
  n = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    before += w < wave ? sums[w] : 0;
    n += sums[w];
  }
  __syncthreads();                               // (sums may be written again)
  return before;
}

// A token's hidden row to its place, and to another where that is not the same; dx of a
// token without one is zero.
__device__ __forceinline__ void gather_row(const BwdTiles &b, int64_t t, int row, int another) {
  const LinearArgs &a = b.a;
  const int lane = threadIdx.x & 63;
  if (row >= 0) {
    const u32x4 *from = (const u32x4 *)(a.x + 2 * t * a.x_stride);
    u32x4 *to = (u32x4 *)(b.x + 2 * (int64_t)row * b.f.dim);
    for (int i = lane; i < a.dim / 8; i += 64) to[i] = from[i];
    if (another == row) return;
    to = (u32x4 *)(b.x + 2 * (int64_t)another * b.f.dim);
    for (int i = lane; i < a.dim / 8; i += 64) to[i] = from[i];
  } else if (a.dx) {
    u32x4 *to = (u32x4 *)(a.dx + (a.g_f32 ? 4 : 2) * t * a.dx_stride);
    for (int i = lane; i < a.dim / (a.g_f32 ? 4 : 8); i += 64) to[i] = u32x4{};
  }
}

// Which tokens have a gradient, in order, and the coefficients of their rows.
__global__ __launch_bounds__(1024) void linear_rows_kernel(BwdTiles b) {
  __shared__ int sums[16];
  int base = 0;
  for (int64_t t0 = 0; t0 < b.a.n_tokens; t0 += 1024) {
    const int64_t t = t0 + threadIdx.x;
    const Coefficients c(b.a, t);
    int n;
    const int before = count_before(c.some, sums, n);
    if (t < b.a.n_tokens) c.store(b, t, base + before);
    base += n;
  }
  if (threadIdx.x == 0) *b.count = base;
}

__global__ __launch_bounds__(256) void linear_gather_kernel(BwdTiles b) {
  const int wave = (int)threadIdx.x >> 6;
  for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < b.a.n_tokens; t += (int64_t)gridDim.x * 4) {
    const int row = (int)min((int64_t)b.place[t], b.a.n_tokens - 1);
    gather_row(b, t, row, row);
  }
}

// Both, of up to kLinearFew tokens: every workgroup finds all places for itself.
__global__ __launch_bounds__(1024) void linear_rows_gather_kernel(BwdTiles b) {
  static_assert(plan::kLinearFew == 1024, "a token a thread");
  __shared__ int sums[16], place[plan::kLinearFew];
  const int64_t t = threadIdx.x;
  const Coefficients c(b.a, t);
  int n;
  const int before = count_before(c.some, sums, n);
  place[t] = c.some ? before : -1;
  if (blockIdx.x == 0) {
    if (t < b.a.n_tokens) c.store(b, t, before);
    if (t == 0) *b.count = n;
  }
  __syncthreads();
  const int wave = (int)threadIdx.x >> 6;
  for (int r = (int)blockIdx.x * 16 + wave; r < b.a.n_tokens; r += (int)gridDim.x * 16) gather_row(b, r, place[r], place[r] + (b.f.copies > 1 ? n : 0));
}

// What rounding to bf16 leaves of x.
__device__ __forceinline__ float left_of(float x) {
  const float r = x - (float)(bf16)x;
  return fabsf(r) < -kNegInf ? r : 0.f;          // (an infinity and a NaN are whole)
}

// dl of a piece.
template <int NQ>
__global__ __launch_bounds__(512, 2) void linear_dl_kernel(BwdTiles b, int tiles_p) {
  typedef typename LogitTile<NQ>::P P;
  static_assert(P::kLds >= 512 * 32 * P::BP, "room for the rows that are stored");
  __shared__ __attribute__((aligned(1024))) char smem[P::kLds];
  const int n = b.rows();
  tile::Place at;
  if (!at.find(blockIdx.x, tiles_p, (n + NQ - 1) / NQ, 1, kGroup)) return;
  P x;
  const int v0 = at.p * P::NP, q0 = at.q * NQ;   // (of the piece)
  const LinearArgs &a = b.a;
  x.run(smem, typename P::LoadP(a.w, a.w_stride, b.v0 + v0, b.v0 + b.n_v, 0, a.dim, x.wave, x.lane),
        typename P::LoadQ(b.x, b.f.dim, q0, n, 0, a.dim, x.wave, x.lane), a.dim);
  const int l32 = x.lane & 31, h = x.lane >> 5;
  const int vw = v0 + x.p0();
#pragma unroll
  for (int q = 0; q < P::BQ; ++q) {
    const int r0 = q0 + x.q0() + 32 * q, r = r0 + l32;
    // (rows from n on are read by nobody)
    const float4 k = r < n ? b.coef[r] : make_float4(0.f, 0.f, 0.f, 0.f);
    const int y = r < n ? b.target[r] - b.v0 - vw : -1;
    const auto each = [&](auto slope) {
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float d = (x.acc[q][p][i] * a.scale - k.x) * kLog2e;
          x.acc[q][p][i] = fast_exp2(fminf(d, 0.f)) * slope(d);
        }
    };
    if (__any(k.z != 0.f)) each([&](float d) { return k.y + k.z * fmaxf(d, -200.f); });
    else each([&](float) { return k.y; });
    if (__any(y >= 0 && y < 32 * P::BP)) {
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) x.acc[q][p][i] += 32 * p + p_of(i, h) == y ? k.w : 0.f;
    }
    // Columns from n_v on: dx's loads take eight at a time, so some of them meet zeros in the
    // place of w's rows, and what their logit of 0 comes to need not be finite.
    if (v0 + P::NP > b.n_v) {
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (vw + 32 * p + p_of(i, h) >= b.n_v) x.acc[q][p][i] = 0.f;
    }
    const auto put = [&](int64_t first, int rows) {
      char *out = b.dl + 2 * (first * b.f.piece + vw);
      put_rows<P::BP, false>(x.acc[q], smem + x.wave * (2048 * P::BP), rows, 32 * P::BP, x.lane,
                             [&](int row, int byte, f32x4 v) { *(f32x4 *)(out + (int64_t)row * 2 * b.f.piece + byte) = v; });
    };
    const bool pairs = NQ <= plan::kLinearTwice && b.f.copies > 1;   // two rows a token
    put(r0, pairs ? n - r0 : 32);
    if (b.f.numbers > 1) {
#pragma unroll
      for (int p = 0; p < P::BP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) x.acc[q][p][i] = left_of(x.acc[q][p][i]);
      put((pairs ? n : b.f.rows) + r0, pairs ? n - r0 : 32);
    }
  }
}

// dl of a piece from logits in parts: eight columns a thread.
__global__ __launch_bounds__(256) void linear_dl_parts_kernel(BwdTiles b, LogitParts z) {
  const int vecs = b.f.piece / 8;
  const int n = b.rows();
  const int64_t all = (int64_t)n * vecs;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / vecs), v = (int)(i - (int64_t)r * vecs) * 8;
    const float4 k = b.coef[r];
    const int y = b.target[r] - v;
    const f32x4 lo = z.at(r, v), hi = z.at(r, v + 4);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = ((e < 4 ? lo[e & 3] : hi[e & 3]) * b.a.scale - k.x) * kLog2e;
      o[e] = fast_exp2(fminf(d, 0.f)) * (k.z != 0.f ? k.y + k.z * fmaxf(d, -200.f) : k.y) + (e == y ? k.w : 0.f);
      if (v + e >= b.n_v) o[e] = 0.f;              // (as above)
    }
    *(u32x4 *)(b.dl + 2 * ((int64_t)r * b.f.piece + v)) = pack<bf16>(o);
    if (b.f.numbers > 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = left_of(o[e]);
      *(u32x4 *)(b.dl + 2 * (((b.f.copies > 1 ? n : b.f.rows) + r) * b.f.piece + v)) = pack<bf16>(o);
    }
  }
}

// Where a product's rows go.
enum Out { kBf16, kF32, kSums };

// Sums of one part: [rows][dim] of its own, added to with a piece after the first.
template <class P, Out OUT, class Row>
__device__ __forceinline__ void put_product(P &x, char *smem, int p0, int q_base, int n_q, int dim, bool add, Row row_of) {
  static_assert(P::kLds >= P::NW * 4096 * P::BP, "room for the rows that are stored");
#pragma unroll
  for (int q = 0; q < P::BQ; ++q) {
    const int r0 = q_base + x.q0() + 32 * q, pw = p0 + x.p0();
    put_rows<P::BP, OUT != kBf16>(x.acc[q], smem + x.wave * (4096 * P::BP), n_q - r0, dim - pw, x.lane, [&](int row, int byte, f32x4 v) {
      char *to = row_of(r0 + row) + (int64_t)pw * (OUT == kBf16 ? 2 : 4) + byte;
      if constexpr (OUT == kSums) {
        if (add) {
          const f32x4 o = *(const f32x4 *)to;
          v += o;
        }
      }
      *(f32x4 *)to = v;
    });
  }
}

// dx of a piece: p: columns, q: gathered rows, k: the piece's vocabulary rows.
template <int NQ>
struct DxTile;
template <>
struct DxTile<256> { typedef Product<kAcross, kAlong, 256, 256, 2, 4> P; };
template <>
struct DxTile<64> { typedef Product<kAcross, kAlong, 256, 64, 4, 2> P; };
// dw: p: columns, q: the piece's vocabulary rows, k: gathered rows.
typedef Product<kAcross, kAcross, 256, 256, 2, 4> DwTile;

// ALONG: times that a product goes over its k's, each time with the next numbers of dl.
template <int NQ, int ALONG>
__device__ __forceinline__ void dx_tile(const BwdTiles &b, int id, char *smem) {
  typedef typename DxTile<NQ>::P P;
  const int n = b.rows() * b.f.copies, dim = b.a.dim;
  tile::Place at;
  if (!at.find(id, b.tiles_dim, (n + NQ - 1) / NQ, b.f.split_x, kGroup)) return;
  P x;
  const int len = (int)plan::round_up(plan::ceil_div(b.f.piece, b.f.split_x), tile::kStep);
  const int k0 = at.part * len, n_k = max(0, min(b.n_v - k0, len));
  const int p0 = at.p * P::NP, q0 = at.q * NQ;
  x.clear();
#pragma unroll
  for (int i = 0; i < ALONG; ++i)
    x.add(smem, typename P::LoadP(b.a.w, b.a.w_stride, p0, dim, b.v0 + k0, n_k, x.wave, x.lane),
          typename P::LoadQ(b.dl + i * (2 * b.f.rows * b.f.piece), b.f.piece, q0, n, k0, n_k, x.wave, x.lane), n_k);
  const auto row = [&](int es) { return [=, &b](int r) { return b.a.dx + b.token(r) * b.a.dx_stride * es; }; };
  if (b.sums_x) {
    float *sums = b.sum_x + (int64_t)at.part * b.f.copies * b.f.rows * dim;
    put_product<P, kSums>(x, smem, p0, q0, n, dim, !b.first, [&](int r) { return (char *)(sums + (int64_t)r * dim); });
  } else if (b.a.g_f32) {
    put_product<P, kF32>(x, smem, p0, q0, n, dim, false, row(4));
  } else {
    put_product<P, kBf16>(x, smem, p0, q0, n, dim, false, row(2));
  }
}

template <int ALONG>
__device__ __forceinline__ void dw_tile(const BwdTiles &b, int id, char *smem) {
  typedef DwTile P;
  const int dim = b.a.dim;
  tile::Place at;
  if (!at.find(id, b.tiles_dim, (int)plan::ceil_div(b.n_v, P::NQ), b.f.split_w, kGroup)) return;
  P x;
  const int n = b.rows() * b.f.copies;
  const int len = (int)plan::round_up(plan::ceil_div(n, b.f.split_w), tile::kStep);
  const int k0 = at.part * len, n_k = max(0, min(n - k0, len));
  const int p0 = at.p * P::NP, q0 = at.q * P::NQ;
  x.clear();
#pragma unroll
  for (int i = 0; i < ALONG; ++i)
    x.add(smem, P::LoadP(b.x, b.f.dim, p0, dim, k0, n_k, x.wave, x.lane),
          P::LoadQ(b.dl + i * (2 * b.f.rows * b.f.piece), b.f.piece, q0, b.n_v, k0, n_k, x.wave, x.lane), n_k);
  const auto row = [&](int es) { return [=, &b](int r) { return b.a.dw + (int64_t)(b.v0 + r) * b.a.dw_stride * es; }; };
  if (b.f.split_w > 1) {
    float *sums = b.sum_w + (int64_t)at.part * b.f.piece * dim;
    put_product<P, kSums>(x, smem, p0, q0, b.n_v, dim, false, [&](int r) { return (char *)(sums + (int64_t)r * dim); });
  } else if (b.a.g_f32) {
    put_product<P, kF32>(x, smem, p0, q0, b.n_v, dim, false, row(4));
  } else {
    put_product<P, kBf16>(x, smem, p0, q0, b.n_v, dim, false, row(2));
  }
}

// dx's tiles, then dw's, of a piece.
template <int NQ, int ALONG>
__global__ __launch_bounds__(512, 2) void linear_grads_kernel(BwdTiles b) {
  constexpr int kX = DxTile<NQ>::P::kLds;
  __shared__ __attribute__((aligned(1024))) char smem[kX > DwTile::kLds ? kX : DwTile::kLds];
  const int id = (int)blockIdx.x;
  if (id < b.grid_x) dx_tile<NQ, ALONG>(b, id, smem);
  else dw_tile<ALONG>(b, id - b.grid_x, smem);
}

// The parts' sums, in order, as rows of the gradient.
template <bool F32, bool DX>
__global__ __launch_bounds__(256) void linear_sums_kernel(BwdTiles b) {
  const int rows = DX ? b.rows() : b.n_v, dim = b.a.dim, parts = DX ? b.f.split_x : b.f.split_w, copies = DX ? b.f.copies : 1;
  const int64_t per = (DX ? (int64_t)b.f.copies * b.f.rows : (int64_t)b.f.piece) * dim;
  const float *sums = DX ? b.sum_x : b.sum_w;
  const int vecs = dim / 4;
  const int64_t n = (int64_t)rows * vecs;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / vecs), c = (int)(i - (int64_t)r * vecs) * 4;
    f32x4 sum = {};
    for (int k = 0; k < copies; ++k) {
      const float *from = sums + ((int64_t)k * rows + r) * dim + c;
      for (int p0 = 0; p0 < parts; p0 += 8) {
        f32x4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = p0 + j < parts ? *(const f32x4 *)(from + (p0 + j) * per) : f32x4{};
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[j];
      }
    }
    char *row = DX ? b.a.dx + b.token(r) * b.a.dx_stride * (F32 ? 4 : 2) : b.a.dw + (int64_t)(b.v0 + r) * b.a.dw_stride * (F32 ? 4 : 2);
    if constexpr (F32) *(f32x4 *)(row + 4 * c) = sum;
    else *(uint2 *)(row + 2 * c) = make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
  }
}

// dw of no tokens.
__global__ __launch_bounds__(256) void linear_zero_kernel(char *dw, int64_t row_bytes, int vecs, int vocab) {
  for (int v = (int)blockIdx.x; v < vocab; v += (int)gridDim.x)
    for (int i = (int)threadIdx.x; i < vecs; i += 256) *(u32x4 *)(dw + v * row_bytes + 16 * i) = u32x4{};
}

template <int NQ>
hipError_t fwd_tiles(const FwdTiles &f, hipStream_t s) {
  linear_logp_tiles_kernel<NQ><<<grid_of((int64_t)f.tiles_p * f.tiles_q), 512, 0, s>>>(f);
  return hipGetLastError();
}

template <int NQ>
hipError_t dl_tiles(const BwdTiles &b, hipStream_t s) {
  const int tiles_p = (int)plan::ceil_div(b.n_v, plan::kTileP);
  linear_dl_kernel<NQ><<<grid_of(tiles_p * (b.f.rows / NQ)), 512, 0, s>>>(b, tiles_p);
  return hipGetLastError();
}

template <int NQ, int ALONG>
hipError_t launch_grads(const BwdTiles &b, hipStream_t s) {
  const int grid = b.grid_x + b.grid_w;
  if (grid > 0) linear_grads_kernel<NQ, ALONG><<<grid, 512, 0, s>>>(b);
  return hipGetLastError();
}

// In one launch, where dx alone would leave compute units idle.  (100 x 704 x 12000: 33
// us apart, 20 together; where both fill them the two together are 1% slower.)
template <int NQ, int ALONG>
hipError_t grads(BwdTiles b, hipStream_t s) {
  b.grid_x = b.a.dx ? grid_of(b.tiles_dim * plan::ceil_div(b.f.copies * b.f.rows, NQ) * b.f.split_x) : 0;
  b.grid_w = b.a.dw ? grid_of(b.tiles_dim * plan::ceil_div(b.n_v, DwTile::NQ) * b.f.split_w) : 0;
  if (b.grid_x <= plan::kUnits || b.grid_w == 0) return launch_grads<NQ, ALONG>(b, s);
  BwdTiles w = b;
  w.grid_x = b.grid_w = 0;
  const hipError_t e = launch_grads<NQ, ALONG>(w, s);
  return e == hipSuccess ? launch_grads<NQ, ALONG>(b, s) : e;
}

template <bool DX>
hipError_t join_sums(const BwdTiles &b, hipStream_t s) {
  const int64_t vecs = (DX ? b.f.rows : (int64_t)b.n_v) * (b.a.dim / 4);
  const int64_t want = plan::ceil_div(vecs, 256);
  const int grid = (int)(want < 8192 ? want : 8192);
  if (b.a.g_f32) linear_sums_kernel<true, DX><<<grid, 256, 0, s>>>(b);
  else linear_sums_kernel<false, DX><<<grid, 256, 0, s>>>(b);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_logp_fwd(const LinearArgs &a, hipStream_t s) {
  const plan::LinearFwd p = plan::linear_fwd(a.n_tokens, a.dim, a.vocab);
  FwdTiles f{};
  f.a = a;
  f.panel = p.panel;
  f.tiles_p = (int)p.tiles_p;
  f.part = (float4 *)(a.ws + p.part_off);
  f.at_target = (float *)(a.ws + p.target_off);
  for (int64_t t0 = 0; t0 < a.n_tokens; t0 += p.panel) {
    f.t0 = t0;
    f.n = (int)(a.n_tokens - t0 < p.panel ? a.n_tokens - t0 : p.panel);
    f.tiles_q = (int)plan::ceil_div(f.n, p.tile);
    hipError_t e;
    if (p.split > 1) {
      const LogitParts z = {a.w, a.x, a.w_stride, a.x_stride, nullptr, f.n, a.vocab, a.dim, p.split, f.tiles_p, p.panel,
                            p.tiles_p * plan::kTileP, (float *)(a.ws + p.z_off)};
      e = logit_parts(z, p.tile, s);
      if (e != hipSuccess) return e;
      linear_logp_stats_kernel<<<(int)plan::ceil_div(f.n * p.tiles_p, 4), 256, 0, s>>>(f, z);
      e = hipGetLastError();
    } else {
      e = p.tile == 32 ? fwd_tiles<32>(f, s) : p.tile == 64 ? fwd_tiles<64>(f, s) : p.tile == 128 ? fwd_tiles<128>(f, s) : fwd_tiles<256>(f, s);
    }
    if (e != hipSuccess) return e;
    linear_logp_join_kernel<<<(f.n + kJoinTokens - 1) / kJoinTokens, kJoinTokens * kJoinStrands, 0, s>>>(f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_linear_logp_bwd(const LinearArgs &a, hipStream_t s) {
  if (a.n_tokens == 0) {
    if (!a.dw) return hipSuccess;
    const int es = a.g_f32 ? 4 : 2;
    linear_zero_kernel<<<a.vocab < 65536 ? a.vocab : 65536, 256, 0, s>>>(a.dw, a.dw_stride * es, a.dim * es / 16, a.vocab);
    return hipGetLastError();
  }
  BwdTiles b{};
  b.a = a;
  b.f = plan::linear_bwd_call(a.n_tokens, a.dim, a.vocab, a.g_f32, a.dx != nullptr, a.dw != nullptr);
  const int along = b.f.numbers / b.f.copies;    // (more than 1: one copy, tiles of 256 tokens of dx)
  b.count = (int *)(a.ws + b.f.count_off);
  b.order = (int *)(a.ws + b.f.order_off);
  b.place = (int *)(a.ws + b.f.place_off);
  b.coef = (float4 *)(a.ws + b.f.coef_off);
  b.target = (int *)(a.ws + b.f.target_off);
  b.x = a.ws + b.f.x_off;
  b.dl = a.ws + b.f.dl_off;
  b.sum_x = (float *)(a.ws + b.f.sum_x_off);
  b.sum_w = (float *)(a.ws + b.f.sum_w_off);
  hipError_t e;
  if (a.n_tokens <= plan::kLinearFew) {
    const int64_t groups = plan::ceil_div(a.n_tokens, 16);
    linear_rows_gather_kernel<<<(int)groups, 1024, 0, s>>>(b);
    e = hipGetLastError();
  } else {
    linear_rows_kernel<<<1, 1024, 0, s>>>(b);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t groups = plan::ceil_div(a.n_tokens, 4);
    linear_gather_kernel<<<(int)(groups < 65536 ? groups : 65536), 256, 0, s>>>(b);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  b.tiles_dim = (int)plan::ceil_div(a.dim, plan::kTileP);
  b.sums_x = b.f.pieces > 1 || b.f.split_x > 1 || b.f.copies > 1;
  for (int p = 0; p < b.f.pieces; ++p) {
    b.v0 = p * b.f.piece;
    b.n_v = a.vocab - b.v0 < b.f.piece ? a.vocab - b.v0 : b.f.piece;
    b.first = p == 0;
    b.last = p == b.f.pieces - 1;
    if (b.f.split_z > 1) {
      const LogitParts z = {a.w, b.x, a.w_stride, b.f.dim, b.count, (int)a.n_tokens, a.vocab, a.dim, b.f.split_z, b.f.piece / plan::kTileP, b.f.rows,
                            b.f.piece, (float *)(a.ws + b.f.z_off)};
      e = logit_parts(z, b.f.tile, s);
      if (e != hipSuccess) return e;
      const int64_t want = plan::ceil_div(b.f.rows * (b.f.piece / 8), 256);
      linear_dl_parts_kernel<<<(int)(want < 8192 ? want : 8192), 256, 0, s>>>(b, z);
      e = hipGetLastError();
    } else {
      e = b.f.tile == 32 ? dl_tiles<32>(b, s) : b.f.tile == 64 ? dl_tiles<64>(b, s) : b.f.tile == 128 ? dl_tiles<128>(b, s) : dl_tiles<256>(b, s);
    }
    if (e == hipSuccess) e = along > 1 ? grads<256, 2>(b, s) : b.f.tile_x == 64 ? grads<64, 1>(b, s) : grads<256, 1>(b, s);
    if (e == hipSuccess && a.dw && b.f.split_w > 1) e = join_sums<false>(b, s);
    if (e == hipSuccess && a.dx && b.last && b.sums_x) e = join_sums<true>(b, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace nsp
