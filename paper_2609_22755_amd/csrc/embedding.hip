// Rows of an embedding table, and its gradient, for gfx950.
//
//     y_t = scale w[i_t],     dw_v = scale sum over t with i_t = v of dy_t
//
// Bound by HBM: the forward reads a row and writes one a token, the backward reads
// one a token and writes every row of the table.  262144 x 4096 bf16 of 131072 rows:
// 536 us (4.8 TB/s; a copy reaches 4.9), its gradient 687 (4.7).
//
// Backward, of few tokens: zeros everywhere, then a kernel whose workgroups find the
// tokens of an id among all.  Of more: the tokens are sorted by their ids, stably
// (counting sort, digit by digit), so that a row's tokens lie side by side in their
// order and every sum has a fixed order, without an atomic on data.  A wave takes a chunk of the sorted list
// and a strip of columns, adds rows as long as the id stays the same and stores each
// id's sum: to the table, or, where the id goes on beyond the chunk, in float32 for
// a second kernel that adds the chunks' sums in order.
//
// The sort keeps few compute units busy and no memory; the rows of ids that no token
// has are zeroed beside its last launch: up to 16384 tokens, which one workgroup
// sorts in LDS, all rows (at most as many again are written), of more those that
// the first pass left without a flag.
#include "row_common.hpp"
#include "vocab_internal.hpp"

namespace nsp {
namespace {

// Half a vector of bf16.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store_half(bf16 *p, const float (&x)[4]) {
  const u32x2_any both = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  __builtin_nontemporal_store(both, (u32x2_any *)p);
}
// N elements (8 to 32 bytes), or the first cnt of them.
template <class T, int N>
__device__ __forceinline__ void store_n(T *p, int cnt, const float (&x)[N]) {
  if (cnt >= N) {
    if constexpr (N < kVec<T>) store_half(p, x);
#pragma unroll
    for (int i = 0; i < N / kVec<T>; ++i) {
      float v[kVec<T>];
#pragma unroll
      for (int e = 0; e < kVec<T>; ++e) v[e] = x[i * kVec<T> + e];
      store16(p + i * kVec<T>, pack<T>(v));
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < cnt) p[e] = (T)x[e];
  }
}

// ----------------------------------------------------------------- forward --

// Vectors of a lane.  A wave takes a strip of so many times 64 of a row, or, of rows
// of at most 64, as many rows as it has lanes for, so many times.
constexpr int kFwdVecs = 4;

template <class W, class Y>
constexpr int kPair = kVec<W> < kVec<Y> ? kVec<W> : kVec<Y>;   // elements of a lane's vector

template <class W, int N>
__device__ __forceinline__ void load_pair(const W *p, bool some, float (&x)[N]) {
  if constexpr (N == kVec<W>) {
    u32x4 raw = {};
    if (some) raw = *(const u32x4_any *)p;
    unpack<W>(raw, x);
  } else {                             // half a vector of bf16
    u32x2_any raw = {};
    if (some) raw = *(const u32x2_any *)p;
    const u32x4 both = {raw[0], raw[1], 0, 0};
    float v8[kVec<W>];
    unpack<W>(both, v8);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = v8[e];
  }
}
template <class Y, int N>
__device__ __forceinline__ void store_pair(Y *p, float scale, float (&x)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] *= scale;
  if constexpr (N == kVec<Y>) store16(p, pack<Y>(x));
  else store_half(p, x);
}

template <class W, class Y>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(EmbedArgs a, int strips) {
  constexpr int N = kPair<W, Y>;
  const int lane = threadIdx.x & 63;
  const int64_t units = (int64_t)a.n_tokens * strips;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int t = (int)(unit / strips), strip = (int)(unit - (int64_t)t * strips);
    const int64_t v = a.tokens[t];
    const bool some = v >= 0 && v < a.vocab;
    const W *w = (const W *)a.w.data + (some ? v : 0) * a.w.ts;
    Y *y = (Y *)a.y.data + t * a.y.ts;
    const int c0 = (strip * kFwdVecs * 64 + lane) * N;
    // the last vector of a row reaches back over its neighbour's elements
    const auto at = [&](int i) { return min(c0 + i * 64 * N, a.dim - N); };
    float x[kFwdVecs][N];
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) load_pair<W, N>(w + at(i), some && c0 + i * 64 * N < a.dim, x[i]);
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i)
      if (c0 + i * 64 * N < a.dim) store_pair<Y, N>(y + at(i), a.scale, x[i]);
  }
}

// Rows of at most 64 vectors, 1 << bits lanes each.
template <class W, class Y>
__global__ __launch_bounds__(256) void embedding_narrow_kernel(EmbedArgs a, int bits) {
  constexpr int N = kPair<W, Y>;
  const int lane = threadIdx.x & 63, per = 64 >> bits;   // rows of a wave at a time
  const int c0 = (lane & ((1 << bits) - 1)) * N;
  const bool there = c0 < a.dim;
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0;
  const int64_t t0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (per * kFwdVecs) + (lane >> bits);
  int64_t v[kFwdVecs];
#pragma unroll
  for (int i = 0; i < kFwdVecs; ++i) {
    const int64_t t = t0 + i * per;
    v[i] = t < a.n_tokens ? a.tokens[t] : -1;
    if (v[i] >= a.vocab) v[i] = -1;
  }
  if (a.dim >= N) {
    float x[kFwdVecs][N];
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) load_pair<W, N>((const W *)a.w.data + (v[i] >= 0 ? v[i] : 0) * a.w.ts + col, v[i] >= 0 && there, x[i]);
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i)
      if (t0 + i * per < a.n_tokens && there) store_pair<Y, N>((Y *)a.y.data + (t0 + i * per) * a.y.ts + col, a.scale, x[i]);
  } else if (there) {                  // less than a vector: a lane a row
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) {
      if (t0 + i * per >= a.n_tokens) continue;
      Y *y = (Y *)a.y.data + (t0 + i * per) * a.y.ts;
      const W *w = (const W *)a.w.data + (v[i] >= 0 ? v[i] : 0) * a.w.ts;
      for (int e = 0; e < a.dim; ++e) y[e] = (Y)(v[i] >= 0 ? to_f32(w[e]) * a.scale : 0.f);
    }
  }
}

// -------------------------------------------------------------------- sort --

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kRounds = plan::kSortBlock / kSortThreads, kWholeRounds = plan::kSortWhole / kSortThreads;
constexpr int kMaxBins = 1 << plan::kSortBits;

struct SortArgs {
  const int64_t *tokens;       // the first pass reads these
  const uint32_t *key_in, *token_in;
  uint32_t *key_out, *token_out, *hist;   // hist: [block][digit], after them the sums
  uint8_t *flags;              // ids that some token has; null: any may have one
  int32_t n_tokens, vocab, blocks, passes, shift, bits;
  bool first;                  // pass
  bool added;                  // hist holds sums over the blocks before
  char *dw;                    // rows to be zeroed by the workgroups past the blocks
  int64_t row_bytes;
  int32_t row_elems, elem_bytes;
  int32_t groups;              // of zero_rows
};

__device__ __forceinline__ uint32_t key_of(int64_t token, int vocab) { return token >= 0 && token < vocab ? (uint32_t)token : (uint32_t)vocab; }

// Rows without a token, by one of the workgroups that a sort's last launch has for
// them: 64 neighbours a workgroup, as many lanes a row as it has vectors, so that
// the chip writes in the order of the addresses (131072 rows of 8 KB: 6.3 TB/s, with
// resident workgroups that step over the table 5.1; a fill of the same 6.8).  Rows
// that lie side by side and are all zeroed go as one, 256 KB a workgroup: beside the
// sort's LDS few workgroups are resident (50021 x 1111 float32 56 us in all, by 16 KB 76).
constexpr int kZeroRows = 64;
constexpr int64_t kZeroBytes = 256 << 10;
constexpr int kZeroGrid = 1 << 20;               // (a launch holds less than 2^32 threads)

// Zeros by THREADS threads, whole lines of 128 bytes.
template <int THREADS>
__device__ __forceinline__ void zero_bytes(char *p, int64_t bytes) {
  const int64_t lead = min(bytes, (int64_t)(-(intptr_t)p & 127)), vecs = (bytes - lead) / 16, tail = lead + 16 * vecs;
  for (int64_t i = threadIdx.x; i < vecs; i += THREADS) *(u32x4 *)(p + lead + 16 * i) = u32x4{};
  const int c = 2 * (int)threadIdx.x;
  if (c < lead) *(uint16_t *)(p + c) = 0;
  if (tail + c < bytes) *(uint16_t *)(p + tail + c) = 0;
}
// A row by `lanes` of them.
__device__ __forceinline__ void zero_row(char *w, int64_t bytes, int at, int lanes) {
  if (bytes >= 16) {                             // the last vector reaches back
    for (int64_t c = 16 * at; c < bytes; c += 16 * lanes) *(u32x4_any *)(w + min(c, bytes - 16)) = u32x4{};
  } else {
    for (int64_t c = 2 * at; c < bytes; c += 2 * lanes) *(uint16_t *)(w + c) = 0;
  }
}

__device__ __forceinline__ void zero_group(const SortArgs &a, int64_t group) {
  const int64_t bytes = (int64_t)a.row_elems * a.elem_bytes;
  if (!a.flags && a.row_bytes == bytes) {
    // (cut at lines)
    const int64_t all = a.vocab * bytes, skew = (intptr_t)a.dw & 127;
    const int64_t lo = max(group * kZeroBytes - skew, (int64_t)0), hi = min(all, (group + 1) * kZeroBytes - skew);
    if (lo < hi) zero_bytes<kSortThreads>(a.dw + lo, hi - lo);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t v0 = group * kZeroRows;
  uint64_t rows = __ballot(v0 + lane < a.vocab && !(a.flags && a.flags[v0 + lane]));
  int lanes = 64;
  while (lanes < kSortThreads && 16 * lanes < bytes) lanes *= 2;
  const int side = (int)threadIdx.x / lanes, sides = kSortThreads / lanes, at = (int)threadIdx.x % lanes;
  for (int i = 0; rows; ++i, rows &= rows - 1) {
    if (i % sides != side) continue;
    zero_row(a.dw + (v0 + __builtin_ctzll(rows)) * a.row_bytes, bytes, at, lanes);
  }
}

// By workgroup `first` of `n`.
__device__ __forceinline__ void zero_rows(const SortArgs &a, int first, int n) {
  for (int g = first; g < a.groups; g += n) zero_group(a, g);
}

// How many of a block's keys have each digit.
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(SortArgs a) {
  __shared__ int bins[kMaxBins];
  const int n_bins = 1 << a.bits;
  for (int i = threadIdx.x; i < n_bins; i += kSortThreads) bins[i] = 0;
  if (a.first) {
    u32x4 *f = (u32x4 *)a.flags;                 // (whole 256 bytes)
    for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < (a.vocab + 15) / 16; i += gridDim.x * kSortThreads) f[i] = u32x4{};
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int i = blockIdx.x * plan::kSortBlock + r * kSortThreads + threadIdx.x;
    if (i < a.n_tokens) {
      const uint32_t k = a.first ? key_of(a.tokens[i], a.vocab) : a.key_in[i];
      atomicAdd(&bins[(k >> a.shift) & (n_bins - 1)], 1);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_bins; i += kSortThreads) a.hist[((int64_t)blockIdx.x << a.bits) + i] = bins[i];
}

// Each digit's counts to sums over the blocks before; a thread a digit.
__global__ __launch_bounds__(64) void embedding_add_kernel(SortArgs a) {
  const int bin = (int)blockIdx.x * 64 + (int)threadIdx.x;
  if (bin >= 1 << a.bits) return;
  uint32_t sum = 0;
  uint32_t *at = a.hist + bin;
  for (int b0 = 0; b0 < a.blocks; b0 += 32) {
    uint32_t c[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) c[i] = b0 + i < a.blocks ? at[(int64_t)(b0 + i) << a.bits] : 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (b0 + i < a.blocks) at[(int64_t)(b0 + i) << a.bits] = sum;
      sum += c[i];
    }
  }
  at[(int64_t)a.blocks << a.bits] = sum;
}

// The sum of the values of the threads before this one.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t up = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(up, d);
    up += lane >= d ? o : 0;
  }
  if (lane == 63) sh[wave] = up;
  __syncthreads();
  uint32_t before = up - x;
  for (int w = 0; w < kSortWaves; ++w) before += w < wave ? sh[w] : 0;
  __syncthreads();                               // (sh may be written again)
  return before;
}

// Lanes whose digit is this lane's.
__device__ __forceinline__ uint64_t alike(uint32_t digit, int bits, bool there) {
  uint64_t m = __ballot(there);
  for (int b = 0; b < bits; ++b) {
    const uint64_t one = __ballot(digit >> b & 1);
    m &= digit >> b & 1 ? one : ~one;
  }
  return m;
}

// A wave's keys (in order, round by round), their ranks among the wave's keys of
// the same digit, and the wave's counts of each digit.
template <int R>
struct Ranks {
  uint32_t key[R], token[R], rank[R];

  template <class C, class Key>
  __device__ __forceinline__ void take(C *counts, int n, int first, int shift, int bits, Key key_at) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = first + 64 * r + lane;
      key[r] = 0;
      token[r] = 0;
      if (i < n) key_at(i, key[r], token[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool there = first + 64 * r + lane < n;
      rank[r] = 0;
      if (first + 64 * r >= n) continue;         // (whole waves)
      const uint32_t d = (key[r] >> shift) & ((1u << bits) - 1);
      const uint64_t m = alike(d, bits, there);
      const uint32_t have = there ? counts[d] : 0;
      rank[r] = have + __popcll(m & ((uint64_t(1) << lane) - 1));
      if (there && (m >> lane) == 1) counts[d] = (C)(have + __popcll(m));   // the last of them
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// The keys of a block to their places by one digit.
__global__ __launch_bounds__(kSortThreads) void embedding_move_kernel(SortArgs a) {
  __shared__ uint32_t counts[kSortWaves][kMaxBins];
  __shared__ uint32_t sums[2][kMaxBins], sh[kSortWaves];
  if ((int)blockIdx.x >= a.blocks) {
    zero_rows(a, (int)blockIdx.x - a.blocks, (int)gridDim.x - a.blocks);
    return;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n_bins = 1 << a.bits;
  for (int i = threadIdx.x; i < kSortWaves * n_bins; i += kSortThreads) counts[i >> a.bits][i & (n_bins - 1)] = 0;
  __syncthreads();
  const int first = blockIdx.x * plan::kSortBlock + wave * (64 * kRounds);
  Ranks<kRounds> x;
  x.take(counts[wave], a.n_tokens, first, a.shift, a.bits, [&](int i, uint32_t &k, uint32_t &t) {
    if (a.first) {
      k = key_of(a.tokens[i], a.vocab);
      t = (uint32_t)i;
      if (k < (uint32_t)a.vocab) a.flags[k] = 1;   // (the same byte from every token of an id)
    } else {
      k = a.key_in[i];
      t = a.token_in[i];
    }
  });
  // Of each digit: the keys of the blocks before this one, and of all (half the
  // threads each a half of the blocks).
  static_assert(kSortThreads == 2 * kMaxBins, "two threads a digit");
  const int bin = threadIdx.x % kMaxBins, half = threadIdx.x / kMaxBins;
  uint32_t before = 0, all = 0;
  if (a.added) {
    if (!half && bin < n_bins) {
      before = a.hist[((int64_t)blockIdx.x << a.bits) + bin];
      all = a.hist[((int64_t)a.blocks << a.bits) + bin];
    }
  } else if (bin < n_bins) {
    const int lo = half ? a.blocks / 2 : 0, hi = half ? a.blocks : a.blocks / 2;
    for (int b0 = lo; b0 < hi; b0 += 16) {
      uint32_t c[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = b0 + i < hi ? a.hist[((int64_t)(b0 + i) << a.bits) + bin] : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        before += b0 + i < (int)blockIdx.x ? c[i] : 0;
        all += c[i];
      }
    }
  }
  if (half) sums[0][bin] = before, sums[1][bin] = all;
  __syncthreads();
  if (!half) before += sums[0][bin], all += sums[1][bin];
  uint32_t at = sum_before(half ? 0 : all, sh) + before;
  if (!half && bin < n_bins)
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = counts[w][bin];
      counts[w][bin] = at;
      at += c;
    }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (first + 64 * r + lane >= a.n_tokens) continue;
    const uint32_t to = counts[wave][(x.key[r] >> a.shift) & (n_bins - 1)] + x.rank[r];
    if (to >= (uint32_t)a.n_tokens) continue;    // (only where something else writes the workspace meanwhile)
    a.key_out[to] = x.key[r];
    a.token_out[to] = x.token[r];
  }
}

// All passes by the first workgroup, in LDS.
template <int R>
__global__ __launch_bounds__(kSortThreads) void embedding_sort_kernel(SortArgs a) {
  __shared__ uint32_t keys[R * kSortThreads], places[R * kSortThreads], sh[kSortWaves];
  __shared__ uint16_t counts[kSortWaves][kMaxBins];
  if (blockIdx.x > 0) {
    zero_rows(a, (int)blockIdx.x - 1, (int)gridDim.x - 1);
    return;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n_bins = 1 << a.bits;
  // as many rounds a wave as the tokens need
  const int rounds = (a.n_tokens + kSortThreads - 1) / kSortThreads, first = wave * (64 * rounds);
  const int n = min(a.n_tokens, first + 64 * rounds);
  for (int p = 0; p < a.passes; ++p) {
    const int shift = p * a.bits;
    for (int i = threadIdx.x; i < kSortWaves * n_bins; i += kSortThreads) counts[i >> a.bits][i & (n_bins - 1)] = 0;
    __syncthreads();
    Ranks<R> x;
    x.take(counts[wave], n, first, shift, a.bits, [&](int i, uint32_t &k, uint32_t &t) {
      k = p == 0 ? key_of(a.tokens[i], a.vocab) : keys[i];
      t = p == 0 ? (uint32_t)i : places[i];
    });
    __syncthreads();
    const int bin = threadIdx.x;
    uint32_t sum = 0;
    if (bin < n_bins)
      for (int w = 0; w < kSortWaves; ++w) sum += counts[w][bin];
    uint32_t at = sum_before(sum, sh);
    if (bin < n_bins)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = counts[w][bin];
        counts[w][bin] = (uint16_t)at;           // (below 16384: the last, past all, is not read)
        at += c;
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (first + 64 * r + lane >= n) continue;
      const uint32_t to = counts[wave][(x.key[r] >> shift) & (n_bins - 1)] + x.rank[r];
      if (p == a.passes - 1) {
        a.key_out[to] = x.key[r];
        a.token_out[to] = x.token[r];
      } else {
        keys[to] = x.key[r];
        places[to] = x.token[r];
      }
    }
    __syncthreads();
  }
}

// Rows alone.
__global__ __launch_bounds__(kSortThreads) void embedding_zero_kernel(SortArgs a) { zero_rows(a, (int)blockIdx.x, (int)gridDim.x); }

// ---------------------------------------------------------------- backward --

struct SumArgs {
  EmbedArgs a;
  const uint32_t *key, *token;  // sorted
  float *part;                  // [chunk][head, tail][dim]
  int strips;                   // of columns
};

constexpr int kAhead = 8;       // rows of a wave in flight

// Float32 sums of a lane's columns, kept between the kernels.
template <int N>
__device__ __forceinline__ void keep(float *to, int cnt, const float (&x)[N]) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  if (cnt >= N) {
#pragma unroll
    for (int e = 0; e < N; e += 4) *(f32x4_any *)(to + e) = f32x4_any{x[e], x[e + 1], x[e + 2], x[e + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < cnt) to[e] = x[e];
  }
}
template <int N>
__device__ __forceinline__ void kept(const float *from, int cnt, float (&x)[N]) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  if (cnt >= N) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const f32x4_any v = *(const f32x4_any *)(from + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[e + i] = v[i];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = e < cnt ? from[e] : 0.f;
  }
}

// A chunk's sums of a strip, by a wave; NARROW: of rows of at most 32 vectors, by
// 1 << bits lanes.  EARLY: the next rows are on their way while these are added: for
// few waves (5003 x 1111 float32 44 us instead of 50); many of them get in each
// other's way in memory (262144 x 4096 850 us instead of 680).
template <class W, class Y, bool NARROW, bool EARLY>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs s, int bits) {
  constexpr int N = kVec<Y>;
  const EmbedArgs &a = s.a;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int chunk, c0;
  if constexpr (NARROW) {
    const int64_t at = (unit << (6 - bits)) + (lane >> bits);
    if (at >= a.f.chunks) return;
    chunk = (int)at;
    c0 = (lane & ((1 << bits) - 1)) * N;
  } else {
    chunk = (int)(unit / s.strips);
    if (chunk >= a.f.chunks) return;
    c0 = ((int)(unit - (int64_t)chunk * s.strips) * 64 + lane) * N;
  }
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0, cnt = a.dim >= N ? N : a.dim;
  const bool there = c0 < a.dim;
  const int lo = chunk * a.f.chunk, hi = min(lo + a.f.chunk, a.n_tokens);
  const Y *dy = (const Y *)a.y.data + col;
  // (a row of dy also where something else writes the workspace meanwhile)
  const auto row_at = [&](int at) { return dy + (int64_t)min(s.token[at], (uint32_t)a.n_tokens - 1) * a.y.ts; };
  float acc[N] = {};
  uint32_t id = s.key[lo];
  bool open = lo > 0 && s.key[lo - 1] == id;       // the id's rows began before the chunk
  const auto end = [&](bool goes_on) {
    if (id < (uint32_t)a.vocab && there) {
      if (open || goes_on) {
        // (of a chunk that lies within one id's rows only the head is used)
        keep(s.part + ((int64_t)chunk * 2 + (open ? 0 : 1)) * a.dim + col, cnt, acc);
      } else {
        float o[N];
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = acc[e] * a.scale;
        store_n<W>((W *)a.w.data + (int64_t)id * a.w.ts + col, cnt, o);
      }
    }
    open = false;
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
  };
  u32x4 raw[kAhead];
  uint32_t ids[kAhead];
  const auto fetch = [&](int p) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int at = min(p + i, hi - 1);
      ids[i] = s.key[at];
      raw[i] = u32x4{};
      if (a.dim >= N && there && p + i < hi && ids[i] < (uint32_t)a.vocab) raw[i] = load16(row_at(at));
    }
  };
  fetch(lo);
  for (int p = lo; p < hi; p += kAhead) {
    u32x4 now[kAhead];
    uint32_t now_id[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) now[i] = raw[i], now_id[i] = ids[i];
    if (EARLY && p + kAhead < hi) fetch(p + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p + i >= hi) break;
      if (now_id[i] != id) {
        end(false);
        id = now_id[i];
      }
      float v[N];
      if (a.dim >= N) unpack<Y>(now[i], v);
      else load_some(row_at(p + i), there && id < (uint32_t)a.vocab ? cnt : 0, 0.f, v);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += v[e];
    }
    if (!EARLY && p + kAhead < hi) fetch(p + kAhead);
  }
  end(hi < a.n_tokens && s.key[hi] == id);
}

// The rows of an id that goes over several chunks: a wave a strip and chunk that one
// begins in.
constexpr int kJoinWaves = 8, kJoinAhead = 8;
template <class W, class Y>
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_join_kernel(SumArgs s) {
  constexpr int N = kVec<Y>;
  const EmbedArgs &a = s.a;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kJoinWaves + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = (int)(unit / s.strips), strip = (int)(unit - (int64_t)chunk * s.strips);
  if (chunk >= a.f.chunks - 1) return;
  const int lo = chunk * a.f.chunk, hi = lo + a.f.chunk;
  const uint32_t id = s.key[hi - 1];
  if (id >= (uint32_t)a.vocab || s.key[hi] != id) return;
  if (s.key[lo] == id && lo > 0 && s.key[lo - 1] == id) return;   // it began before
  // the chunks after this one that begin with the id
  int more = 0;
  for (bool all = true; all;) {
    const int64_t at = (int64_t)(chunk + 1 + more + lane) * a.f.chunk;
    const uint64_t has = __ballot(at < a.n_tokens && s.key[at] == id);
    const int run = ~has ? __builtin_ctzll(~has) : 64;
    more += run;
    all = run == 64;
  }
  const int c0 = (strip * 64 + lane) * N;
  if (c0 >= a.dim) return;
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0, cnt = a.dim >= N ? N : a.dim;
  // the tail of this chunk, then the heads of those after it
  const float *head = s.part + (int64_t)chunk * 2 * a.dim + col;
  float acc[N];
  kept(head + a.dim, cnt, acc);
  for (int i0 = 1; i0 <= more; i0 += kJoinAhead) {
    float v[kJoinAhead][N];
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j) kept(head + (int64_t)min(i0 + j, more) * 2 * a.dim, cnt, v[j]);
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += i0 + j <= more ? v[j][e] : 0.f;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] *= a.scale;
  store_n<W>((W *)a.w.data + (int64_t)id * a.w.ts + col, cnt, acc);
}

// Zeros in `rows` rows of `bytes` bytes, a vector a thread: a workgroup that stores
// once and ends keeps the chip writing in the order of the addresses (1 GB: 6.9 TB/s by
// 4 KB a workgroup, 5.5 to 6.1 by 8 to 256 KB).  lanes: of a row, up to 256.
using plan::kFillBytes;
using plan::kFillThreads;

__global__ __launch_bounds__(kFillThreads) void embedding_fill_kernel(char *dw, int64_t rows, int64_t bytes, int64_t row_bytes, int64_t strips, int lanes) {
  if (rows == 1) {                               // side by side: cut at lines
    const int64_t skew = (intptr_t)dw & 127;
    for (int64_t unit = blockIdx.x; unit < strips; unit += gridDim.x) {
      const int64_t at = unit * kFillBytes - skew + 16 * (int)threadIdx.x;
      if (at >= 0 && at + 16 <= bytes) *(u32x4 *)(dw + at) = u32x4{};
      else
        for (int64_t c = max(at, (int64_t)0); c < min(at + 16, bytes); c += 2) *(uint16_t *)(dw + c) = 0;
    }
    return;
  }
  const int per = kFillThreads / lanes;
  const int64_t groups = (rows + per - 1) / per;
  for (int64_t unit = blockIdx.x; unit < groups * strips; unit += gridDim.x) {
    const int64_t group = unit / strips, v = group * per + threadIdx.x / lanes, c = (unit - group * strips) * kFillBytes + 16 * ((int)threadIdx.x % lanes);
    if (v >= rows || c >= bytes) continue;
    char *const w = dw + v * row_bytes;
    if (bytes >= 16) *(u32x4_any *)(w + min(c, bytes - 16)) = u32x4{};   // (the last vector reaches back)
    else
      for (int i = 0; i < bytes; i += 2) *(uint16_t *)(w + i) = 0;
  }
}

// Few tokens, after the zeros: a workgroup a token and strip of columns, its waves a
// run of the tokens each.  They find those of the workgroup's id, and if none comes
// before its own add their rows, the runs' sums in order.
constexpr int kFewWaves = 4;

template <class W, class Y>
__global__ __launch_bounds__(64 * kFewWaves) void embedding_few_kernel(EmbedArgs a, int strips) {
  constexpr int N = kVec<Y>, kIds = plan::kEmbedFew / 64 / kFewWaves;
  static_assert(64 * kFewWaves * kIds == plan::kEmbedFew, "a place for every token");
  __shared__ float sums[kFewWaves - 1][N][64];
  __shared__ int earlier[kFewWaves];
  const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)blockIdx.x / strips, c0 = (((int)blockIdx.x - t * strips) * 64 + lane) * N;
  const int groups = (a.n_tokens + 64 * kFewWaves - 1) / (64 * kFewWaves), first = 64 * groups * wave;   // of 64 a run
  int64_t id[kIds];
#pragma unroll
  for (int i = 0; i < kIds; ++i) id[i] = i < groups && first + 64 * i + lane < a.n_tokens ? a.tokens[first + 64 * i + lane] : -1;
  const int64_t v = a.tokens[t];
  if (v < 0 || v >= a.vocab) return;
  uint64_t same[kIds];
  bool before = false;
#pragma unroll
  for (int i = 0; i < kIds; ++i) {
    same[i] = __ballot(id[i] == v);
    const int left = t - first - 64 * i;         // tokens of the group before this one
    before |= left > 0 && (same[i] & (left < 64 ? (uint64_t(1) << left) - 1 : ~uint64_t(0)));
  }
  if (lane == 0) earlier[wave] = before;
  __syncthreads();
  for (int w = 0; w < kFewWaves; ++w)
    if (earlier[w]) return;
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0, cnt = a.dim >= N ? N : a.dim;
  const Y *dy = (const Y *)a.y.data + col;
  float acc[N] = {};
#pragma unroll
  for (int i = 0; i < kIds; ++i) {
    uint64_t in = same[i];
    while (in) {
      int at[kAhead], some = 0;                  // as many in flight; the last again where there are fewer
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        at[k] = in ? first + 64 * i + __builtin_ctzll(in) : at[k > 0 ? k - 1 : 0];
        some += in != 0;
        in &= in - 1;
      }
      if (a.dim >= N) {
        u32x4 raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) raw[k] = *(const u32x4_any *)(dy + (int64_t)at[k] * a.y.ts);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (k >= some) break;
          float x[N];
          unpack<Y>(raw[k], x);
#pragma unroll
          for (int e = 0; e < N; ++e) acc[e] += x[e];
        }
      } else {
        for (int k = 0; k < some; ++k) {
          float x[N];
          load_some(dy + (int64_t)at[k] * a.y.ts, cnt, 0.f, x);
#pragma unroll
          for (int e = 0; e < N; ++e) acc[e] += x[e];
        }
      }
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < N; ++e) sums[wave - 1][e][lane] = acc[e];
  }
  __syncthreads();
  if (wave > 0 || c0 >= a.dim) return;
#pragma unroll
  for (int w = 0; w < kFewWaves - 1; ++w)
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] += sums[w][e][lane];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] *= a.scale;
  store_n<W>((W *)a.w.data + v * a.w.ts + col, cnt, acc);
}

template <class W, class Y>
hipError_t fwd(const EmbedArgs &a, hipStream_t s) {
  const int64_t vecs = plan::ceil_div(a.dim, kPair<W, Y>);
  if (vecs <= 64) {
    int bits = 0;
    while ((1 << bits) < vecs) ++bits;
    embedding_narrow_kernel<W, Y><<<(int)plan::ceil_div(a.n_tokens, 4 * kFwdVecs * (64 >> bits)), 256, 0, s>>>(a, bits);
    return hipGetLastError();
  }
  const int strips = (int)plan::ceil_div(vecs, 64 * kFwdVecs);
  const int64_t groups = plan::ceil_div((int64_t)a.n_tokens * strips, 4);
  embedding_fwd_kernel<W, Y><<<(int)(groups < (1 << 20) ? groups : 1 << 20), 256, 0, s>>>(a, strips);
  return hipGetLastError();
}

template <class W, class Y>
hipError_t bwd(const EmbedArgs &a, hipStream_t s) {
  const plan::EmbedBwd &f = a.f;
  if (plan::embed_few(a.n_tokens, a.dim, (int)sizeof(Y))) {   // (also of none)
    const int64_t row_bytes = a.w.ts * (int64_t)sizeof(W);
    const plan::EmbedFill z = plan::embed_fill(a.vocab, a.dim * (int64_t)sizeof(W), row_bytes);
    embedding_fill_kernel<<<z.grid, kFillThreads, 0, s>>>(a.w.data, z.rows, z.bytes, row_bytes, z.strips, z.lanes);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_tokens == 0) return e;
    const int sum_strips = (int)plan::ceil_div(a.dim, 64 * kVec<Y>);
    embedding_few_kernel<W, Y><<<a.n_tokens * sum_strips, 64 * kFewWaves, 0, s>>>(a, sum_strips);
    return hipGetLastError();
  }
  SortArgs k{};
  k.tokens = a.tokens;
  k.n_tokens = a.n_tokens;
  k.vocab = a.vocab;
  k.blocks = f.blocks;
  k.passes = f.passes;
  k.bits = f.bits;
  k.dw = a.w.data;
  k.row_bytes = a.w.ts * (int64_t)sizeof(W);
  k.row_elems = a.dim;
  k.elem_bytes = (int)sizeof(W);
  const bool flags = f.blocks > 0, side_by_side = !flags && k.row_bytes == (int64_t)a.dim * (int)sizeof(W);
  k.groups = (int)(side_by_side ? plan::ceil_div(a.vocab * k.row_bytes + 127, kZeroBytes) : plan::ceil_div(a.vocab, kZeroRows));
  const int zero = k.groups < kZeroGrid ? k.groups : kZeroGrid;
  uint32_t *const key[2] = {(uint32_t *)(a.ws + f.key_off[0]), (uint32_t *)(a.ws + f.key_off[1])};
  uint32_t *const token[2] = {(uint32_t *)(a.ws + f.token_off[0]), (uint32_t *)(a.ws + f.token_off[1])};
  int in = 0;                                    // where the sorted list ends up
  hipError_t e = hipSuccess;
  if (f.blocks == 0) {
    k.key_out = key[0];
    k.token_out = token[0];
    if (a.n_tokens <= kRounds * kSortThreads) embedding_sort_kernel<kRounds><<<1 + zero, kSortThreads, 0, s>>>(k);
    else if (a.n_tokens <= 2 * kRounds * kSortThreads) embedding_sort_kernel<2 * kRounds><<<1 + zero, kSortThreads, 0, s>>>(k);
    else embedding_sort_kernel<kWholeRounds><<<1 + zero, kSortThreads, 0, s>>>(k);
    e = hipGetLastError();
  } else {
    k.hist = (uint32_t *)(a.ws + f.hist_off);
    k.flags = (uint8_t *)(a.ws + f.flag_off);
    for (int p = 0; p < f.passes && e == hipSuccess; ++p) {
      k.first = p == 0;
      k.shift = p * f.bits;
      k.key_in = key[in];
      k.token_in = token[in];
      if (p > 0) in ^= 1;
      k.key_out = key[in];
      k.token_out = token[in];
      embedding_count_kernel<<<f.blocks, kSortThreads, 0, s>>>(k);
      if ((e = hipGetLastError()) != hipSuccess) break;
      // every workgroup adds the others' counts itself, unless that would be most of its work
      k.added = f.blocks > 128;
      if (k.added) embedding_add_kernel<<<(1 << f.bits) / 64 + 1, 64, 0, s>>>(k);
      if ((e = hipGetLastError()) != hipSuccess) break;
      // (after one pass alone the flags are not all set before its end)
      const bool zeroes = p == f.passes - 1 && p > 0;
      embedding_move_kernel<<<f.blocks + (zeroes ? zero : 0), kSortThreads, 0, s>>>(k);
      e = hipGetLastError();
    }
    if (e == hipSuccess && f.passes == 1) {
      embedding_zero_kernel<<<zero, kSortThreads, 0, s>>>(k);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  SumArgs r{};
  r.a = a;
  r.key = key[in];
  r.token = token[in];
  r.part = (float *)(a.ws + f.part_off);
  r.strips = (int)plan::ceil_div(a.dim, 64 * kVec<Y>);
  int bits = 0;
  while ((1 << bits) < plan::ceil_div(a.dim, kVec<Y>)) ++bits;
  const int64_t waves = (int64_t)f.chunks * r.strips;
  if (bits < 6) embedding_sum_kernel<W, Y, true, true><<<(int)plan::ceil_div(f.chunks, 4 * (64 >> bits)), 256, 0, s>>>(r, bits);
  else if (waves <= 8192) embedding_sum_kernel<W, Y, false, true><<<(int)plan::ceil_div(waves, 4), 256, 0, s>>>(r, bits);
  else embedding_sum_kernel<W, Y, false, false><<<(int)plan::ceil_div(waves, 4), 256, 0, s>>>(r, bits);
  e = hipGetLastError();
  if (e != hipSuccess || f.chunks == 1) return e;
  embedding_join_kernel<W, Y><<<(int)plan::ceil_div((f.chunks - 1) * (int64_t)r.strips, kJoinWaves), 64 * kJoinWaves, 0, s>>>(r);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_fwd(bool w_f32, bool y_f32, const EmbedArgs &a, hipStream_t s) {
  if (w_f32) return y_f32 ? fwd<float, float>(a, s) : fwd<float, bf16>(a, s);
  return y_f32 ? fwd<bf16, float>(a, s) : fwd<bf16, bf16>(a, s);
}
hipError_t launch_embedding_bwd(bool w_f32, bool y_f32, const EmbedArgs &a, hipStream_t s) {
  if (w_f32) return y_f32 ? bwd<float, float>(a, s) : bwd<float, bf16>(a, s);
  return y_f32 ? bwd<bf16, float>(a, s) : bwd<bf16, bf16>(a, s);
}

}  // namespace nsp
