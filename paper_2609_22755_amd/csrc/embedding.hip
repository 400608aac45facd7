// Rows of an embedding table, and its gradient, for gfx950.
//
//     y_t = scale w[i_t],     dw_v = scale sum over t with i_t = v of dy_t
//
// Bound by HBM: the forward reads a row and writes one a token, the backward reads
// one a token and writes every row of the table.
//
// Backward: the tokens are sorted by their ids, stably (counting sort, digit by
// digit), so that a row's tokens lie side by side in their order and every sum has
// a fixed order, without an atomic.  A wave takes a chunk of the sorted list and a
// strip of columns, adds rows as long as the id stays the same and stores each id's
// sum: to the table, or, where the id goes on beyond the chunk, in float32 for a
// second kernel that adds the chunks' sums in order.  Rows of ids that no token has
// are zeroed beside that.
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

// Vectors of a lane: a wave takes a strip of so many times 64 of a row.
constexpr int kFwdVecs = 4;

template <class W, class Y>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(EmbedArgs a, int strips) {
  constexpr int N = kVec<W> < kVec<Y> ? kVec<W> : kVec<Y>;   // elements of a lane's vector
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
    if (a.dim >= N) {
#pragma unroll
      for (int i = 0; i < kFwdVecs; ++i) {
        if constexpr (N == kVec<W>) {
          u32x4 raw = {};
          if (some && c0 + i * 64 * N < a.dim) raw = *(const u32x4_any *)(w + at(i));
          unpack<W>(raw, x[i]);
        } else {                       // half a vector of bf16
          u32x2_any raw = {};
          if (some && c0 + i * 64 * N < a.dim) raw = *(const u32x2_any *)(w + at(i));
          const u32x4 both = {raw[0], raw[1], 0, 0};
          float v8[kVec<W>];
          unpack<W>(both, v8);
#pragma unroll
          for (int e = 0; e < N; ++e) x[i][e] = v8[e];
        }
      }
#pragma unroll
      for (int i = 0; i < kFwdVecs; ++i) {
        if (c0 + i * 64 * N >= a.dim) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) x[i][e] *= a.scale;
        if constexpr (N == kVec<Y>) store16(y + at(i), pack<Y>(x[i]));
        else store_half(y + at(i), x[i]);
      }
    } else if (c0 < a.dim) {           // (less than a vector: one lane)
      for (int e = 0; e < a.dim; ++e) y[e] = (Y)(some ? to_f32(w[e]) * a.scale : 0.f);
    }
  }
}

// -------------------------------------------------------------------- sort --

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortRounds = plan::kSortBlock / kSortThreads;
constexpr int kMaxBins = 1 << 10;

struct SortArgs {
  const int64_t *tokens;       // the first pass reads these
  const uint32_t *key_in, *token_in;
  uint32_t *key_out, *token_out, *hist;
  uint8_t *flags;
  int32_t n_tokens, vocab, blocks, shift, bits;
  bool first;                  // pass
};

__device__ __forceinline__ uint32_t key_of(int64_t token, int vocab) { return token >= 0 && token < vocab ? (uint32_t)token : (uint32_t)vocab; }

__device__ __forceinline__ void clear_flags(uint8_t *flags, int vocab, int first, int step) {
  u32x4 *f = (u32x4 *)flags;                     // (whole 256 bytes)
  for (int i = first; i < (vocab + 15) / 16; i += step) f[i] = u32x4{};
}

// How many of a block's keys have each digit.
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(SortArgs a) {
  __shared__ int bins[kMaxBins];
  const int n_bins = 1 << a.bits;
  for (int i = threadIdx.x; i < n_bins; i += kSortThreads) bins[i] = 0;
  if (a.first) clear_flags(a.flags, a.vocab, blockIdx.x * kSortThreads + threadIdx.x, gridDim.x * kSortThreads);
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = blockIdx.x * plan::kSortBlock + r * kSortThreads + threadIdx.x;
    if (i < a.n_tokens) {
      const uint32_t k = a.first ? key_of(a.tokens[i], a.vocab) : a.key_in[i];
      atomicAdd(&bins[(k >> a.shift) & (n_bins - 1)], 1);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_bins; i += kSortThreads) a.hist[(int64_t)i * a.blocks + blockIdx.x] = bins[i];
}

// The sum of the values of the threads before this one; `total`: of all.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *sh, uint32_t &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t up = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(up, d);
    up += lane >= d ? o : 0;
  }
  __syncthreads();                               // (sh may still be read)
  if (lane == 63) sh[wave] = up;
  __syncthreads();
  uint32_t before = up - x;
  total = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    const uint32_t s = sh[w];
    before += w < wave ? s : 0;
    total += s;
  }
  return before;
}

// Counts to places: one workgroup over digits, then blocks.
__global__ __launch_bounds__(kSortThreads) void embedding_scan_kernel(SortArgs a) {
  __shared__ uint32_t sh[kSortWaves];
  const int64_t n = (int64_t)a.blocks << a.bits;
  uint32_t base = 0;
  for (int64_t i0 = 0; i0 < n; i0 += 8 * kSortThreads) {
    const int64_t i = i0 + 8 * (int64_t)threadIdx.x;
    uint32_t v[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = i + e < n ? a.hist[i + e] : 0;
      sum += v[e];
    }
    uint32_t total;
    uint32_t at = base + sum_before(sum, sh, total);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (i + e < n) a.hist[i + e] = at;
      at += v[e];
    }
    base += total;
  }
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
struct Ranks {
  uint32_t key[kSortRounds], token[kSortRounds], rank[kSortRounds];

  template <class Key>
  __device__ __forceinline__ void take(uint32_t *counts, int n, int first, int shift, int bits, Key key_at) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      const int i = first + 64 * r + lane;
      const bool there = i < n;
      key[r] = 0;
      token[r] = 0;
      if (there) key_at(i, key[r], token[r]);
      const uint32_t d = (key[r] >> shift) & ((1u << bits) - 1);
      const uint64_t m = alike(d, bits, there);
      const uint32_t have = there ? counts[d] : 0;
      rank[r] = have + __popcll(m & ((uint64_t(1) << lane) - 1));
      if (there && (m >> lane) == 1) counts[d] = have + __popcll(m);   // the last of them
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// The keys of a block to their places by one digit.
__global__ __launch_bounds__(kSortThreads) void embedding_move_kernel(SortArgs a) {
  __shared__ uint32_t counts[kSortWaves][kMaxBins];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n_bins = 1 << a.bits;
  for (int i = threadIdx.x; i < kSortWaves * n_bins; i += kSortThreads) counts[i >> a.bits][i & (n_bins - 1)] = 0;
  __syncthreads();
  const int first = blockIdx.x * plan::kSortBlock + wave * (64 * kSortRounds);
  Ranks x;
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
  __syncthreads();
  for (int b = threadIdx.x; b < n_bins; b += kSortThreads) {
    uint32_t at = a.hist[(int64_t)b * a.blocks + blockIdx.x];
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = counts[w][b];
      counts[w][b] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (first + 64 * r + lane >= a.n_tokens) continue;
    const uint32_t at = counts[wave][(x.key[r] >> a.shift) & (n_bins - 1)] + x.rank[r];
    a.key_out[at] = x.key[r];
    a.token_out[at] = x.token[r];
  }
}

// All passes of one block, in LDS.
__global__ __launch_bounds__(kSortThreads) void embedding_sort_kernel(SortArgs a, int passes) {
  __shared__ uint32_t counts[kSortWaves][kMaxBins];
  __shared__ uint32_t keys[plan::kSortBlock], places[plan::kSortBlock], sh[kSortWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n_bins = 1 << a.bits;
  clear_flags(a.flags, a.vocab, threadIdx.x, kSortThreads);
  __syncthreads();
  const int first = wave * (64 * kSortRounds);
  for (int p = 0; p < passes; ++p) {
    const int shift = p * a.bits;
    for (int i = threadIdx.x; i < kSortWaves * n_bins; i += kSortThreads) counts[i >> a.bits][i & (n_bins - 1)] = 0;
    __syncthreads();
    Ranks x;
    x.take(counts[wave], a.n_tokens, first, shift, a.bits, [&](int i, uint32_t &k, uint32_t &t) {
      if (p == 0) {
        k = key_of(a.tokens[i], a.vocab);
        t = (uint32_t)i;
        if (k < (uint32_t)a.vocab) a.flags[k] = 1;
      } else {
        k = keys[i];
        t = places[i];
      }
    });
    __syncthreads();
    uint32_t sum = 0, total;
    if ((int)threadIdx.x < n_bins)
      for (int w = 0; w < kSortWaves; ++w) sum += counts[w][threadIdx.x];
    uint32_t at = sum_before(sum, sh, total);
    if ((int)threadIdx.x < n_bins)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = counts[w][threadIdx.x];
        counts[w][threadIdx.x] = at;
        at += c;
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      if (first + 64 * r + lane >= a.n_tokens) continue;
      const uint32_t to = counts[wave][(x.key[r] >> shift) & (n_bins - 1)] + x.rank[r];
      if (p == passes - 1) {
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

// ---------------------------------------------------------------- backward --

struct SumArgs {
  EmbedArgs a;
  const uint32_t *key, *token;  // sorted
  const uint8_t *flags;
  float *part;                  // [chunk][head, tail][dim]
  int strips, sum_groups;       // strips of columns; workgroups that sum (the others zero)
};

constexpr int kAhead = 8;       // rows of a wave in flight

// A chunk's sums of a strip.
template <class W, class Y>
__device__ __forceinline__ void sum_chunk(const SumArgs &s, int chunk, int strip) {
  constexpr int N = kVec<Y>;
  const EmbedArgs &a = s.a;
  const int lane = threadIdx.x & 63;
  const int c0 = (strip * 64 + lane) * N;
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0, cnt = a.dim >= N ? N : a.dim;
  const bool there = c0 < a.dim;
  const int lo = chunk * a.f.chunk, hi = min(lo + a.f.chunk, a.n_tokens);
  const Y *dy = (const Y *)a.y.data + col;
  float acc[N] = {};
  uint32_t id = s.key[lo];
  bool open = lo > 0 && s.key[lo - 1] == id;       // the id's rows began before the chunk
  const auto end = [&](bool goes_on) {
    if (id < (uint32_t)a.vocab && there) {
      if (open || goes_on) {
        // (of a chunk that lies within one id's rows only the head is used)
        float *to = s.part + ((int64_t)chunk * 2 + (open ? 0 : 1)) * a.dim + col;
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < cnt) to[e] = acc[e];
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
  for (int p = lo; p < hi; p += kAhead) {
    u32x4 raw[kAhead];
    float few[N];
    uint32_t ids[kAhead];
    if (a.dim >= N) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = min(p + i, hi - 1);
        ids[i] = s.key[at];
        raw[i] = u32x4{};
        if (there && p + i < hi && ids[i] < (uint32_t)a.vocab) raw[i] = load16(dy + (int64_t)s.token[at] * a.y.ts);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ids[i] = s.key[min(p + i, hi - 1)];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p + i >= hi) break;
      if (ids[i] != id) {
        end(false);
        id = ids[i];
      }
      if (a.dim >= N) {
        unpack<Y>(raw[i], few);
      } else {
        load_some(dy + (int64_t)s.token[p + i] * a.y.ts, there && id < (uint32_t)a.vocab ? cnt : 0, 0.f, few);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += few[e];
    }
  }
  end(hi < a.n_tokens && s.key[hi] == id);
}

template <class W, class Y>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs s) {
  const EmbedArgs &a = s.a;
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < s.sum_groups) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunk = (int)(unit / s.strips), strip = (int)(unit - (int64_t)chunk * s.strips);
    if (chunk < a.f.chunks) sum_chunk<W, Y>(s, chunk, strip);
    return;
  }
  // rows without tokens
  constexpr int N = kVec<W>;
  const int64_t step = (int64_t)(gridDim.x - s.sum_groups) * 4;
  for (int64_t v = (int64_t)(blockIdx.x - s.sum_groups) * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6); v < a.vocab; v += step) {
    if (s.flags && s.flags[v]) continue;
    W *w = (W *)a.w.data + v * a.w.ts;
    if (a.dim >= N) {
      for (int c = lane * N; c < a.dim; c += 64 * N) store16(w + min(c, a.dim - N), u32x4{});
    } else if (lane < a.dim) {
      w[lane] = (W)0.f;
    }
  }
}

// The rows of an id that goes over several chunks: a workgroup a strip and chunk
// that one begins in; its waves take the chunks in turn.
template <class W, class Y>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs s) {
  constexpr int N = kVec<Y>;
  __shared__ float sh[4][64][N + 1];
  const EmbedArgs &a = s.a;
  const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = (int)(blockIdx.x / s.strips), strip = (int)(blockIdx.x - (int64_t)chunk * s.strips);
  const int lo = chunk * a.f.chunk, hi = lo + a.f.chunk;    // (never the last chunk)
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
  const int col = a.dim >= N ? min(c0, a.dim - N) : 0, cnt = a.dim >= N ? N : a.dim;
  const bool there = c0 < a.dim;
  float acc[N] = {};
  if (there) {
    // part 0 is the tail of this chunk, part i the head of the i-th after it
    const float *from = s.part + col;
    const auto at = [&](int i) { return from + ((int64_t)(chunk + i) * 2 + (i == 0 ? 1 : 0)) * a.dim; };
    for (int i0 = wave; i0 <= more; i0 += 16) {
      float v[4][N];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) v[j][e] = i0 + 4 * j <= more && e < cnt ? at(i0 + 4 * j)[e] : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += v[j][e];
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) sh[wave][lane][e] = acc[e];
  __syncthreads();
  if (wave != 0 || !there) return;
  float o[N];
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = ((sh[0][lane][e] + sh[1][lane][e]) + (sh[2][lane][e] + sh[3][lane][e])) * a.scale;
  store_n<W>((W *)a.w.data + (int64_t)id * a.w.ts + col, cnt, o);
}

template <class W, class Y>
hipError_t fwd(const EmbedArgs &a, hipStream_t s) {
  constexpr int N = kVec<W> < kVec<Y> ? kVec<W> : kVec<Y>;
  const int strips = (int)plan::ceil_div(a.dim, 64 * N * kFwdVecs);
  const int64_t groups = plan::ceil_div((int64_t)a.n_tokens * strips, 4);
  embedding_fwd_kernel<W, Y><<<(int)(groups < (1 << 20) ? groups : 1 << 20), 256, 0, s>>>(a, strips);
  return hipGetLastError();
}

template <class W, class Y>
hipError_t bwd(const EmbedArgs &a, hipStream_t s) {
  const plan::EmbedBwd &f = a.f;
  const int64_t rows = plan::ceil_div(a.vocab, 4);
  const int zero_groups = (int)(rows < 65536 ? rows : 65536);
  SumArgs r{};
  r.a = a;
  if (a.n_tokens == 0) {
    embedding_sum_kernel<W, Y><<<zero_groups, 256, 0, s>>>(r);
    return hipGetLastError();
  }
  SortArgs k{};
  k.tokens = a.tokens;
  k.n_tokens = a.n_tokens;
  k.vocab = a.vocab;
  k.blocks = f.blocks;
  k.bits = f.bits;
  k.hist = (uint32_t *)(a.ws + f.hist_off);
  k.flags = (uint8_t *)(a.ws + f.flag_off);
  uint32_t *const key[2] = {(uint32_t *)(a.ws + f.key_off[0]), (uint32_t *)(a.ws + f.key_off[1])};
  uint32_t *const token[2] = {(uint32_t *)(a.ws + f.token_off[0]), (uint32_t *)(a.ws + f.token_off[1])};
  int in = 0;                                    // where the sorted list ends up
  hipError_t e = hipSuccess;
  if (f.blocks == 1) {
    k.key_out = key[0];
    k.token_out = token[0];
    embedding_sort_kernel<<<1, kSortThreads, 0, s>>>(k, f.passes);
    e = hipGetLastError();
  } else {
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
      embedding_scan_kernel<<<1, kSortThreads, 0, s>>>(k);
      if ((e = hipGetLastError()) != hipSuccess) break;
      embedding_move_kernel<<<f.blocks, kSortThreads, 0, s>>>(k);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  r.key = key[in];
  r.token = token[in];
  r.flags = k.flags;
  r.part = (float *)(a.ws + f.part_off);
  r.strips = (int)plan::ceil_div(a.dim, 64 * kVec<Y>);
  r.sum_groups = (int)plan::ceil_div((int64_t)f.chunks * r.strips, 4);
  embedding_sum_kernel<W, Y><<<r.sum_groups + zero_groups, 256, 0, s>>>(r);
  e = hipGetLastError();
  if (e != hipSuccess || f.chunks == 1) return e;
  embedding_join_kernel<W, Y><<<(int)((f.chunks - 1) * (int64_t)r.strips), 256, 0, s>>>(r);
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
