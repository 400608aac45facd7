// Log probabilities of given tokens with entropy and top alternatives, and the
// gradient of the logits, for gfx950.
//
// Bound by HBM: the forward reads the logits once (2 bytes of bf16 and one
// exponential an element), the backward reads and writes them once.
//
// Forward: one pass with a running reference r, sum s = sum 2^d and weighted sum
// u = sum 2^d d of d = z scale log2(e) - r in every lane, so
//     lse = ln 2 (r + log2 s),   entropy = ln 2 (log2 s - u / s).
// The reference need not be the maximum: a lane moves it only when a vector's
// largest logit lies more than 16 powers of two above it (2^16 times the sum
// of a vocabulary is far from float32's range), which after the first vectors
// hardly ever happens.
//
// Top alternatives, in two steps.  In the pass each lane keeps the largest
// logit of its own elements, one comparison a vector.  The k-th largest of the
// lanes' maxima is a bar that k logits at least reach, and that hardly more
// do; so only the lanes whose maximum reaches it, about k of them, can hold
// alternatives, and only their elements (a 256th of the row each) are read
// once more.  A wave keeps the best keys (the logit in an order-keeping whole
// number, then the complement of the index, 64 bits) one a lane, sorted; a key
// that passes the k-th is inserted by the rank that a ballot gives, the keys
// below moving one lane up.
//
// A workgroup takes a row, or a part of one where there are few rows; the
// parts' sums and keys are then joined by one wave a row.
#include "nsp_internal.hpp"
#include "row_common.hpp"

namespace nsp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxGrid = 1 << 22;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Logits up to here are masked (-inf, and the lowest values of the types).
constexpr float kMasked = -0x1p126f;
// The reference of no logit yet: the next number above, so that a masked one
// is 2^102 or more below it.
constexpr float kNoRef = -0x1.fffffep125f;
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The largest of three, ignoring NaN.  (fmaxf first quiets what it cannot know
// to be quiet, such as bits just unpacked: an instruction an element.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// ------------------------------------------------------------ running sums --

struct Sums {
  float r, s = 0.f, u = 0.f;

  // c: scale log2(e), 2^-64 .. 2^65.
  __device__ __forceinline__ explicit Sums(float c) : r(fmaxf(kNoRef * c, -0x1.fffffep126f)) {}
  // The same sums with a reference to >= r.
  __device__ __forceinline__ void move(float to) {
    const float d = fmaxf(r - to, -1e4f);        // (an exponential of 0 long before; keeps d s finite)
    const float f = exp2_fast(d);
    u = f * (u + d * s);
    s *= f;
    r = to;
  }
};

// Over the lanes of a wave, in every lane.
__device__ __forceinline__ void wave_join(Sums &x) {
  x.move(wave_max(x.r));
  x.s = group_sum<64>(x.s);
  x.u = group_sum<64>(x.u);
}

// -------------------------------------------------------------------- keys --

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 is 0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}
// Each lane's x of the lane below (lane 0: 0).
__device__ __forceinline__ uint32_t from_below(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, false);   // wave_shr:1
}

// A wave's best keys, lane i the i-th; 0 where there is none.
struct TopKeys {
  uint64_t key = 0;

  __device__ __forceinline__ uint64_t kth(int k) const { return lane_key(key, k - 1); }
  __device__ __forceinline__ void insert(uint64_t cand) {   // cand: the same in every lane
    const int rank = __popcll(__ballot(key > cand)), lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)from_below((uint32_t)(key >> 32)) << 32) | from_below((uint32_t)key);
    key = lane > rank ? below : lane == rank ? cand : key;
  }
  // A key of each lane (0: none).
  __device__ __forceinline__ void offer(uint64_t cand, int k) {
    uint64_t least = kth(k);
    uint64_t in = __ballot(cand > least);
    while (in) {
      const int l = __builtin_ctzll(in);
      in &= in - 1;
      const uint64_t c = lane_key(cand, l);
      if (c <= least) continue;
      insert(c);
      least = kth(k);
    }
  }
};

// A number that at least k of the lanes' x[] reach (0 if fewer have any): the
// k-th largest to its upper 16 bits.
template <int N>
__device__ __forceinline__ uint32_t kth_of(const uint32_t (&x)[N], int k) {
  uint32_t bar = 0;
  for (int b = 31; b >= 16; --b) {
    const uint32_t t = bar | (1u << b);
    int have = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) have += __popcll(__ballot(x[i] >= t));
    if (have >= k) bar = t;
  }
  return bar;
}

// ----------------------------------------------------------------- forward --

// The target of a row and its logit.
struct Target {
  bool given = false;
  float z = 0.f;
  template <class T>
  __device__ __forceinline__ void load(const LogpArgs &a, int row, const T *z_row) {
    if (!a.logp) return;
    const int64_t y = a.targets[row];
    given = y >= 0 && y < a.vocab;
    if (given) z = to_f32(z_row[y]);
  }
};

// What a row comes to, by one wave that holds its sums and keys.
__device__ __forceinline__ void finish_row(const LogpArgs &a, int row, float c, const Sums &x, const TopKeys &top,
                                           const Target &y) {
  const int lane = threadIdx.x & 63;
  const float log_s = log2f(x.s);
  const bool none = x.s == 0.f;                 // nothing but masked logits
  const auto logp = [&](float z) { return none ? kNegInf : (fmaf(z, c, -x.r) - log_s) * kLn2; };
  if (lane == 0) {
    a.lse[row] = none ? kNegInf : (x.r + log_s) * kLn2;
    if (a.entropy) a.entropy[row] = none ? 0.f : (log_s - x.u / x.s) * kLn2;
    if (a.logp) a.logp[row] = y.given ? logp(y.z) : 0.f;
  }
  if (lane < a.top) {
    const int64_t at = (int64_t)row * a.top + lane;
    const bool some = top.key != 0;
    a.top_logp[at] = some ? logp(value_of((uint32_t)(top.key >> 32))) : kNegInf;
    a.top_index[at] = some ? (int64_t)(int32_t)~(uint32_t)top.key : -1;
  }
}

// The wave's alternatives among elements lo .. hi of a row, whose lanes'
// largest are in `largest` (of all threads; mine: this thread's).
template <class T>
__device__ __forceinline__ TopKeys find_top(const T *z, int lo, int hi, int k, const float *largest, float mine) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t x[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const float m = largest[i * 64 + lane];
    x[i] = m > kMasked ? order_of(m) : 0;
  }
  const uint32_t bar = kth_of(x, k);
  TopKeys top;
  uint64_t lanes = __ballot(mine > kMasked && order_of(mine) >= bar);
  // a lane's vectors, `each` lanes of the wave on one lane's
  const int vecs = (hi - lo + kThreads * V - 1) / (kThreads * V);
  int shift = 0;
  while (shift < 6 && (1 << shift) < vecs) ++shift;
  const int each = 1 << shift;
  while (lanes) {
    int of = -1;
    for (int g = 0; g < 64 && lanes; g += each) {
      if ((lane & -each) == g) of = __builtin_ctzll(lanes);
      lanes &= lanes - 1;
    }
    for (int j0 = 0; j0 < vecs; j0 += each) {
      const int e0 = lo + ((j0 + (lane & (each - 1))) * kThreads + wave * 64 + of) * V;
      float v[V];
      load_vec(z + e0, of < 0 ? 0 : hi - e0, kNegInf, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t o = order_of(v[e]);
        top.offer(v[e] > kMasked && o >= bar ? ((uint64_t)o << 32) | (uint32_t)~(e0 + e) : 0, k);
      }
    }
  }
  return top;
}

template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logp_fwd_kernel(LogpArgs a) {
  constexpr int V = kVec<T>;
  constexpr int U = 4;                          // vectors of a lane in flight
  __shared__ float4 sums[kWaves];
  __shared__ uint64_t keys[kWaves][64];
  __shared__ float largest[kThreads];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float c = a.scale * kLog2e;
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = (int)(unit / a.parts), part = (int)(unit - (int64_t)row * a.parts);
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    const int lo = part * a.part_len, hi = min(a.vocab, lo + a.part_len);
    Sums x(c);
    Target y;
    if (threadIdx.x == 0 && a.parts == 1) y.load(a, row, z);
    float mine = kNegInf;
    const auto take = [&](const float (&v)[V]) {
      float most = max3(v[0], v[1], v[2]);
#pragma unroll
      for (int e = 3; e < V; e += 2) most = max3(most, v[e], v[e + 1 < V ? e + 1 : e]);
      const bool up = fmaf(most, c, -x.r) > 16.f;
      if (__ballot(up)) x.move(up ? most * c : x.r);
      if constexpr (TOP) mine = fmaxf(mine, most);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = fmaf(v[e], c, -x.r);
        const float p = exp2_fast(d);
        x.s += p;
        x.u = fmaf(p, fmaxf(d, -200.f), x.u);   // (a masked one: 0, not 0 times infinity; a NaN stays one in p)
      }
    };
    int b0 = lo;
    for (; b0 + kThreads * V * U <= hi; b0 += kThreads * V * U) {
      u32x4 raw[U];
#pragma unroll
      for (int i = 0; i < U; ++i) raw[i] = load16(z + b0 + (i * kThreads + (int)threadIdx.x) * V);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        float v[V];
        unpack<T>(raw[i], v);
        take(v);
      }
    }
    for (; b0 < hi; b0 += kThreads * V) {
      const int e0 = b0 + (int)threadIdx.x * V;
      float v[V];
      load_vec(z + e0, hi - e0, kNegInf, v);
      take(v);
    }
    wave_join(x);
    if (lane == 0) sums[wave] = make_float4(x.r, x.s, x.u, 0.f);
    TopKeys top;
    if constexpr (TOP) {
      largest[threadIdx.x] = mine;
      __syncthreads();
      top = find_top(z, lo, hi, a.top, largest, mine);
      keys[wave][lane] = lane < a.top ? top.key : 0;
    }
    __syncthreads();
    if (wave == 0) {
      const float4 f = sums[lane & (kWaves - 1)];
      x.r = f.x;
      x.s = lane < kWaves ? f.y : 0.f;
      x.u = lane < kWaves ? f.z : 0.f;
      wave_join(x);
      if constexpr (TOP)
        for (int w = 1; w < kWaves; ++w) top.offer(keys[w][lane], a.top);
      if (a.parts == 1) {
        finish_row(a, row, c, x, top, y);
      } else {
        if (lane == 0) a.part_sums[unit] = make_float4(x.r, x.s, x.u, 0.f);
        if constexpr (TOP)
          if (lane < a.top) a.part_top[((int64_t)row * a.top + lane) * a.parts + part] = top.key;
      }
    }
    __syncthreads();                            // before the next unit's sums and keys
  }
}

// One wave a row: its parts' sums, a part a lane, and the parts' keys, the best
// of all parts first.
template <class T>
__global__ __launch_bounds__(64) void token_logp_join_kernel(LogpArgs a) {
  const int lane = threadIdx.x, row = blockIdx.x;
  const float c = a.scale * kLog2e;
  Target y;
  if (lane == 0) y.load(a, row, (const T *)a.logits + (int64_t)row * a.row_stride);
  const float4 f = a.part_sums[(int64_t)row * a.parts + min(lane, a.parts - 1)];
  TopKeys top;
  const int keys = a.parts * a.top;
  const uint64_t *from = a.part_top + (int64_t)row * keys;
  uint64_t key = lane < keys ? from[lane] : 0;
  for (int i = 0; i < keys; i += 64) {
    const uint64_t next = i + 64 + lane < keys ? from[i + 64 + lane] : 0;
    if (i == 0) {
      const uint32_t x[1] = {(uint32_t)(key >> 32)};
      if (x[0] < kth_of(x, a.top)) key = 0;     // (as many as are wanted reach it)
    }
    top.offer(key, a.top);
    key = next;
  }
  Sums x(c);
  x.r = f.x;
  x.s = lane < a.parts ? f.y : 0.f;
  x.u = lane < a.parts ? f.z : 0.f;
  wave_join(x);
  finish_row(a, row, c, x, top, y);
}

// ---------------------------------------------------------------- backward --

constexpr int kBwdVecs = 4;   // vectors of a lane

template <class T>
__global__ __launch_bounds__(kThreads) void token_logp_bwd_kernel(LogpBwdArgs a, int chunks) {
  constexpr int V = kVec<T>;
  const int64_t units = (int64_t)a.n_tokens * chunks;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = (int)(unit / chunks), chunk = (int)(unit - (int64_t)row * chunks);
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    T *dz = (T *)a.dlogits + (int64_t)row * a.d_row_stride;
    const int64_t target = a.g_logp ? a.targets[row] : -1;
    const bool given = target >= 0 && target < a.vocab;
    const int y = given ? (int)target : -1;
    const float gl = given ? a.g_logp[row] : 0.f;
    const float gs = a.g_lse ? a.g_lse[row] : 0.f, ge = a.g_entropy ? a.g_entropy[row] : 0.f;
    const float lse = a.lse[row];
    const bool zero = lse == kNegInf || (gl == 0.f && gs == 0.f && ge == 0.f);
    // dz = p (k0 + k1 d), d = (z - lse) log2(e)
    const float k0 = a.scale * (gs - gl - (ge != 0.f ? ge * a.entropy[row] : 0.f));
    const float k1 = -a.scale * ge * kLn2, at_y = a.scale * gl;
    const int first = chunk * (kThreads * V * kBwdVecs);
    float v[kBwdVecs][V];
    if (zero) {
#pragma unroll
      for (int r = 0; r < kBwdVecs; ++r) {
        const int e0 = first + (r * kThreads + (int)threadIdx.x) * V;
        const float o[V] = {};
        store_vec(dz + e0, a.vocab - e0, o);
      }
      continue;
    }
#pragma unroll
    for (int r = 0; r < kBwdVecs; ++r) {
      const int e0 = first + (r * kThreads + (int)threadIdx.x) * V;
      load_vec(z + e0, a.vocab - e0, kNegInf, v[r]);
    }
#pragma unroll
    for (int r = 0; r < kBwdVecs; ++r) {
      const int e0 = first + (r * kThreads + (int)threadIdx.x) * V;
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = (v[r][e] * a.scale - lse) * kLog2e;
        const float p = exp2_fast(d);
        o[e] = p * (k0 + k1 * fmaxf(d, -200.f));
      }
      if ((uint32_t)(y - e0) < (uint32_t)V) {
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += y - e0 == e ? at_y : 0.f;
      }
      store_vec(dz + e0, a.vocab - e0, o);
    }
  }
}

template <class T>
hipError_t fwd(LogpArgs a, hipStream_t s) {
  constexpr int V = kVec<T>;
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  a.part_len = (((a.vocab + a.parts - 1) / a.parts) + V - 1) / V * V;
  const int grid = (int)(units < kMaxGrid ? units : kMaxGrid);
  if (a.top > 0) token_logp_fwd_kernel<T, true><<<grid, kThreads, 0, s>>>(a);
  else token_logp_fwd_kernel<T, false><<<grid, kThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  token_logp_join_kernel<T><<<a.n_tokens, 64, 0, s>>>(a);
  return hipGetLastError();
}

template <class T>
hipError_t bwd(const LogpBwdArgs &a, hipStream_t s) {
  constexpr int per = kThreads * kVec<T> * kBwdVecs;
  const int chunks = (int)(((int64_t)a.vocab + per - 1) / per);
  const int64_t units = (int64_t)a.n_tokens * chunks;
  token_logp_bwd_kernel<T><<<(int)(units < kMaxGrid ? units : kMaxGrid), kThreads, 0, s>>>(a, chunks);
  return hipGetLastError();
}

}  // namespace

int token_logp_parts(int64_t n_tokens, int vocab) {
  if (n_tokens <= 0) return 1;
  int64_t p = (2048 + n_tokens - 1) / n_tokens;
  const int64_t most = (vocab + 2047) / 2048;
  if (p > most) p = most;
  if (p > kLogpMaxParts) p = kLogpMaxParts;
  return (int)p;
}

hipError_t launch_token_logp_fwd(bool f32, const LogpArgs &a, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_token_logp_bwd(bool f32, const LogpBwdArgs &a, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace nsp
