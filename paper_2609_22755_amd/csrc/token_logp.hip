// Log probabilities of given tokens with entropy and top alternatives, and the
// gradient of the logits, for gfx950.
//
// Bound by HBM: the forward reads the logits once (2 bytes of bf16 and one
// exponential an element), the backward reads and writes them once.
//
// Forward: one pass with a running reference m, sum s = sum 2^d and weighted
// sum u = sum 2^d d of d = (z - m) log2(e) in every lane, so
//     lse = m + ln s,   entropy = ln s - ln 2 u / s.
// The reference need not be the maximum: a lane moves it only when a vector's
// largest logit lies more than 16 powers of two above it (2^16 times the sum
// of a vocabulary is far from float32's range), which after the first vectors
// hardly ever happens.
//
// Top alternatives: a wave keeps its best keys (the logit in an order-keeping
// whole number, then the complement of the index, 64 bits) one a lane, sorted.
// A vector costs one comparison of its largest logit with the wave's k-th best
// as long as nothing enters.  Where more lanes than k have a candidate, the
// k-th largest of the lanes' maxima is a bar that k logits reach: only what
// reaches it is inserted, one after another (rank by a ballot, the keys below
// move one lane up).
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

// ------------------------------------------------------------ running sums --

struct Sums {
  float m = kNoRef, s = 0.f, u = 0.f;

  // The same sums with reference r >= m; c = scale log2(e).
  __device__ __forceinline__ void move(float r, float c) {
    const float d = fmaxf((m - r) * c, -1e4f);   // (an exponential of 0 long before; keeps d s finite)
    const float f = exp2_fast(d);
    u = f * (u + d * s);
    s *= f;
    m = r;
  }
  __device__ __forceinline__ void add(const Sums &o) { s += o.s; u += o.u; }
};

// Over the lanes of a wave, in every lane.
__device__ __forceinline__ void wave_join(Sums &x, float c) {
  x.move(wave_max(x.m), c);
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
__device__ __forceinline__ uint64_t key_of(float x, int index) {
  return ((uint64_t)order_of(x) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// A wave's best keys, lane i the i-th; 0 where there is none.
struct TopKeys {
  uint64_t key = 0;

  __device__ __forceinline__ uint64_t kth(int k) const { return lane_key(key, k - 1); }
  // The logit that a new one has to pass.
  __device__ __forceinline__ float threshold(int k) const {
    const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), k - 1);
    return o ? value_of(o) : kMasked;
  }
  __device__ __forceinline__ void insert(uint64_t cand) {   // cand: the same in every lane
    const int rank = __popcll(__ballot(key > cand));
    const uint32_t hi = __shfl_up((uint32_t)(key >> 32), 1), lo = __shfl_up((uint32_t)key, 1);
    const int lane = threadIdx.x & 63;
    if (lane > rank) key = ((uint64_t)hi << 32) | lo;
    else if (lane == rank) key = cand;
  }
};

// A number that at least k of the lanes' x reach (0 if fewer have any): the
// k-th largest to 16 bits.
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t x, int k) {
  uint32_t bar = 0;
  for (int b = 31; b >= 16; --b) {
    const uint32_t t = bar | (1u << b);
    if (__popcll(__ballot(x >= t)) >= k) bar = t;
  }
  return bar;
}

// Vectors of V logits, lane l's with indices base + l V ..; `most`: a lane's largest.
template <int V>
__device__ __forceinline__ void offer(TopKeys &top, float &thr, int k, const float (&z)[V], float most, int base) {
  const uint64_t some = __ballot(most > thr);
  if (!some) return;
  // Earlier vectors have lower indices: their equals stay.  Within this one an
  // equal of the k-th so far may have the lower index, which the key decides.
  const float old = thr;
  float bar = old;
  if (__popcll(some) > k) {
    const uint32_t o = kth_of_lanes(most > old ? order_of(most) : 0u, k);
    if (o) bar = value_of(o);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    uint64_t in = __ballot(z[e] > old && z[e] >= bar);
    if (!in) continue;
    while (in) {
      const int l = __builtin_ctzll(in);
      in &= in - 1;
      const float v = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(z[e]), l));
      top.insert(key_of(v, base + l * V + e));
    }
    thr = top.threshold(k);
    bar = fmaxf(bar, thr);
  }
}

// A sorted key of each lane (0: none).
__device__ __forceinline__ bool offer_keys(TopKeys &top, int k, uint64_t key) {
  const uint64_t some = __ballot(key > top.kth(k));
  if (!some) return false;
  uint32_t bar = 0;
  if (__popcll(some) > k) bar = kth_of_lanes((uint32_t)(key >> 32), k);
  uint64_t in = __ballot(key > top.kth(k) && (uint32_t)(key >> 32) >= bar);
  while (in) {
    const int l = __builtin_ctzll(in);
    in &= in - 1;
    top.insert(lane_key(key, l));
  }
  return true;
}

// ----------------------------------------------------------------- forward --

// What a row comes to, by one wave that holds its sums and keys.
template <class T>
__device__ __forceinline__ void finish_row(const LogpArgs &a, int row, const Sums &x, const TopKeys &top) {
  const int lane = threadIdx.x & 63;
  const float ln_s = __logf(x.s);
  const bool none = x.s == 0.f;                 // nothing but masked logits
  const float lse = none ? kNegInf : x.m * a.scale + ln_s;
  if (lane == 0) {
    a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = none ? 0.f : ln_s - kLn2 * (x.u / x.s);
    if (a.logp) {
      const int64_t y = a.targets[row];
      float lp = 0.f;
      if (y >= 0 && y < a.vocab) {
        const float z = to_f32(((const T *)a.logits + (int64_t)row * a.row_stride)[y]);
        lp = none ? kNegInf : (z - x.m) * a.scale - ln_s;
      }
      a.logp[row] = lp;
    }
  }
  if (lane < a.top) {
    const int64_t at = (int64_t)row * a.top + lane;
    const bool some = top.key != 0;
    a.top_logp[at] = some ? (value_of((uint32_t)(top.key >> 32)) - x.m) * a.scale - ln_s : kNegInf;
    a.top_index[at] = some ? (int64_t)(int32_t)~(uint32_t)top.key : -1;
  }
}

template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logp_fwd_kernel(LogpArgs a) {
  constexpr int V = kVec<T>;
  constexpr int U = 4;                          // vectors of a lane in flight
  __shared__ float4 sums[kWaves];
  __shared__ uint64_t keys[kWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float c = a.scale * kLog2e;
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = (int)(unit / a.parts), part = (int)(unit - (int64_t)row * a.parts);
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    const int lo = part * a.part_len, hi = min(a.vocab, lo + a.part_len);
    Sums x;
    TopKeys top;
    float thr = kMasked;
    for (int b0 = lo; b0 < hi; b0 += kThreads * V * U) {
      float v[U][V];
#pragma unroll
      for (int r = 0; r < U; ++r) {
        const int e0 = b0 + (r * kThreads + (int)threadIdx.x) * V;
        load_vec(z + e0, hi - e0, kNegInf, v[r]);
      }
#pragma unroll
      for (int r = 0; r < U; ++r) {
        float most = v[r][0];
#pragma unroll
        for (int e = 1; e < V; ++e) most = fmaxf(most, v[r][e]);
        const bool up = (most - x.m) * c > 16.f;
        if (__ballot(up)) x.move(up ? most : x.m, c);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = (v[r][e] - x.m) * c;
          const float p = exp2_fast(d);
          x.s += p;
          x.u += p * fmaxf(d, -200.f);          // (a masked one: 0, not 0 times infinity; a NaN stays one in p)
        }
        if constexpr (TOP) offer<V>(top, thr, a.top, v[r], most, b0 + (r * kThreads + wave * 64) * V);
      }
    }
    wave_join(x, c);
    if (lane == 0) sums[wave] = make_float4(x.m, x.s, x.u, 0.f);
    if constexpr (TOP) keys[wave][lane] = lane < a.top ? top.key : 0;
    __syncthreads();
    if (wave == 0) {
      Sums all;
      const float4 f = sums[lane & (kWaves - 1)];
      all.m = f.x;
      all.s = lane < kWaves ? f.y : 0.f;
      all.u = lane < kWaves ? f.z : 0.f;
      wave_join(all, c);
      if constexpr (TOP)
        for (int w = 1; w < kWaves; ++w) offer_keys(top, a.top, keys[w][lane]);
      if (a.parts == 1) {
        finish_row<T>(a, row, all, top);
      } else {
        if (lane == 0) a.part_sums[unit] = make_float4(all.m, all.s, all.u, 0.f);
        if constexpr (TOP)
          if (lane < a.top) a.part_top[unit * a.top + lane] = top.key;
      }
    }
    __syncthreads();                            // before the next unit's sums and keys
  }
}

// One wave a row: its parts' sums and keys, a part a lane.
template <class T>
__global__ __launch_bounds__(64) void token_logp_join_kernel(LogpArgs a) {
  const int lane = threadIdx.x, row = blockIdx.x;
  const int64_t unit = (int64_t)row * a.parts + min(lane, a.parts - 1);
  const float4 f = a.part_sums[unit];
  Sums x;
  x.m = f.x;
  x.s = lane < a.parts ? f.y : 0.f;
  x.u = lane < a.parts ? f.z : 0.f;
  wave_join(x, a.scale * kLog2e);
  TopKeys top;
  for (int j = 0; j < a.top; ++j)
    if (!offer_keys(top, a.top, lane < a.parts ? a.part_top[unit * a.top + j] : 0)) break;
  finish_row<T>(a, row, x, top);
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
