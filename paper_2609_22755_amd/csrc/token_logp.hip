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
// logit of its own vectors, where it was, and the largest of its other
// vectors.  The k-th largest of the lanes' maxima is a bar that k logits at
// least reach, and that hardly more do: about k lanes have alternatives, nearly
// all of them in their best vector alone, which is read once more (a lane whose
// second vector reaches the bar too reads all of its own).  Whatever reaches the
// bar is gathered in LDS as a key (the logit in an order-keeping whole number,
// then the complement of the index, 64 bits), in any order: a key's rank is the
// number of larger ones.  Only where more gather than there is room for (rows
// of equal logits) a wave keeps its best keys one a lane, sorted, and inserts
// what passes the k-th by the rank that a ballot gives.
//
// A workgroup takes a row, or a part of one where there are few rows; the
// parts' sums and keys are then joined by one workgroup a row.
//
// 4096 x 151643 bf16 200 us, 6.2 TB/s (a read: 7.1; some ten vector operations
// an element, an exponential counting four, keep the vector units busy most of
// that time); 777 x 50021 float32 with 20 alternatives 36 us, 4.3 TB/s; 8 x 131072
// with eight 11 us, two launches.  The gradient of 8192 x 131072 bf16 698 us, 6.1
// TB/s read and written.
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
constexpr float kNan = __builtin_nanf("");

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The largest of three, ignoring NaN.  (fmaxf first quiets what it cannot know
// to be quiet, such as bits just unpacked: an instruction an element.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// ------------------------------------------------------------ running sums --

// From |r| = 2^28 on, r is a rounded number of whole exponents: logits next to
// each other lie further apart than a softmax sees, but their products with
// log2(e) round past each other.  There d is taken from the differences of the
// logits themselves (an operation more an element).
__device__ __forceinline__ bool is_far(float r) { return fabsf(r) >= 0x1p28f; }

struct Sums {
  float r, m = kNoRef, s = 0.f, u = 0.f;        // m: the logit that r = m scale log2(e) comes from

  // c: scale log2(e), 2^-64 .. 2^65.
  __device__ __forceinline__ explicit Sums(float c) : r(fmaxf(kNoRef * c, -0x1.fffffep126f)) {}
  __device__ __forceinline__ Sums(const float4 &f) : r(f.x), m(f.w), s(f.y), u(f.z) {}
  __device__ __forceinline__ float4 packed() const { return make_float4(r, s, u, m); }
  // The same sums with the reference of a logit to >= m (to_r: its r).
  __device__ __forceinline__ void move(float to, float to_r, float c) {
    const float d = fmaxf(is_far(to_r) ? (m - to) * c : r - to_r, -1e4f);   // (an exponential of 0 long before; keeps d s finite)
    const float f = exp2_fast(d);
    u = f * (u + d * s);
    s *= f;
    m = to;
    r = to_r;
  }
};

// Over the lanes of a wave, in every lane.
__device__ __forceinline__ void wave_join(Sums &x, float c) {
  const float to = wave_max(x.m), to_r = wave_max(x.r);   // (r grows with m)
  x.move(to, to_r, c);
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

constexpr int kRoom = kThreads;   // keys that a workgroup gathers

struct Shared {
  float4 sums[kWaves];
  float firsts[kThreads];
  uint64_t keys[kRoom];
  int gathered;
};

// A lane's largest logit, the element its vector starts at, and the largest of
// its other vectors.
struct Largest {
  float first = kNegInf, second = kNegInf;
  int at = 0;
  __device__ __forceinline__ void take(float most, int e0) {
    second = fmaxf(second, fminf(first, most));
    at = most > first ? e0 : at;
    first = fmaxf(first, most);
  }
};

// What a row comes to, from its sums (in every thread) and its alternatives
// (thread i: the i-th, 0 if there is none).
struct Finish {
  float r, m, log_s, c;
  bool none;                 // nothing but masked logits
  // The reference is taken from its logit again: what the sums hold is cut off at
  // -2^127.  Past float32 it leaves nothing of the row but NaN.
  __device__ __forceinline__ Finish(const Sums &x, float scale_log2)
      : r(reference(x.m, scale_log2)), m(x.m), log_s(fabsf(r) < -kNegInf ? log2f(x.s) : kNan), c(scale_log2), none(x.s == 0.f) {}
  __device__ __forceinline__ static float reference(float m, float c) {
#pragma clang fp contract(off)
    return m * c;            // (rounded, as it was subtracted)
  }
  __device__ __forceinline__ float logp(float z) const {
    return none ? kNegInf : ((is_far(r) ? (z - m) * c : fmaf(z, c, -r)) - log_s) * kLn2;
  }
  template <class T>
  __device__ __forceinline__ void row(const LogpArgs &a, int row, const Sums &x, int64_t y, float z) const {
    a.lse[row] = none ? kNegInf : (r + log_s) * kLn2;
    if (a.entropy) a.entropy[row] = none ? 0.f : (log_s - x.u / x.s) * kLn2;
    if (a.logp) a.logp[row] = y >= 0 && y < a.vocab ? logp(z <= kMasked ? kNegInf : z) : 0.f;
  }
  __device__ __forceinline__ void top(const LogpArgs &a, int row, int i, uint64_t key) const {
    const int64_t at = (int64_t)row * a.top + i;
    a.top_logp[at] = key ? logp(value_of((uint32_t)(key >> 32))) : kNegInf;
    a.top_index[at] = key ? (int64_t)(int32_t)~(uint32_t)key : -1;
  }
};

// put(i, key) of the i-th best key, i < k (0: there is none), by any thread.
// each(bar, f) hands f the keys of the thread that reach the bar, whole waves
// together (0: none).  first: the thread's largest logit.  Every thread of the
// workgroup calls this; nothing else of `sh` is read any more.
template <class Each, class Put>
__device__ __forceinline__ void block_top(Shared &sh, int k, float first, Each each, Put put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  sh.firsts[threadIdx.x] = first;
  if (threadIdx.x == 0) sh.gathered = 0;
  __syncthreads();
  uint32_t x[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const float m = sh.firsts[i * 64 + lane];
    x[i] = m > kMasked ? order_of(m) : 0;
  }
  const uint32_t bar = kth_of(x, k);
  each(bar, [&](uint64_t key) {
    if (key) {
      const int at = atomicAdd(&sh.gathered, 1);
      if (at < kRoom) sh.keys[at] = key;
    }
  });
  __syncthreads();
  const int n = sh.gathered;
  if (n <= kRoom) {
    const uint64_t mine = (int)threadIdx.x < n ? sh.keys[threadIdx.x] : 0;
    int rank = (int)threadIdx.x < n ? 0 : (int)threadIdx.x;
    if ((wave << 6) < n) {
      int larger = 0;
      for (int i = 0; i < n; ++i) larger += sh.keys[i] > mine;
      if (mine) rank = larger;
    }
    if (rank < k) put(rank, mine);
  } else {                                      // too many alike: each wave's best, then of the waves'
    TopKeys top;
    each(bar, [&](uint64_t key) { top.offer(key, k); });
    __syncthreads();
    sh.keys[threadIdx.x] = lane < k ? top.key : 0;
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < kWaves; ++w) top.offer(sh.keys[w * 64 + lane], k);
      if (lane < k) put(lane, top.key);
    }
  }
}

template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logp_fwd_kernel(LogpArgs a) {
  constexpr int V = kVec<T>;
  constexpr int U = 4;                          // vectors of a lane in flight
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float c = a.scale * kLog2e;
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = (int)a.by_parts.quot((uint32_t)unit), part = (int)unit - row * a.parts;
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    const int lo = part * a.part_len, hi = min(a.vocab, lo + a.part_len);
    int64_t y = -1;
    float zy = 0.f;
    if (threadIdx.x == 0 && a.parts == 1 && a.logp) {
      y = a.targets[row];
      if (y >= 0 && y < a.vocab) zy = to_f32(z[y]);
    }
    Sums x(c);
    bool far = true;                            // of a lane of the wave (as long as one has no logit yet, too)
    Largest mine;
    const auto take = [&](const float (&v)[V], int e0) {
      float most = max3(v[0], v[1], v[2]);
#pragma unroll
      for (int e = 3; e < V; e += 2) most = max3(most, v[e], v[e + 1 < V ? e + 1 : e]);
      const bool up = (far ? (most - x.m) * c : fmaf(most, c, -x.r)) > 16.f;
      if (__ballot(up)) {
        x.move(up ? most : x.m, up ? most * c : x.r, c);
        far = __any(is_far(x.r));
      }
      if constexpr (TOP) mine.take(most, e0);
      const auto add = [&](float d) {
        const float p = exp2_fast(d);
        x.s += p;
        x.u = fmaf(p, fmaxf(d, -200.f), x.u);   // (a masked one: 0, not 0 times infinity; a NaN stays one in p)
      };
      if (far) {
#pragma unroll
        for (int e = 0; e < V; ++e) add((v[e] - x.m) * c);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) add(fmaf(v[e], c, -x.r));
      }
    };
    const auto place = [&](int b0, int i) { return b0 + (i * kThreads + (int)threadIdx.x) * V; };
    int b0 = lo;
    const auto stream = [&](auto load) {
      for (; b0 + kThreads * V * U <= hi; b0 += kThreads * V * U) {
        u32x4 raw[U];
#pragma unroll
        for (int i = 0; i < U; ++i) raw[i] = load(z + place(b0, i));
#pragma unroll
        for (int i = 0; i < U; ++i) {
          float v[V];
          unpack<T>(raw[i], v);
          take(v, place(b0, i));
        }
      }
    };
    if (sizeof(T) == 2 && ((uintptr_t)z & 2)) stream([](const T *p) { return load16_odd(p); });
    else stream([](const T *p) { return load16(p); });
    if (b0 < hi) {                              // what is left, in flight together too
      float v[U][V];
#pragma unroll
      for (int i = 0; i < U; ++i) load_vec(z + place(b0, i), hi - place(b0, i), kNegInf, v[i]);
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (place(b0, i) - lane * V < hi) take(v[i], place(b0, i));   // (whole waves)
    }
    wave_join(x, c);
    if (lane == 0) sh.sums[wave] = x.packed();
    __syncthreads();
    x = Sums(sh.sums[lane & (kWaves - 1)]);
    if (lane >= kWaves) x.s = x.u = 0.f;
    wave_join(x, c);
    if (a.parts == 1) {
      const Finish end(x, c);
      if (threadIdx.x == 0) end.row<T>(a, row, x, y, zy);
    } else if (threadIdx.x == 0) {
      a.part_sums[unit] = x.packed();
    }
    if constexpr (TOP) {
      const auto each = [&](uint32_t bar, auto f) {
        const auto vec = [&](int e0, int cnt) {
          float v[V];
          load_vec(z + e0, cnt, kNegInf, v);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const uint32_t o = order_of(v[e]);
            f(v[e] > kMasked && o >= bar ? ((uint64_t)o << 32) | (uint32_t)~(e0 + e) : 0);
          }
        };
        const auto reaches = [&](float m) { return m > kMasked && order_of(m) >= bar; };
        const bool all = reaches(mine.second);
        vec(mine.at, reaches(mine.first) && !all ? hi - mine.at : 0);
        // all vectors of a lane, one a lane
        for (uint64_t lanes = __ballot(all); lanes; lanes &= lanes - 1) {
          const int from = lo + (wave * 64 + __builtin_ctzll(lanes)) * V;
          for (int j0 = 0; from + j0 * kThreads * V < hi; j0 += 64) {
            const int e0 = from + (j0 + lane) * kThreads * V;
            vec(e0, hi - e0);
          }
        }
      };
      const Finish end(x, c);
      block_top(sh, a.top, mine.first, each, [&](int i, uint64_t key) {
        if (a.parts == 1) end.top(a, row, i, key);
        else a.part_top[((int64_t)row * a.parts + part) * a.top + i] = key;
      });
    }
    __syncthreads();                            // before the next unit's sums and keys
  }
}

// One workgroup a row: its parts' sums, a part a lane, and the parts' keys.
template <class T>
__global__ __launch_bounds__(kThreads) void token_logp_join_kernel(LogpArgs a) {
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, row = blockIdx.x;
  const float c = a.scale * kLog2e;
  int64_t y = -1;
  float zy = 0.f;
  if (threadIdx.x == 0 && a.logp) {
    y = a.targets[row];
    if (y >= 0 && y < a.vocab) zy = to_f32(((const T *)a.logits + (int64_t)row * a.row_stride)[y]);
  }
  const float4 f = a.part_sums[(int64_t)row * a.parts + min(lane, a.parts - 1)];
  constexpr int U = kLogpMaxParts * 64 / kThreads;   // most keys of a thread
  const int keys = a.parts * a.top;
  uint64_t key[U];
  float first = kNegInf;
  if (a.top > 0) {
    const uint64_t *from = a.part_top + (int64_t)row * keys;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      key[i] = at < keys ? from[at] : 0;
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) most = max(most, (uint32_t)(key[i] >> 32));
    if (most) first = value_of(most);
  }
  Sums x(f);
  if (lane >= a.parts) x.s = x.u = 0.f;
  wave_join(x, c);
  const Finish end(x, c);
  if (threadIdx.x == 0) end.row<T>(a, row, x, y, zy);
  if (a.top > 0)
    block_top(
        sh, a.top, first,
        [&](uint32_t bar, auto f) {
#pragma unroll
          for (int i = 0; i < U; ++i) f((uint32_t)(key[i] >> 32) >= bar ? key[i] : 0);
        },
        [&](int i, uint64_t k) { end.top(a, row, i, k); });
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
    const float nan = lse < -kNegInf ? 0.f : kNan;     // (without an lse there is no p)
    const float k0 = a.scale * (gs - gl - (ge != 0.f ? ge * a.entropy[row] : 0.f)) + nan;
    const float k1 = -a.scale * ge * kLn2, at_y = zero ? 0.f : a.scale * gl;
    const auto gradient = [&](const float (&v)[V], int e0, float (&o)[V]) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = (v[e] * a.scale - lse) * kLog2e;
        const float p = exp2_fast(fminf(d, 0.f));   // (of 2^24 and more, lse is rounded by whole numbers)
        o[e] = zero ? 0.f : p * (k0 + k1 * fmaxf(d, -200.f));
      }
      if ((uint32_t)(y - e0) < (uint32_t)V) {
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += y - e0 == e ? at_y : 0.f;
      }
    };
    const int first = chunk * (kThreads * V * kBwdVecs) + (int)threadIdx.x * V;
    float v[kBwdVecs][V];
#pragma unroll
    for (int r = 0; r < kBwdVecs; ++r) {
      const int e0 = first + r * kThreads * V;
      load_vec(z + e0, zero ? 0 : a.vocab - e0, kNegInf, v[r]);   // (a row without a gradient is not read)
    }
#pragma unroll
    for (int r = 0; r < kBwdVecs; ++r) {
      const int e0 = first + r * kThreads * V;
      float o[V];
      gradient(v[r], e0, o);
      store_vec(dz + e0, a.vocab - e0, o);
    }
  }
}

template <class T>
hipError_t fwd(LogpArgs a, hipStream_t s) {
  constexpr int V = kVec<T>;
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  a.part_len = plan::logp_part_len(a.vocab, a.parts, V);
  a.by_parts = FastDiv(a.parts);
  const int grid = (int)(units < kMaxGrid ? units : kMaxGrid);
  if (a.top > 0) token_logp_fwd_kernel<T, true><<<grid, kThreads, 0, s>>>(a);
  else token_logp_fwd_kernel<T, false><<<grid, kThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  token_logp_join_kernel<T><<<a.n_tokens, kThreads, 0, s>>>(a);
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

int token_logp_parts(int64_t n_tokens, int vocab) { return plan::logp_parts(n_tokens, vocab); }

hipError_t launch_token_logp_fwd(bool f32, const LogpArgs &a, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_token_logp_bwd(bool f32, const LogpBwdArgs &a, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace nsp
