// The loss of a row of logits against a teacher's top alternatives, and its
// gradient, for gfx950.
//
//     q_k = exp(t_k - c),   loss = sum_k q_k (t_k - c - (z_ik - lse))
//     dz_v = scale g (S p_v - sum of the q_k with i_k = v),   S = sum_k q_k
//
// Bound by HBM: the forward reads the logits once, the backward reads and writes
// them once; what the alternatives cost (12 bytes and a few operations each) has to
// hide behind that.  bf16, 4096 x 151643 with 64 alternatives: 192 us (6.5 TB/s);
// backward 8192 x 131072 with 64: 693 (6.2).
//
// Forward: the running sums of the log probabilities' pass (logit_sums.hpp)
// without its weighted one; a workgroup takes a row, or a part of one where there
// are few, and ends it with one alternative a thread.
//
// Backward: a workgroup takes 16 to 64 KB of a row, 16 KB at a time: more of them
// weigh the alternatives more often, and stream better.  The first vectors
// are on their way while every wave weighs the alternatives for itself (no
// barrier before the sums); all are stored as if there were no alternatives, and
// after a barrier the threads whose alternative lies in this part store its element
// anew, each token once with all the weight that it has.
#include "logit_sums.hpp"
#include "vocab_internal.hpp"

namespace nsp {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxGrid = 1 << 22;
constexpr int kPerLane = kDistillMaxTop / 64;   // alternatives of a lane

// An alternative as it counts: its token, -1 if it is none, and its value.
struct Alternative {
  int at = -1;
  float t = kNegInf;
  __device__ __forceinline__ Alternative() {}
  __device__ __forceinline__ Alternative(const DistillArgs &a, int64_t row, int k) {
    const int64_t i = a.index[row * a.top + k];
    t = a.teacher[row * a.top + k];
    if (!(t < -kNegInf)) t = kNan;              // (+inf is no log probability)
    if (i >= 0 && i < a.vocab && !(t <= kMasked)) at = (int)i;
    else t = kNegInf;
  }
  __device__ __forceinline__ float weight(float c) const { return at >= 0 ? exp2_fast((t - c) * kLog2e) : 0.f; }
};

// A row's alternatives, all of them in every wave.
struct Weighed {
  float c = 0.f, sum = 0.f;    // c, S
  bool any;
  __device__ __forceinline__ Weighed(const DistillArgs &a, int64_t row) {
    const int lane = threadIdx.x & 63;
    Alternative x[kPerLane];
    bool mine = false;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
      if (64 * j < a.top && 64 * j + lane < a.top) {
        x[j] = Alternative(a, row, 64 * j + lane);
        mine |= x[j].at >= 0;
      }
    any = __any(mine);
    if (a.normalized && any) {
      float most = kNegInf, s = 0.f;
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) most = fmaxf(most, x[j].t);   // (a NaN comes through the sum)
      most = fmaxf(wave_max(most), -0x1p126f);
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) s += x[j].weight(most);
      c = most + log2f(group_sum<64>(s)) * kLn2;
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) s += x[j].weight(c);
    sum = group_sum<64>(s);
  }
};

// ----------------------------------------------------------------- forward --

struct Shared {
  float4 sums[kWaves];
  float loss[kWaves];
};

// What a row comes to, from its sums (in every thread); by the whole workgroup.
template <class T>
__device__ __forceinline__ void finish(const DistillArgs &a, int row, const Sums &x, Shared &sh) {
#pragma clang fp contract(off)
  const float c = a.scale * kLog2e;
  const float r = x.m * c;
  const bool none = x.s == 0.f;
  const float log_s = fabsf(r) < -kNegInf ? log2f(x.s) : kNan;
  const Weighed w(a, row);
  float loss = 0.f;
  if ((int)threadIdx.x < a.top) {
    const Alternative t(a, row, threadIdx.x);
    if (t.at >= 0) {
      const float z = to_f32(((const T *)a.logits + (int64_t)row * a.row_stride)[t.at]);
      const float q = t.weight(w.c);
      // of the logits' differences where the reference is rounded by whole numbers
      const float lp = none || z <= kMasked ? kNegInf : ((is_far(r) ? (z - x.m) * c : __builtin_fmaf(z, c, -r)) - log_s) * kLn2;
      loss = !none && log_s != log_s ? kNan : q == 0.f ? 0.f : q * ((t.t - w.c) - lp);
    }
  }
  loss = group_sum<64>(loss);
  if ((threadIdx.x & 63) == 0) sh.loss[threadIdx.x >> 6] = loss;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.lse[row] = none ? kNegInf : (r + log_s) * kLn2;
    if (a.loss) a.loss[row] = w.any ? (sh.loss[0] + sh.loss[1]) + (sh.loss[2] + sh.loss[3]) : 0.f;
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_fwd_kernel(DistillArgs a) {
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
    Sums x(c);
    bool far = true;
    const auto take = [&](const float (&v)[V]) {
      float most = max3(v[0], v[1], v[2]);
#pragma unroll
      for (int e = 3; e < V; e += 2) most = max3(most, v[e], v[e + 1 < V ? e + 1 : e]);
      const bool up = (far ? (most - x.m) * c : fmaf(most, c, -x.r)) > 16.f;
      if (__ballot(up)) {
        x.move(up ? most : x.m, up ? most * c : x.r, c);
        far = __any(is_far(x.r));
      }
      if (far) {
#pragma unroll
        for (int e = 0; e < V; ++e) x.s += exp2_fast((v[e] - x.m) * c);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x.s += exp2_fast(fmaf(v[e], c, -x.r));
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
          take(v);
        }
      }
    };
    if (sizeof(T) == 2 && ((uintptr_t)z & 2)) stream([](const T *p) { return load16_odd(p); });
    else stream([](const T *p) { return load16(p); });
    if (b0 < hi) {
      float v[U][V];
#pragma unroll
      for (int i = 0; i < U; ++i) load_vec(z + place(b0, i), hi - place(b0, i), kNegInf, v[i]);
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (place(b0, i) - lane * V < hi) take(v[i]);   // (whole waves)
    }
    wave_join(x, c);
    if (lane == 0) sh.sums[wave] = x.packed();
    __syncthreads();
    x = Sums(sh.sums[lane & (kWaves - 1)]);
    if (lane >= kWaves) x.s = x.u = 0.f;
    wave_join(x, c);
    if (a.parts == 1) finish<T>(a, row, x, sh);
    else if (threadIdx.x == 0) a.part_sums[unit] = x.packed();
    __syncthreads();                            // before the next unit's sums
  }
}

// One workgroup a row: its parts' sums, a part a lane.
template <class T>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(DistillArgs a) {
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, row = blockIdx.x;
  const float c = a.scale * kLog2e;
  Sums x(a.part_sums[(int64_t)row * a.parts + min(lane, a.parts - 1)]);
  if (lane >= a.parts) x.s = x.u = 0.f;
  wave_join(x, c);
  finish<T>(a, row, x, sh);
}

// ---------------------------------------------------------------- backward --

constexpr int kBwdVecs = 4;    // vectors of a lane in flight

// TURNS: times that a workgroup takes as many.
template <class T, int TURNS>
__global__ __launch_bounds__(kThreads) void distill_bwd_kernel(DistillArgs a, int parts) {
  constexpr int V = kVec<T>, kTurn = kThreads * V * kBwdVecs, kPart = kTurn * TURNS;
  __shared__ int4 at[kDistillMaxTop / 4];
  __shared__ float4 q[kDistillMaxTop / 4];
  static_assert(kDistillMaxTop == kThreads, "an alternative a thread");
  const int64_t units = (int64_t)a.n_tokens * parts;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int row = (int)(unit / parts), part = (int)(unit - (int64_t)row * parts);
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    T *dz = (T *)a.dlogits + (int64_t)row * a.d_row_stride;
    const float g = a.g_loss[row], lse = a.lse_in[row];
    const bool still = lse == kNegInf || g == 0.f;
    const int64_t from = (int64_t)part * kPart;
    const int lo = (int)from, hi = (int)min((int64_t)a.vocab, from + kPart);
    u32x4 raw[kBwdVecs];
    const auto fetch = [&](int base) {             // (a row without a gradient is not read)
#pragma unroll
      for (int r = 0; r < kBwdVecs; ++r) {
        const int e0 = base + (r * kThreads + (int)threadIdx.x) * V;
        if (!still && e0 + V <= hi) raw[r] = load16(z + e0);
      }
    };
    fetch(lo);
    const Weighed w(a, row);
    const bool zero = still || !w.any;
    const float nan = lse < -kNegInf ? 0.f : kNan, gs = a.scale * g, k0 = gs * w.sum + nan;
    const auto slope = [&](float v) {
      const float d = (v * a.scale - lse) * kLog2e;
      return exp2_fast(fminf(d, 0.f)) * k0;
    };
    Alternative mine;
    float zk = 0.f;
    if ((int)threadIdx.x < a.top) mine = Alternative(a, row, threadIdx.x);
    ((int *)at)[threadIdx.x] = mine.at;
    ((float *)q)[threadIdx.x] = mine.weight(w.c);
    if ((int)threadIdx.x < a.top) {
      if (mine.at < lo || mine.at >= hi || zero) mine.at = -1;
      if (mine.at >= 0) zk = to_f32(z[mine.at]);   // (before it may be overwritten)
    }
    __syncthreads();
    float weight = 0.f;
    if (mine.at >= 0) {
      bool first = true;
      for (int k = 0; k < a.top; k += 4) {
        const int4 i = at[k / 4];
        const float4 x = q[k / 4];
        weight += i.x == mine.at ? x.x : 0.f;
        weight += i.y == mine.at ? x.y : 0.f;
        weight += i.z == mine.at ? x.z : 0.f;
        weight += i.w == mine.at ? x.w : 0.f;
        const int before = (int)threadIdx.x - k;
        first &= !((i.x == mine.at && before > 0) || (i.y == mine.at && before > 1) || (i.z == mine.at && before > 2) ||
                   (i.w == mine.at && before > 3));
      }
      if (!first) mine.at = -1;                    // the first of them stores
    }
    for (int base = lo; base < hi; base += kTurn) {
      u32x4 now[kBwdVecs];
#pragma unroll
      for (int r = 0; r < kBwdVecs; ++r) now[r] = raw[r];
      if (base + kTurn < hi) fetch(base + kTurn);
#pragma unroll
      for (int r = 0; r < kBwdVecs; ++r) {
        const int e0 = base + (r * kThreads + (int)threadIdx.x) * V;
        if (e0 + V <= hi) {
          float v[V];
          unpack<T>(now[r], v);
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = slope(v[e]);
          u32x4 o = pack<T>(v);
          if (zero) o = u32x4{};
          store16(dz + e0, o);
        } else if (e0 < hi) {                      // the row's end
          for (int e = e0; e < hi; ++e) dz[e] = zero ? (T)0.f : (T)slope(to_f32(z[e]));
        }
      }
    }
    __syncthreads();
    if (mine.at >= 0) dz[mine.at] = (T)(slope(zk) - gs * weight);
  }
}

template <class T>
hipError_t fwd(DistillArgs a, hipStream_t s) {
  const int64_t units = (int64_t)a.n_tokens * a.parts;
  a.part_len = plan::logp_part_len(a.vocab, a.parts, kVec<T>);
  a.by_parts = FastDiv(a.parts);
  distill_fwd_kernel<T><<<(int)(units < kMaxGrid ? units : kMaxGrid), kThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  distill_join_kernel<T><<<a.n_tokens, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class T, int TURNS>
hipError_t bwd_turns(const DistillArgs &a, hipStream_t s) {
  const int parts = (int)plan::ceil_div(a.vocab, kThreads * kVec<T> * kBwdVecs * TURNS);
  const int64_t units = (int64_t)a.n_tokens * parts;
  distill_bwd_kernel<T, TURNS><<<(int)(units < kMaxGrid ? units : kMaxGrid), kThreads, 0, s>>>(a, parts);
  return hipGetLastError();
}

template <class T>
hipError_t bwd(const DistillArgs &a, hipStream_t s) {
  // (us at one, two and four turns. 8192 x 131072 bf16, 8 alternatives: 679, 691, 742;
  // 20: 700, 680, 736; 64: 760, 692, 738; 256: 1413, 878, 809.  777 x 50021 float32, 20:
  // 55, 57, 65; 64: 59, 62, 68; 256: 108, 80, 84.  Of few rows the weighing of the alternatives is
  // the time, and their number alone may decide: 24 x 131072 bf16 at one turn and as here, 64: 7.4
  // and 7.8; 256: 16.1 and 17.4; one row, 256: 17.4 and 16.6)
  return a.top * kVec<T> <= 128 ? bwd_turns<T, 1>(a, s) : a.top <= 128 ? bwd_turns<T, 2>(a, s) : bwd_turns<T, 4>(a, s);
}

}  // namespace

hipError_t launch_distill_fwd(bool f32, const DistillArgs &a, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_distill_bwd(bool f32, const DistillArgs &a, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace nsp
