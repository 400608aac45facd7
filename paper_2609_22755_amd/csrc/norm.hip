// Norms of rows (with and without the mean), forward and backward, for gfx950.
//
// Bound by HBM: the forward reads x and writes y, the backward reads x and dy
// and writes dx; some ten float32 operations an element are far below what
// the vector units do in that time.  A row stays in registers between its
// reductions, so memory is passed over once.
//
// A group of LPR lanes takes a row, CH vectors of 16 bytes a lane.  Up to 64
// lanes the sums stay within a wave; wider rows take several waves, which
// exchange their sums through LDS (one barrier a sum: the slots alternate).
// The columns of a lane are the same for all its rows, so the weights are
// loaded once, and the backward sums its part of dw and db in registers over
// the rows that a workgroup takes in turn; the workgroups' sums go to the
// workspace and a second kernel adds them, in the same order every time.
//
// 65536 x 8192 bf16 backward 555 us, 5.8 TB/s (two reads and a write: 5.8); 2 M
// heads of 128 264 us, 6.1; forward 5.8 to 6.1 TB/s; rows of 1111 float32 5.6,
// bf16 (every second one at an odd element) 4.4; 24 rows forward 4.5 us.  Heads of
// 64, half the lanes idle: forward 4.1, backward 4.3.
#include <type_traits>

#include "nsp_internal.hpp"
#include "row_common.hpp"

namespace nsp {
namespace {

template <class T>
__device__ __forceinline__ T *row_at(const RowView &v, const FastDiv &heads, int row) {
  const uint32_t t = heads.quot((uint32_t)row);
  return (T *)v.data + (int64_t)t * v.ts + (int64_t)((uint32_t)row - t * heads.d) * v.hs;
}

// V weights from element e0 on (all within the row).
template <int V>
__device__ __forceinline__ void load_weights(const void *w, bool f32, int e0, float none, float (&x)[V]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = none;
  } else if (f32) {
    struct __attribute__((packed, aligned(4))) W { float v[V]; } v = *(const W *)((const float *)w + e0);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = v.v[e];
  } else {
    struct __attribute__((packed, aligned(2))) W { unsigned short v[V]; } v = *(const W *)((const bf16 *)w + e0);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = __uint_as_float((uint32_t)v.v[e] << 16);
  }
}

// The same where only `cnt` lie within the row (the others: 0).
template <int V>
__device__ __forceinline__ void some_weights(const void *w, bool f32, int e0, int cnt, float none, float (&x)[V]) {
  if (!w || cnt >= V) return load_weights<V>(w, f32, e0, none, x);
#pragma unroll
  for (int e = 0; e < V; ++e)
    x[e] = e >= cnt ? 0.f : f32 ? ((const float *)w)[e0 + e] : to_f32(((const bf16 *)w)[e0 + e]);
}

// Threads of a workgroup, and the rows that it takes at a time.
template <int LPR>
constexpr int kBlock = LPR < 256 ? 256 : LPR;
template <int LPR>
constexpr int kGroups = kBlock<LPR> / LPR;

// The vectors of a lane: each starts at element e0, and its elements from `own`
// on are the lane's.  The last vector of a row that is no whole number of them
// reaches back over its neighbour's elements (both then store the same there:
// every lane has loaded before any stores), and a lane past the end holds the
// first vector of the row, with none of its own.
template <int LPR, int CH, int V>
struct Columns {
  int e0[CH], own[CH];
  bool some[CH];             // a lane of the wave does not own all of its vector
  __device__ __forceinline__ Columns(int n, int lane) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LPR + lane) * V;
      e0[c] = at + V <= n ? at : at < n ? n - V : 0;
      own[c] = at < n ? at - e0[c] : V;
      some[c] = __any(own[c] > 0);
    }
  }
};

// Sums of NV values over the LPR lanes of a row, in every one of them.
template <int LPR, int NV>
struct RowSum {
  static constexpr int W = LPR / 64;
  __device__ __forceinline__ static void run(float (&x)[NV], float *slots, int &turn) {
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = group_sum<(LPR < 64 ? 16 : 64)>(x[i]);
    if constexpr (LPR > 64) {
      float *s = slots + ((turn & 1) * kGroups<LPR> + threadIdx.x / LPR) * (W * NV);
      turn ^= 1;
      const int lane = threadIdx.x & 15, wave = (threadIdx.x % LPR) >> 6;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) s[wave * NV + i] = x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i) x[i] = group_sum<16>(lane < W ? s[lane * NV + i] : 0.f);
    }
  }
};

// A row's result, kept until the next row's turn: a store goes out before the
// loads of the row after that, whose arrival is then not waited for behind it
// (loads and stores retire in the order they were issued).  Rows of 128 bf16:
// 5.8 TB/s, 5.4 without.  (The backward has no registers left for it.)
template <class T, int LPR, int CH>
struct Done {
  T *row = nullptr;
  u32x4 v[CH];
  __device__ __forceinline__ void store(const Columns<LPR, CH, kVec<T>> &col) {
    if (!row) return;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (col.own[c] < kVec<T>) store16(row + col.e0[c], v[c]);
  }
};

template <class T, int LPR, int CH>
__global__ __launch_bounds__(kBlock<LPR>) void norm_fwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  constexpr int RPB = kGroups<LPR>;
  __shared__ float slots[2 * RPB * (LPR / 64 + 1)];
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  int turn = 0;
  const Columns<LPR, CH, V> col(a.n, lane);
  // a group past the end takes the last row once more and stores nothing
  u32x4 raw[CH];
  const auto fetch = [&](int64_t row0) {
    const T *x = row_at<const T>(a.x, a.heads, (int)min(row0 + group, (int64_t)a.rows - 1));
#pragma unroll
    for (int c = 0; c < CH; ++c) raw[c] = load16(x + col.e0[c]);
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row0 = (int64_t)blockIdx.x * RPB;
  fetch(row0);
  float w[CH][V], b[CH][V];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    load_weights<V>(a.w, a.w_f32, col.e0[c], 1.f, w[c]);
    load_weights<V>(a.b, a.w_f32, col.e0[c], 0.f, b[c]);
  }
  const float inv_n = 1.f / (float)a.n;
  Done<T, LPR, CH> done;
  for (; row0 < a.rows; row0 += step) {
    float v[CH][V];
#pragma unroll
    for (int c = 0; c < CH; ++c) unpack<T>(raw[c], v[c]);
    done.store(col);
    if (row0 + step < a.rows) fetch(row0 + step);
    float mean = 0.f;
    if (!a.rms) {
      float sum[1] = {0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (col.some[c]) {
#pragma unroll
          for (int e = 0; e < V; ++e) sum[0] += e >= col.own[c] ? v[c][e] : 0.f;
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) sum[0] += v[c][e];
        }
      }
      RowSum<LPR, 1>::run(sum, slots, turn);
      mean = sum[0] * inv_n;
    }
    float sq[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[c][e] -= mean;
      if (col.some[c]) {
#pragma unroll
        for (int e = 0; e < V; ++e) sq[0] += e >= col.own[c] ? v[c][e] * v[c][e] : 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) sq[0] += v[c][e] * v[c][e];
      }
    }
    RowSum<LPR, 1>::run(sq, slots, turn);
    const float rstd = rsqrtf(sq[0] * inv_n + a.eps);   // (the instruction alone takes subnormal variances for 0)
    const bool live = row0 + group < a.rows;
    const int row = live ? (int)row0 + group : a.rows - 1;
    done.row = live ? row_at<T>(a.y, a.heads, row) : nullptr;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = v[c][e] * rstd * w[c][e] + b[c][e];
      done.v[c] = pack<T>(o);
    }
    if (lane == 0 && live) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
  done.store(col);
}

// Sums of V columns over the strands of a workgroup (strand: the threads that
// share threadIdx.x / LANES) into out[i], i < LANES V: by shuffles within a
// wave, the waves in order.
template <int WAVES, int LANES, int V>
__device__ __forceinline__ void strand_sums(float (&s)[V], float (*lds)[LANES * V], float *out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int m = LANES; m < 64; m <<= 1) s[e] += __shfl_xor(s[e], m);
    if (lane < LANES) lds[wave][lane * V + e] = s[e];
  }
  __syncthreads();
  if (threadIdx.x < LANES * V) {
    float t = 0.f;
#pragma unroll
    for (int p = 0; p < WAVES; ++p) t += lds[p][threadIdx.x];
    *out = t;
  }
}

__device__ __forceinline__ void store_weight(void *out, bool f32, int c, float t) {
  if (f32) ((float *)out)[c] = t;
  else ((bf16 *)out)[c] = (bf16)t;
}

// dw, db straight from x and dy, by the workgroup `block` of those that do: 4 or
// 8 lanes' vectors of columns, the rows first .. last in strands of so many lanes.
// Where rows are few, the parts of a workgroup for each would be as much memory as
// the rows themselves, and a kernel more; where dx leaves x and dy alone, it is
// formed beside this.  PART: a part of the rows, left at `part`.
template <class T, int THREADS, bool PART = false>
__device__ __forceinline__ void norm_columns(const NormArgs &a, int block, uint32_t first, uint32_t last, float *part = nullptr) {
  constexpr int V = kVec<T>, LANES = THREADS > 256 ? 8 : 4, STRANDS = THREADS / LANES;
  __shared__ float lds[THREADS / 64][LANES * V];
  const int col = block * (LANES * V) + (threadIdx.x % LANES) * V, cnt = a.n - col;
  float dw[V] = {}, db[V] = {}, t;
  if (cnt > 0) {
#pragma unroll 8
    for (uint32_t row = first + threadIdx.x / LANES; row < last; row += STRANDS) {
      float x[V], g[V];
      load_vec_kept(row_at<const T>(a.x, a.heads, (int)row) + col, cnt, 0.f, x);
      load_vec_kept(row_at<const T>(a.dy, a.heads, (int)row) + col, cnt, 0.f, g);
      const float mean = a.rms ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dw[e] += g[e] * ((x[e] - mean) * rstd);
        db[e] += g[e];
      }
    }
  }
  const int c = block * (LANES * V) + threadIdx.x;
  const bool mine = threadIdx.x < LANES * V && c < a.n;
  if (a.dw) {
    strand_sums<THREADS / 64, LANES, V>(dw, lds, &t);
    if (mine) store_weight(PART ? part : a.dw, PART || a.w_f32, c, t);
  }
  if (a.db) {
    strand_sums<THREADS / 64, LANES, V>(db, lds, &t);
    if (mine) store_weight(PART ? part + a.n : a.db, PART || a.w_f32, c, t);
  }
}
template <class T, int THREADS>
int column_blocks(int n) {
  const int per = (THREADS > 256 ? 8 : 4) * kVec<T>;
  return (n + per - 1) / per;
}

// By all workgroups of a launch; PART: of `per` rows for each of its y.
template <class T, bool PART>
__global__ __launch_bounds__(1024) void norm_columns_kernel(NormArgs a, uint32_t per) {
  if constexpr (PART) {
    const uint32_t first = min(blockIdx.y * per, (uint32_t)a.rows);
    norm_columns<T, 1024, true>(a, blockIdx.x, first, min(first + per, (uint32_t)a.rows), a.part + (int64_t)blockIdx.y * 2 * a.n);
  } else {
    norm_columns<T, 1024>(a, blockIdx.x, 0, a.rows);
  }
}

// A row is kept as it was loaded until it is done: unpacking it twice is
// cheaper than the registers of its float32 form, which the next row's vectors,
// on their way meanwhile, take.
//
// COLUMNS: the first a.column_blocks workgroups form dw and db (a kernel of its
// own: with both in one, heads of 128 took 342 us instead of 265).
template <class T, int LPR, int CH, bool COLUMNS>
__global__ __launch_bounds__(kBlock<LPR>) void norm_bwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  constexpr int RPB = kGroups<LPR>;
  if constexpr (COLUMNS)
    if ((int)blockIdx.x < a.column_blocks) return norm_columns<T, kBlock<LPR>>(a, blockIdx.x, 0, a.rows);
  const int before = COLUMNS ? a.column_blocks : 0, block = (int)blockIdx.x - before, blocks = (int)gridDim.x - before;
  __shared__ float slots[2 * 2 * RPB * (LPR / 64 + 1)];
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  int turn = 0;
  const Columns<LPR, CH, V> col(a.n, lane);
  // a group past the end loads the last row once more, counts it as 0 and stores nothing
  struct Row {
    u32x4 x[CH], g[CH];
    float mean, rstd;
  };
  Row cur, next;
  const auto fetch = [&](int64_t row0, Row &r) {
    const bool live = row0 + group < a.rows;
    const int row = live ? (int)row0 + group : a.rows - 1;
    const T *x = row_at<const T>(a.x, a.heads, row), *dy = row_at<const T>(a.dy, a.heads, row);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      r.x[c] = load16(x + col.e0[c]);
      r.g[c] = load16(dy + col.e0[c]);
    }
    r.mean = a.rms ? 0.f : a.mean_in[row];
    r.rstd = a.rstd_in[row];
  };
  const int64_t step = (int64_t)blocks * RPB;
  int64_t row0 = (int64_t)block * RPB;
  // (1024 lanes have 128 registers each: no room for a row ahead, which spilled and
  // ran at 3.0 TB/s for float32 rows of 16384)
  constexpr bool AHEAD = LPR < 1024;
  if constexpr (AHEAD) fetch(row0, next);
  float w[CH][V], dw[CH][V], db[CH][V];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    load_weights<V>(a.w, a.w_f32, col.e0[c], 1.f, w[c]);
#pragma unroll
    for (int e = 0; e < V; ++e) dw[c][e] = db[c][e] = 0.f;
  }
  const float inv_n = 1.f / (float)a.n;
  for (; row0 < a.rows; row0 += step) {
    if constexpr (AHEAD) {
      cur = next;
      if (row0 + step < a.rows) fetch(row0 + step, next);
    } else {
      fetch(row0, cur);
    }
    const bool live = row0 + group < a.rows;
    if (RPB > 1 && !live) {
      cur.mean = cur.rstd = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c) cur.x[c] = cur.g[c] = u32x4{0, 0, 0, 0};
    }
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float xh[V], g[V];
      unpack<T>(cur.x[c], xh);
      unpack<T>(cur.g[c], g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        xh[e] = (xh[e] - cur.mean) * cur.rstd;
        dw[c][e] += g[e] * xh[e];
        db[c][e] += g[e];
        g[e] *= w[c][e];
      }
      if (col.some[c]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sums[0] += e >= col.own[c] ? g[e] : 0.f;
          sums[1] += e >= col.own[c] ? g[e] * xh[e] : 0.f;
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sums[0] += g[e];
          sums[1] += g[e] * xh[e];
        }
      }
    }
    RowSum<LPR, 2>::run(sums, slots, turn);
    const float m0 = a.rms ? 0.f : sums[0] * inv_n, m1 = sums[1] * inv_n;
    if (!live) continue;
    T *dx = row_at<T>(a.y, a.heads, (int)row0 + group);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float xh[V], g[V], o[V];
      // (or the compiler would keep what it unpacked before the barrier)
      asm volatile("" : "+v"(cur.x[c]), "+v"(cur.g[c]));
      unpack<T>(cur.x[c], xh);
      unpack<T>(cur.g[c], g);
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (g[e] * w[c][e] - m0 - (xh[e] - cur.mean) * cur.rstd * m1) * cur.rstd;
      if (col.own[c] < V) store16(dx + col.e0[c], pack<T>(o));
    }
  }
  if (!a.part) return;
  float *part = a.part + (int64_t)block * 2 * a.n;
  if constexpr (LPR < 64) {
    // sixteen groups: their sums in the order of the groups, an element a thread
    // (added up by the first group's lanes alone, heads of 128 took 319 us instead of 266)
    __shared__ float lds[256 * V];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) lds[group * (LPR * V) + lane * V + e] = k ? db[c][e] : dw[c][e];
        __syncthreads();
        for (int i = threadIdx.x; i < LPR * V; i += 256) {
          // element i of the group's vectors: of lane i / V, its own or not
          const int at = (c * LPR + i / V) * V, e0 = at + V <= a.n ? at : a.n - V, e = e0 + i % V;
          float s = 0.f;
#pragma unroll
          for (int g2 = 0; g2 < RPB; ++g2) s += lds[g2 * (LPR * V) + i];
          if (at < a.n && e >= at) part[k * a.n + e] = s;
        }
      }
    return;
  }
  // a few groups: the others' sums, added to the first one's in the order of the
  // groups (1000 x 4096 bf16 16.4 us; element by element as above 19.4)
  if constexpr (LPR >= 64 && RPB > 1) {
    __shared__ float lds[RPB - 1][CH * V * 2][LPR];
    if (group > 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          lds[group - 1][(c * V + e) * 2][lane] = dw[c][e];
          lds[group - 1][(c * V + e) * 2 + 1][lane] = db[c][e];
        }
    }
    __syncthreads();
    if (group > 0) return;
    for (int g = 0; g < RPB - 1; ++g)
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dw[c][e] += lds[g][(c * V + e) * 2][lane];
          db[c][e] += lds[g][(c * V + e) * 2 + 1][lane];
        }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float *to = part + col.e0[c];
    if (col.own[c] == 0) {
      typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        *(f32x4_any *)(to + e) = f32x4_any{dw[c][e], dw[c][e + 1], dw[c][e + 2], dw[c][e + 3]};
        *(f32x4_any *)(to + a.n + e) = f32x4_any{db[c][e], db[c][e + 1], db[c][e + 2], db[c][e + 3]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= col.own[c]) {
          to[e] = dw[c][e];
          to[a.n + e] = db[c][e];
        }
    }
  }
}

// Rows wider than the lanes of a workgroup hold (or less than a vector wide):
// several passes over a row, which is in the caches after the first (8192 x 20000
// bf16 forward 2.2 TB/s; backward with the launch for dw and db 1.4).
template <class T>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float slots[2 * 17];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = row_at<const T>(a.x, a.heads, (int)row);
    T *y = row_at<T>(a.y, a.heads, (int)row);
    float mean = 0.f;
    if (!a.rms) {
      float s[1] = {0.f};
      for (int i = threadIdx.x * V; i < a.n; i += 1024 * V) {
        float v[V];
        load_vec(x + i, a.n - i, 0.f, v);
#pragma unroll
        for (int e = 0; e < V; ++e) s[0] += v[e];
      }
      RowSum<1024, 1>::run(s, slots, turn);
      mean = s[0] / (float)a.n;
    }
    float sq[1] = {0.f};
    for (int i = threadIdx.x * V; i < a.n; i += 1024 * V) {
      float v[V];
      load_vec(x + i, a.n - i, mean, v);
#pragma unroll
      for (int e = 0; e < V; ++e) sq[0] += (v[e] - mean) * (v[e] - mean);
    }
    RowSum<1024, 1>::run(sq, slots, turn);
    const float rstd = rsqrtf(sq[0] / (float)a.n + a.eps);
    for (int i = threadIdx.x * V; i < a.n; i += 1024 * V) {
      float v[V], w[V], b[V];
      load_vec(x + i, a.n - i, 0.f, v);
      some_weights<V>(a.w, a.w_f32, i, a.n - i, 1.f, w);
      some_weights<V>(a.b, a.w_f32, i, a.n - i, 0.f, b);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = (v[e] - mean) * rstd * w[e] + b[e];
      store_vec(y + i, a.n - i, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T>
__global__ __launch_bounds__(1024) void norm_bwd_wide_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float slots[2 * 2 * 17];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = row_at<const T>(a.x, a.heads, (int)row), *dy = row_at<const T>(a.dy, a.heads, (int)row);
    T *dx = row_at<T>(a.y, a.heads, (int)row);
    const float mean = a.rms ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
    float sums[2] = {0.f, 0.f};
    float v[V], g[V], w[V];
    for (int i = threadIdx.x * V; i < a.n; i += 1024 * V) {
      load_vec(x + i, a.n - i, 0.f, v);
      load_vec(dy + i, a.n - i, 0.f, g);
      some_weights<V>(a.w, a.w_f32, i, a.n - i, 1.f, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = g[e] * w[e];
        sums[0] += h;
        sums[1] += h * ((v[e] - mean) * rstd);
      }
    }
    RowSum<1024, 2>::run(sums, slots, turn);
    const float m0 = a.rms ? 0.f : sums[0] / (float)a.n, m1 = sums[1] / (float)a.n;
    for (int i = threadIdx.x * V; i < a.n; i += 1024 * V) {
      load_vec(x + i, a.n - i, 0.f, v);
      load_vec(dy + i, a.n - i, 0.f, g);
      some_weights<V>(a.w, a.w_f32, i, a.n - i, 1.f, w);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = (g[e] * w[e] - m0 - (v[e] - mean) * rstd * m1) * rstd;
      store_vec(dx + i, a.n - i, v);
    }
  }
}

// dw, db: the sum of the workgroups' parts, 32 columns a workgroup, the parts
// in 128 strands.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *part, int parts, int n, void *dw, void *db, bool f32) {
  __shared__ float lds[16][32];
  const int which = blockIdx.y, col = blockIdx.x * 32 + (threadIdx.x & 7) * 4;
  void *out = which ? db : dw;
  if (!out) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, t;
  if (col < n) {
#pragma unroll 8
    for (int p = threadIdx.x >> 3; p < parts; p += 128) {
      float v[4];
      load_vec(part + ((int64_t)p * 2 + which) * n + col, n - col, 0.f, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
  }
  strand_sums<16, 8, 4>(s, lds, &t);
  const int c = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x < 32 && c < n) store_weight(out, f32, c, t);
}

// f(lanes, vectors) of the shape s among `shapes`, as compile-time numbers; false
// if it is none of them.
template <const auto &SHAPES, size_t I = 0, class F>
bool with_shape(plan::NormShape s, F f) {
  if constexpr (I < sizeof(SHAPES) / sizeof(SHAPES[0])) {
    if (s.lpr != SHAPES[I].lpr || s.ch != SHAPES[I].ch) return with_shape<SHAPES, I + 1>(s, f);
    f(std::integral_constant<int, SHAPES[I].lpr>(), std::integral_constant<int, SHAPES[I].ch>());
    return true;
  } else {
    return false;
  }
}

template <class T>
hipError_t fwd(const NormArgs &a, hipStream_t s) {
  constexpr bool f32 = sizeof(T) == 4;
  const plan::NormShape sh = plan::norm_fwd_shape(a.n, f32);
  const int grid = plan::norm_fwd_grid(a.rows, sh);
  const auto launch = [&](auto lpr, auto ch) {
    constexpr int L = decltype(lpr)::value, C = decltype(ch)::value;
    norm_fwd_kernel<T, L, C><<<grid, kBlock<L>, 0, s>>>(a);
  };
  bool known = true;
  if (sh.lpr == 0) norm_fwd_wide_kernel<T><<<grid, 1024, 0, s>>>(a);
  else if constexpr (f32) known = with_shape<plan::kNormFwdF32>(sh, launch);
  else known = with_shape<plan::kNormFwdBf16>(sh, launch);
  return known ? hipGetLastError() : hipErrorInvalidValue;
}

template <class T>
hipError_t bwd(const NormArgs &a, hipStream_t s) {
  constexpr bool f32 = sizeof(T) == 4;
  const plan::NormShape sh = plan::norm_bwd_shape(a.n, f32);
  const int parts = plan::norm_parts(a.rows, a.n, f32);
  const bool columns = (a.dw || a.db) && parts == 0;
  hipError_t e = hipSuccess;
  NormArgs b = a;
  if (parts == 0) b.part = nullptr;
  if ((a.dw || a.db) && (a.rows == 0 || sh.lpr == 0)) {   // (before dx, which may lie over x or dy)
    const int strips = column_blocks<T, 1024>(a.n);
    if (b.part) norm_columns_kernel<T, true><<<dim3(strips, parts), 1024, 0, s>>>(b, ((uint32_t)a.rows + parts - 1) / parts);
    else norm_columns_kernel<T, false><<<strips, 1024, 0, s>>>(b, 0);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.rows == 0) return e;
  const int grid = plan::norm_bwd_grid(a.rows, sh, b.part ? parts : 0);
  const auto launch = [&](auto lpr, auto ch) {
    constexpr int L = decltype(lpr)::value, C = decltype(ch)::value;
    b.column_blocks = columns ? column_blocks<T, kBlock<L>>(a.n) : 0;
    // dw and db read what dx in place would overwrite: by a launch of their own, before
    if (columns && (a.y.data == a.x.data || a.y.data == a.dy.data)) {
      norm_bwd_kernel<T, L, C, true><<<b.column_blocks, kBlock<L>, 0, s>>>(b);
      b.column_blocks = 0;
    }
    if (b.column_blocks > 0) norm_bwd_kernel<T, L, C, true><<<grid + b.column_blocks, kBlock<L>, 0, s>>>(b);
    else norm_bwd_kernel<T, L, C, false><<<grid, kBlock<L>, 0, s>>>(b);
  };
  bool known = true;
  if (sh.lpr == 0) norm_bwd_wide_kernel<T><<<grid, 1024, 0, s>>>(b);
  else if constexpr (f32) known = with_shape<plan::kNormBwdF32>(sh, launch);
  else known = with_shape<plan::kNormBwdBf16>(sh, launch);
  e = known ? hipGetLastError() : hipErrorInvalidValue;
  if (e == hipSuccess && b.part) {
    norm_weight_kernel<<<dim3((a.n + 31) / 32, 2), 1024, 0, s>>>(a.part, parts, a.n, a.dw, a.db, a.w_f32);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

int norm_bwd_parts(int64_t rows, int n, bool f32) { return plan::norm_parts(rows, n, f32); }

hipError_t launch_norm_fwd(bool f32, const NormArgs &a, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_norm_bwd(bool f32, const NormArgs &a, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace nsp
