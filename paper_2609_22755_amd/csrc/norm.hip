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
#include "nsp_internal.hpp"
#include "row_common.hpp"

namespace nsp {
namespace {

template <class T>
__device__ __forceinline__ T *row_at(const RowView &v, const FastDiv &heads, int row) {
  const uint32_t t = heads.quot((uint32_t)row);
  return (T *)v.data + (int64_t)t * v.ts + (int64_t)((uint32_t)row - t * heads.d) * v.hs;
}

// Weights of the elements e0 .. e0 + V - 1 (cnt of them within the row).
template <int V>
__device__ __forceinline__ void load_weights(const void *w, bool f32, int e0, int cnt, float none, float (&x)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) x[e] = none;
  if (!w) return;
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < cnt) x[e] = f32 ? ((const float *)w)[e0 + e] : to_f32(((const bf16 *)w)[e0 + e]);
}

// Sums of NV values over the LPR lanes of a row, in every one of them.
template <int LPR, int NV>
struct RowSum {
  static constexpr int W = LPR / 64;
  __device__ __forceinline__ static void run(float (&x)[NV], float *slots, int &turn) {
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = group_sum<(LPR < 64 ? LPR : 64)>(x[i]);
    if constexpr (LPR > 64) {
      float *s = slots + (turn & 1) * (W * NV);
      turn ^= 1;
      const int lane = threadIdx.x & 63, wave = (threadIdx.x % LPR) >> 6;
      if (lane == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) s[wave * NV + i] = x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        // every wave adds the W sums the same way
        float v = lane < W ? s[lane * NV + i] : 0.f;
        v = group_sum<(W < 2 ? 2 : W)>(v);
        x[i] = __shfl(v, 0);
      }
    }
  }
};

template <class T, int LPR, int CH>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void norm_fwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  constexpr int RPB = LPR < 256 ? 256 / LPR : 1;
  __shared__ float slots[2 * (LPR / 64 + 1)];
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  int turn = 0;
  float w[CH][V], b[CH][V];
  int cnt[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int e0 = (c * LPR + lane) * V;
    cnt[c] = min(V, max(0, a.n - e0));
    load_weights<V>(a.w, a.w_f32, e0, cnt[c], 1.f, w[c]);
    load_weights<V>(a.b, a.w_f32, e0, cnt[c], 0.f, b[c]);
  }
  const float inv_n = 1.f / (float)a.n;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const bool live = row0 + group < a.rows;         // (a group past the end repeats the last row and stores nothing)
    const int row = live ? (int)row0 + group : a.rows - 1;
    const T *x = row_at<const T>(a.x, a.heads, row);
    float v[CH][V];
    float sum[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      load_vec(x + (c * LPR + lane) * V, cnt[c], 0.f, v[c]);
#pragma unroll
      for (int e = 0; e < V; ++e) sum[0] += v[c][e];
    }
    float mean = 0.f;
    if (!a.rms) {
      RowSum<LPR, 1>::run(sum, slots, turn);
      mean = sum[0] * inv_n;
    }
    float sq[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = e < cnt[c] ? v[c][e] - mean : 0.f;
        v[c][e] = d;
        sq[0] += d * d;
      }
    RowSum<LPR, 1>::run(sq, slots, turn);
    const float rstd = 1.f / sqrtf(sq[0] * inv_n + a.eps);
    if (!live) continue;
    T *y = row_at<T>(a.y, a.heads, row);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = v[c][e] * rstd * w[c][e] + b[c][e];
      store_vec(y + (c * LPR + lane) * V, cnt[c], o);
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T, int LPR, int CH>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void norm_bwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  constexpr int RPB = LPR < 256 ? 256 / LPR : 1;
  __shared__ float slots[2 * 2 * (LPR / 64 + 1)];
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  int turn = 0;
  float w[CH][V], dw[CH][V], db[CH][V];
  int cnt[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int e0 = (c * LPR + lane) * V;
    cnt[c] = min(V, max(0, a.n - e0));
    load_weights<V>(a.w, a.w_f32, e0, cnt[c], 1.f, w[c]);
#pragma unroll
    for (int e = 0; e < V; ++e) dw[c][e] = db[c][e] = 0.f;
  }
  const float inv_n = 1.f / (float)a.n;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const bool live = row0 + group < a.rows;
    const int row = live ? (int)row0 + group : a.rows - 1;
    const T *x = row_at<const T>(a.x, a.heads, row), *dy = row_at<const T>(a.dy, a.heads, row);
    const float mean = a.rms ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
    float xh[CH][V], g[CH][V];
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      load_vec(x + (c * LPR + lane) * V, cnt[c], mean, xh[c]);
      load_vec(dy + (c * LPR + lane) * V, live ? cnt[c] : 0, 0.f, g[c]);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        xh[c][e] = (xh[c][e] - mean) * rstd;
        dw[c][e] += g[c][e] * xh[c][e];
        db[c][e] += g[c][e];
        g[c][e] *= w[c][e];
        sums[0] += g[c][e];
        sums[1] += g[c][e] * xh[c][e];
      }
    RowSum<LPR, 2>::run(sums, slots, turn);
    if (!live) continue;
    const float m0 = a.rms ? 0.f : sums[0] * inv_n, m1 = sums[1] * inv_n;
    T *dx = row_at<T>(a.y, a.heads, row);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (g[c][e] - m0 - xh[c][e] * m1) * rstd;
      store_vec(dx + (c * LPR + lane) * V, cnt[c], o);
    }
  }
  if (!a.part) return;
  float *part = a.part + (int64_t)blockIdx.x * 2 * a.n;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e0 = (c * LPR + lane) * V;
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < cnt[c]) {
          part[e0 + e] = dw[c][e];
          part[a.n + e0 + e] = db[c][e];
        }
    }
  } else {
    // the groups' sums, added in the order of the groups
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
          const int e0 = c * LPR * V + i;
          float s = 0.f;
#pragma unroll
          for (int g2 = 0; g2 < RPB; ++g2) s += lds[g2 * (LPR * V) + i];
          if (e0 < a.n) part[k * a.n + e0] = s;
        }
      }
  }
}

// Rows wider than the lanes of a workgroup hold: several passes over a row,
// which is in the caches after the first.
template <class T>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(NormArgs a) {
  __shared__ float slots[2 * 17];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = row_at<const T>(a.x, a.heads, (int)row);
    T *y = row_at<T>(a.y, a.heads, (int)row);
    float mean = 0.f;
    if (!a.rms) {
      float s[1] = {0.f};
      for (int i = threadIdx.x; i < a.n; i += 1024) s[0] += to_f32(x[i]);
      RowSum<1024, 1>::run(s, slots, turn);
      mean = s[0] / (float)a.n;
    }
    float sq[1] = {0.f};
    for (int i = threadIdx.x; i < a.n; i += 1024) {
      const float d = to_f32(x[i]) - mean;
      sq[0] += d * d;
    }
    RowSum<1024, 1>::run(sq, slots, turn);
    const float rstd = 1.f / sqrtf(sq[0] / (float)a.n + a.eps);
    for (int i = threadIdx.x; i < a.n; i += 1024) {
      float w[1], b[1];
      load_weights<1>(a.w, a.w_f32, i, 1, 1.f, w);
      load_weights<1>(a.b, a.w_f32, i, 1, 0.f, b);
      y[i] = (T)((to_f32(x[i]) - mean) * rstd * w[0] + b[0]);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T>
__global__ __launch_bounds__(1024) void norm_bwd_wide_kernel(NormArgs a) {
  __shared__ float slots[2 * 2 * 17];
  int turn = 0;
  float *part = a.part ? a.part + (int64_t)blockIdx.x * 2 * a.n : nullptr;
  bool first = true;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = row_at<const T>(a.x, a.heads, (int)row), *dy = row_at<const T>(a.dy, a.heads, (int)row);
    T *dx = row_at<T>(a.y, a.heads, (int)row);
    const float mean = a.rms ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
    float sums[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < a.n; i += 1024) {
      float w[1];
      load_weights<1>(a.w, a.w_f32, i, 1, 1.f, w);
      const float h = to_f32(dy[i]) * w[0];
      sums[0] += h;
      sums[1] += h * ((to_f32(x[i]) - mean) * rstd);
    }
    RowSum<1024, 2>::run(sums, slots, turn);
    const float m0 = a.rms ? 0.f : sums[0] / (float)a.n, m1 = sums[1] / (float)a.n;
    for (int i = threadIdx.x; i < a.n; i += 1024) {
      float w[1];
      load_weights<1>(a.w, a.w_f32, i, 1, 1.f, w);
      const float g = to_f32(dy[i]), xh = (to_f32(x[i]) - mean) * rstd;
      if (part) {                                    // (this thread's own columns: no other reads or writes them)
        part[i] = g * xh + (first ? 0.f : part[i]);
        part[a.n + i] = g + (first ? 0.f : part[a.n + i]);
      }
      dx[i] = (T)((g * w[0] - m0 - xh * m1) * rstd);
    }
    first = false;
  }
}

// dw, db: the sum of the workgroups' parts, 32 columns a workgroup, the parts
// in 32 strands that are then added in order.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *part, int parts, int n, void *dw, void *db, bool f32) {
  __shared__ float lds[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), strand = threadIdx.x >> 5, which = blockIdx.y;
  float s = 0.f;
  if (col < n)
    for (int p = strand; p < parts; p += 32) s += part[((int64_t)p * 2 + which) * n + col];
  lds[strand][threadIdx.x & 31] = s;
  __syncthreads();
  if (threadIdx.x >= 32 || col >= n) return;
  s = 0.f;
#pragma unroll
  for (int p = 0; p < 32; ++p) s += lds[p][threadIdx.x];
  void *out = which ? db : dw;
  if (!out) return;
  if (f32) ((float *)out)[col] = s;
  else ((bf16 *)out)[col] = (bf16)s;
}

// Lanes of a row, and its vectors a lane; 0 lanes: the wide kernels.  1024
// lanes hold 16 elements each (four waves a SIMD leave 128 registers a lane,
// and the backward wants six an element).
struct NormShape {
  int lpr, ch;
};

NormShape norm_shape(int n, bool f32) {
  const int v = f32 ? 4 : 8, vecs = (n + v - 1) / v;
  for (int lpr : {16, 64, 256, 1024})
    for (int ch : {1, 2, 4})
      if (lpr * ch >= vecs && (lpr < 1024 || ch * v <= 16)) return {lpr, ch};
  return {0, 0};
}

template <class T, int LPR>
void launch_fwd(int ch, int grid, const NormArgs &a, hipStream_t s) {
  constexpr int threads = LPR < 256 ? 256 : LPR;
  if (ch == 1) norm_fwd_kernel<T, LPR, 1><<<grid, threads, 0, s>>>(a);
  else if (ch == 2) norm_fwd_kernel<T, LPR, 2><<<grid, threads, 0, s>>>(a);
  else if constexpr (LPR < 1024 || sizeof(T) == 4) norm_fwd_kernel<T, LPR, 4><<<grid, threads, 0, s>>>(a);
}

template <class T, int LPR>
void launch_bwd(int ch, int grid, const NormArgs &a, hipStream_t s) {
  constexpr int threads = LPR < 256 ? 256 : LPR;
  if (ch == 1) norm_bwd_kernel<T, LPR, 1><<<grid, threads, 0, s>>>(a);
  else if (ch == 2) norm_bwd_kernel<T, LPR, 2><<<grid, threads, 0, s>>>(a);
  else if constexpr (LPR < 1024 || sizeof(T) == 4) norm_bwd_kernel<T, LPR, 4><<<grid, threads, 0, s>>>(a);
}

template <class T>
hipError_t fwd(const NormArgs &a, hipStream_t s) {
  const NormShape sh = norm_shape(a.n, sizeof(T) == 4);
  const int rpb = sh.lpr > 0 && sh.lpr < 256 ? 256 / sh.lpr : 1;
  int64_t grid = ((int64_t)a.rows + rpb - 1) / rpb;
  if (grid > 4096) grid = 4096;
  switch (sh.lpr) {
    case 16: launch_fwd<T, 16>(sh.ch, (int)grid, a, s); break;
    case 64: launch_fwd<T, 64>(sh.ch, (int)grid, a, s); break;
    case 256: launch_fwd<T, 256>(sh.ch, (int)grid, a, s); break;
    case 1024: launch_fwd<T, 1024>(sh.ch, (int)grid, a, s); break;
    default: norm_fwd_wide_kernel<T><<<(int)grid, 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <class T>
hipError_t bwd(const NormArgs &a, hipStream_t s) {
  int parts = 0;
  if (a.rows > 0) {
    const NormShape sh = norm_shape(a.n, sizeof(T) == 4);
    parts = norm_bwd_parts(a.rows, a.n, sizeof(T) == 4);
    switch (sh.lpr) {
      case 16: launch_bwd<T, 16>(sh.ch, parts, a, s); break;
      case 64: launch_bwd<T, 64>(sh.ch, parts, a, s); break;
      case 256: launch_bwd<T, 256>(sh.ch, parts, a, s); break;
      case 1024: launch_bwd<T, 1024>(sh.ch, parts, a, s); break;
      default: norm_bwd_wide_kernel<T><<<parts, 1024, 0, s>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dw || a.db) {
    norm_weight_kernel<<<dim3((a.n + 31) / 32, 2), 1024, 0, s>>>(a.part, parts, a.n, a.dw, a.db, a.w_f32);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

int norm_bwd_parts(int64_t rows, int n, bool f32) {
  const NormShape sh = norm_shape(n, f32);
  const int rpb = sh.lpr > 0 && sh.lpr < 256 ? 256 / sh.lpr : 1;
  const int64_t groups = (rows + rpb - 1) / rpb;
  const int most = sh.lpr == 0 || sh.lpr == 1024 ? kNormMaxParts / 4 : kNormMaxParts;
  return (int)(groups < most ? groups : most);
}

hipError_t launch_norm_fwd(bool f32, const NormArgs &a, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_norm_bwd(bool f32, const NormArgs &a, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace nsp
