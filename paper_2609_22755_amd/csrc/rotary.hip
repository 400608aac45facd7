// Rotary positions of query and key heads for gfx950.
//
// Bound by HBM: every element is read and written once (2 x 2 bytes of bf16
// for 3 multiply-adds).  What could cost more is the angles: a sine and a
// cosine in float32, of an angle that is reduced to a turn in 64 bits, are
// worth some 60 instructions, as much as memory gives time for in two vectors
// of eight elements.  A token's angles are the same for all its heads, so a
// workgroup takes a few whole tokens, forms their (cos, sin) once, in LDS, and
// then turns all heads of these tokens with them.
//
// A task is one vector (16 bytes) of each half of a head, or one vector of
// neighbouring pairs; the unrotated rest of a head is copied by tasks of one
// vector (none in place).
#include "nsp_internal.hpp"
#include "row_common.hpp"

namespace nsp {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = 1 << 22;   // workgroups of a launch (its threads stay below 2^32)

struct RotaryShape {
  int tokens;                // of a workgroup
  int rot_tasks, row_tasks;  // of a head row: rotated, all
  FastDiv half, row, token;  // pairs of a token, tasks of a row, rows of a token
};

template <class T, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryShape sh) {
  extern __shared__ float2 turn[];   // [token][pair]
  constexpr int V = kVec<T>;
  for (int64_t t0 = (int64_t)blockIdx.x * sh.tokens; t0 < a.n_tokens; t0 += (int64_t)gridDim.x * sh.tokens) {
    const int nt = (int)min((int64_t)sh.tokens, a.n_tokens - t0);
    for (int i = threadIdx.x; i < nt * a.half; i += kThreads) {
      const int tl = sh.half.quot(i), p = i - tl * a.half;
      const double angle = (double)a.positions[t0 + tl] * a.freqs[p];
      const double turns = angle * 0.15915494309189533576888376337251;   // 1 / (2 pi)
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      turn[i] = make_float2(c * a.scale, s * (a.scale * a.sign));
    }
    __syncthreads();

    const int rows = a.heads[0] + a.heads[1];
    const int total = nt * rows * sh.row_tasks;
    for (int i = threadIdx.x; i < total; i += kThreads) {
      const int r = sh.row.quot(i), c = i - r * sh.row_tasks;
      const int tl = sh.token.quot(r);
      int h = r - tl * rows;
      const int kind = h >= a.heads[0];
      h -= kind ? a.heads[0] : 0;
      const RowView xv = kind ? a.x[1] : a.x[0], yv = kind ? a.y[1] : a.y[0];
      const T *x = (const T *)xv.data + (t0 + tl) * xv.ts + h * xv.hs;
      T *y = (T *)yv.data + (t0 + tl) * yv.ts + h * yv.hs;
      if (c >= sh.rot_tasks) {
        if (!(kind ? a.copy[1] : a.copy[0])) continue;
        const int e0 = 2 * a.half + (c - sh.rot_tasks) * V, cnt = a.head_dim - e0;
        if (cnt >= V) {
          store16(y + e0, load16(x + e0));
        } else {
          for (int e = 0; e < cnt; ++e) y[e0 + e] = x[e0 + e];
        }
        continue;
      }
      const float2 *cs = turn + tl * a.half;
      if constexpr (PAIRS) {
        const int e0 = c * V, cnt = 2 * a.half - e0;
        float v[V], o[V];
        load_vec(x + e0, cnt, 0.f, v);
  #pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          const float2 w = 2 * e < cnt ? cs[e0 / 2 + e] : make_float2(0.f, 0.f);
          o[2 * e] = v[2 * e] * w.x - v[2 * e + 1] * w.y;
          o[2 * e + 1] = v[2 * e + 1] * w.x + v[2 * e] * w.y;
        }
        store_vec(y + e0, cnt, o);
      } else {
        const int e0 = c * V, cnt = a.half - e0;
        float v1[V], v2[V], o1[V], o2[V];
        load_vec(x + e0, cnt, 0.f, v1);
        load_vec(x + a.half + e0, cnt, 0.f, v2);
  #pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 w = e < cnt ? cs[e0 + e] : make_float2(0.f, 0.f);
          o1[e] = v1[e] * w.x - v2[e] * w.y;
          o2[e] = v2[e] * w.x + v1[e] * w.y;
        }
        store_vec(y + e0, cnt, o1);
        store_vec(y + a.half + e0, cnt, o2);
      }
    }
    __syncthreads();   // before the next tokens' angles
  }
}

template <class T, bool PAIRS>
hipError_t launch(const RotaryArgs &a, hipStream_t s) {
  constexpr int V = kVec<T>;
  RotaryShape sh;
  const int rows = a.heads[0] + a.heads[1];
  sh.rot_tasks = ((PAIRS ? 2 : 1) * a.half + V - 1) / V;
  const bool copies = a.copy[0] || a.copy[1];
  sh.row_tasks = sh.rot_tasks + (copies ? (a.head_dim - 2 * a.half + V - 1) / V : 0);
  sh.tokens = 1;
  while (sh.tokens < 16 && 2 * sh.tokens * a.half <= kThreads && a.n_tokens / sh.tokens > 4096) sh.tokens *= 2;
  sh.half = FastDiv(a.half);
  sh.row = FastDiv(sh.row_tasks);
  sh.token = FastDiv(rows);
  int64_t grid = (a.n_tokens + sh.tokens - 1) / sh.tokens;
  if (grid > kMaxGrid) grid = kMaxGrid;
  rotary_kernel<T, PAIRS><<<dim3((uint32_t)grid), kThreads, sh.tokens * a.half * sizeof(float2), s>>>(a, sh);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(bool pairs, bool f32, const RotaryArgs &a, hipStream_t s) {
  if (f32) return pairs ? launch<float, true>(a, s) : launch<float, false>(a, s);
  return pairs ? launch<bf16, true>(a, s) : launch<bf16, false>(a, s);
}

}  // namespace nsp
