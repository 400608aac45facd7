// Rotary positions of query and key heads for gfx950.
//
// Bound by HBM: every element is read and written once (2 x 2 bytes of bf16
// for 3 multiply-adds).  What could cost more is the angles: a sine and a
// cosine in float32, of an angle that is reduced to a turn in 64 bits, are
// worth some 60 instructions, as much as memory gives time for in two vectors
// of eight elements.  A token's angles are the same for all its heads, so a
// wave takes a token (or, where there are few, a run of a token's heads): its
// lanes form the pairs' (cos, sin) once, each some of them, pass them through
// LDS, and keep those of their own columns in registers for all its heads.
//
// A lane holds one vector (16 bytes) of a head, 64 / (vectors of a head) heads a
// wave at a time, so every load and store of a wave is one run of memory
// wherever the heads lie side by side; the other half of a pair comes from the
// lane that holds it.  (A lane that loaded both its halves itself, in runs of
// half a head, left half-used lines behind: heads of 96, 3.0 TB/s.)
//
// 65536 tokens x 36 heads of 128 bf16: 200 us, 6.0 TB/s (a copy: 5.7); half of
// each head rotated 198, float32 5.6 TB/s, 15 heads of 80 with 20 rotated (no whole
// vectors) 94 us in halves, 81 in pairs, 3.4 and 3.9; 24 tokens 4 us.
#include "nsp_internal.hpp"
#include "row_common.hpp"

namespace nsp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxGrid = 1 << 20;

struct RotaryShape {
  int vecs, at_once;         // vectors of a head, heads of a wave at a time
  int chunks, run;           // a token's heads in `chunks` runs of `run`
  FastDiv by_vecs, by_chunks;
};

// What one wave wrote to LDS is there for its other lanes (which run in step).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// WHOLE: halves (or rotated parts) and heads are whole numbers of vectors.
template <class T, bool PAIRS, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryShape sh) {
  constexpr int V = kVec<T>;
  constexpr int U = 3;       // heads of a lane in flight (36 of 128 in 9 turns; 1000 tokens 5.9 us, with two 6.8, six 6.4)
  __shared__ float2 angles[kWaves][kRotaryMaxDim / 2];
  __shared__ u32x4 stage[WHOLE ? 1 : kWaves][WHOLE ? 1 : 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = sh.by_vecs.quot(lane), vec = lane - slot * sh.vecs, e0 = vec * V;   // the lane's head of those at once, its vector
  const int rot = 2 * a.half, heads = a.heads[0] + a.heads[1];
  const bool turned = e0 < rot;
  const int cnt = min(V, a.head_dim - e0);
  const int64_t units = a.n_tokens * sh.chunks;
  for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
    const int token = (int)sh.by_chunks.quot((uint32_t)unit), chunk = (int)unit - token * sh.chunks;
    const int end = min(heads, (chunk + 1) * sh.run);
    int head = chunk * sh.run + slot;
    const auto mine = [&](int h) { return slot < sh.at_once && h < end; };
    const auto place = [&](const RowView (&v)[2], int h) {
      const bool key = h >= a.heads[0];
      const RowView &r = key ? v[1] : v[0];
      return r.data + ((int64_t)token * r.ts + (int64_t)(key ? h - a.heads[0] : h) * r.hs + e0) * (int)sizeof(T);
    };
    u32x4 raw[U];
    const auto load = [&](int h0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = h0 + i * sh.at_once;
        if (!mine(h)) continue;
        const T *x = (const T *)place(a.x, h);
        if (WHOLE || cnt == V) {
          raw[i] = load16(x);
        } else {
          float v[V];
          load_some(x, cnt, 0.f, v);
          raw[i] = pack<T>(v);
        }
      }
    };
    load(head);                                  // (on its way while the angles are formed)
    const double position = (double)a.positions[token];
    for (int p = lane; p < a.half; p += 64) {
      const double turns = position * a.freqs[p] * 0.15915494309189533576888376337251;   // 1 / (2 pi)
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      angles[wave][p] = make_float2(c * a.scale, s * (a.scale * a.sign));
    }
    wave_sync();
    // y = x cos + other sin', sin' with the sign of the element's half
    float cs[V], sn[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int i = e0 + e;
      const bool second = PAIRS ? e & 1 : WHOLE ? e0 >= a.half : i >= a.half;
      const int p = PAIRS ? i >> 1 : second ? i - a.half : i;
      const float2 w = i < rot ? angles[wave][p] : make_float2(1.f, 0.f);
      cs[e] = w.x;
      sn[e] = second ? w.y : -w.y;
    }
    wave_sync();                                 // before the next unit's angles
    for (; __any(mine(head)); head += U * sh.at_once) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = head + i * sh.at_once;
        float x[V], other[V], y[V];
        unpack<T>(raw[i], x);
        if constexpr (PAIRS && WHOLE) {
#pragma unroll
          for (int e = 0; e < V; ++e) other[e] = x[e ^ 1];
        } else if constexpr (WHOLE) {
          const int from = e0 < a.half ? lane + a.half / V : lane - a.half / V;
          u32x4 o;
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = (uint32_t)__shfl((int)raw[i][k], from);
          unpack<T>(o, other);
        } else {
          stage[wave][lane] = raw[i];
          wave_sync();
          const T *row = (const T *)&stage[wave][min(slot, sh.at_once - 1) * sh.vecs];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int at = e0 + e, o = PAIRS ? at ^ 1 : at < a.half ? at + a.half : at - a.half;
            other[e] = at < rot ? to_f32(row[o]) : 0.f;
          }
          wave_sync();
        }
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = WHOLE || e0 + e < rot ? x[e] * cs[e] + other[e] * sn[e] : x[e];
        if (!mine(h)) continue;
        T *out = (T *)place(a.y, h);
        if (turned) {
          if (WHOLE || cnt == V) store16(out, pack<T>(y));
          else store_some(out, cnt, y);
        } else if (h < a.heads[0] ? a.copy[0] : a.copy[1]) {
          if (WHOLE || cnt == V) store16(out, raw[i]);
          else store_some(out, cnt, x);
        }
      }
      load(head + U * sh.at_once);
    }
  }
}

template <class T, bool PAIRS>
hipError_t launch(const RotaryArgs &a, hipStream_t s) {
  constexpr int V = kVec<T>;
  RotaryShape sh;
  sh.vecs = (a.head_dim + V - 1) / V;
  sh.at_once = 64 / sh.vecs;
  // a token's heads in runs, as long as there are not 16 waves a compute unit
  // (1000 tokens 5.9 us; with 8 waves 6.8, 32 6.9)
  const int heads = a.heads[0] + a.heads[1], rounds = (heads + sh.at_once - 1) / sh.at_once;
  int chunks = (int)(4096 / a.n_tokens);
  chunks = chunks < 1 ? 1 : chunks > rounds ? rounds : chunks;
  sh.run = (rounds + chunks - 1) / chunks * sh.at_once;
  sh.chunks = (heads + sh.run - 1) / sh.run;
  sh.by_vecs = FastDiv(sh.vecs);
  sh.by_chunks = FastDiv(sh.chunks);
  const int64_t blocks = (a.n_tokens * sh.chunks + kWaves - 1) / kWaves;
  const int grid = (int)(blocks < kMaxGrid ? blocks : kMaxGrid);
  const bool whole = a.head_dim % V == 0 && (PAIRS ? 2 * a.half : a.half) % V == 0;
  if (whole) rotary_kernel<T, PAIRS, true><<<grid, kThreads, 0, s>>>(a, sh);
  else rotary_kernel<T, PAIRS, false><<<grid, kThreads, 0, s>>>(a, sh);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(bool pairs, bool f32, const RotaryArgs &a, hipStream_t s) {
  if (f32) return pairs ? launch<float, true>(a, s) : launch<float, false>(a, s);
  return pairs ? launch<bf16, true>(a, s) : launch<bf16, false>(a, s);
}

}  // namespace nsp
