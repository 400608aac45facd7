// A tile of a matrix product on the matrix cores, for the operators that work
// on the vocabulary's weight: C^T[q][p] = sum_k P(p, k) Q(q, k), bf16 operands,
// float32 sums.  P is the matrix instruction's row side, Q its column side, so a
// lane holds one q and, of each 32 x 32 block, the p's 8 (i / 4) + 4 (lane / 32)
// + i % 4 of its 16 elements i.
//
// An operand lies in memory with k along its rows (kAlong: row p or q, elements
// k) or across them (kAcross: row k, elements p or q).  Both go through LDS by
// direct loads of 16 bytes a lane, 32 k a step, four stages deep; the first is
// read back a row of 8 k a lane, the second transposed on the way
// (ds_read_b64_tr_b16).  Elements outside the operand are zeros: their loads are
// out of the resource's range, which touches no memory.
//
// Step t (its loads and those of t + 1 have landed): the loads of t + 3 go out
// into the stage that t - 1 left, and while the products of a half of the step
// run, the operands of the next half are read; one barrier a step.
#pragma once

#include "device_common.hpp"

namespace nsp {
namespace tile {

constexpr int kStep = 32;      // k a step
constexpr int kStages = 4;
// An offset out of every resource's range.
constexpr unsigned kOutside = 0x80000000u;

enum Lie { kAlong, kAcross };

// Rows (bytes of an operand's stage: 2 * kStep a row or column).
template <Lie LIE, int N>
struct Stage {
  static constexpr int kBytes = N * 2 * kStep;
  static constexpr int kInstr = kBytes / 1024;   // direct loads of a wave's 1 KB
  static_assert(N % 16 == 0 && (LIE == kAlong || N % 128 == 0), "whole instructions");
};

// 16-byte chunk c (of 4) of row r of a kAlong stage, 64 bytes a row: 16 rows at the
// same chunk, as a quarter wave reads them, fall on all 64 banks.
__device__ __forceinline__ int along_slot(int r, int c) { return c ^ ((r >> 2) & 3); }

// The loads of one operand: N rows (or columns) from `base` on by the NW waves of
// a workgroup.
template <Lie LIE, int N, int NW>
struct Loader {
  static constexpr int PER_WAVE = Stage<LIE, N>::kInstr >= NW ? Stage<LIE, N>::kInstr / NW : 1;
  static_assert(Stage<LIE, N>::kInstr % NW == 0 || NW % Stage<LIE, N>::kInstr == 0, "the loads split evenly");
  const char *base;            // of the step that is loaded next (uniform)
  int64_t step_bytes;
  unsigned voff[PER_WAVE];
  int kk[PER_WAVE];            // the k (of the step) that a lane's 16 bytes lie at
  int lds;                     // of the wave's first load in a stage

  // kAlong: rows first .. first + N - 1 of `data` (row stride `stride` elements),
  // those from `end` on outside; kAcross: the same of columns.  k starts at k0.
  __device__ __forceinline__ Loader(const void *data, int64_t stride, int64_t first, int64_t end, int64_t k0, int wave, int lane) {
    constexpr int I = Stage<LIE, N>::kInstr;
    const int w = I >= NW ? wave * PER_WAVE : wave % I;   // (with fewer loads than waves some waves load the same)
    lds = w * 1024;
    if constexpr (LIE == kAlong) {
      base = (const char *)data + 2 * (first * stride + k0);
      step_bytes = 2 * kStep;
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        const int r = (w + i) * 16 + lane / 4, c = along_slot(r, lane % 4);
        kk[i] = 8 * c;
        voff[i] = first + r < end ? (unsigned)(2 * (r * (int)stride + 8 * c)) : kOutside;
      }
    } else {
      base = (const char *)data + 2 * (k0 * stride + first);
      step_bytes = 2 * kStep * stride;
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        const int at = (w + i) % 8, sub = (w + i) / 8;     // 4 rows of a part of 128 columns
        const int r = at * 4 + lane / 16, c = 128 * sub + 8 * ((lane % 16) ^ swz<128>(r));
        kk[i] = r;
        voff[i] = first + c < end ? (unsigned)(2 * (r * (int)stride + c)) : kOutside;
      }
    }
  }
  // The next step into `stage`; `left`: k's from its first on.
  __device__ __forceinline__ void load(char *stage, int left) {
    const uint64_t at = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) load_lds_untracked<16>(rs, kk[i] < left ? voff[i] : kOutside, stage + lds + i * 1024);
    base += step_bytes;
  }
};

// Addresses (bytes, in LDS) of a wave's operands of stage 0: blocks of 32 rows or
// columns from `first` on.
template <Lie LIE, int BLOCKS>
struct Reader {
  unsigned at[LIE == kAlong ? 2 : 2 * BLOCKS];
  __device__ __forceinline__ Reader(unsigned ring, int first, int lane) {
    const int l32 = lane & 31, h = lane >> 5, g = lane >> 4, j = lane & 15;
    if constexpr (LIE == kAlong) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int r = first + l32;
        at[kb] = ring + (unsigned)(r * 2 * kStep + 16 * along_slot(r, 2 * kb + h));
        asm volatile("" : "+v"(at[kb]));
      }
    } else {
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int c = first + 32 * b + 16 * (g & 1) + 4 * (j & 3), r = 8 * h + 4 * hi + (j >> 2);
          at[2 * b + hi] = ring + (unsigned)((c / 128) * 128 * 2 * kStep + 2 * tile_off<128>(r, c % 128));
          asm volatile("" : "+v"(at[2 * b + hi]));
        }
    }
  }
  // Operand of block b, k's 16 kb + 8 (lane / 32) .. + 7, of the stage `off` bytes on.
  __device__ __forceinline__ bf16x8 operand(const char *smem, int kb, int b, unsigned off) const {
    if constexpr (LIE == kAlong) {
      return *(const bf16x8 *)(smem + at[kb] + off + 32 * 2 * kStep * b);
    } else {
      const unsigned o = off + kb * 16 * 256;
      return cat4(lds_read_tr4((const bf16 *)(smem + at[2 * b] + o)), lds_read_tr4((const bf16 *)(smem + at[2 * b + 1] + o)));
    }
  }
};

// A workgroup of WP x WQ waves makes a tile of NP x NQ.
template <Lie LP, Lie LQ, int NP_, int NQ_, int WP_, int WQ_>
struct Product {
  static constexpr int NP = NP_, NQ = NQ_, WP = WP_, WQ = WQ_, NW = WP * WQ;
  static constexpr int BP = NP / WP / 32, BQ = NQ / WQ / 32;   // blocks of a wave
  static constexpr int kBytesP = Stage<LP, NP>::kBytes, kBytesQ = Stage<LQ, NQ>::kBytes;
  static constexpr int kLds = kStages * (kBytesP + kBytesQ);
  static constexpr unsigned kRingQ = kStages * kBytesP;
  using LoadP = Loader<LP, NP, NW>;
  using LoadQ = Loader<LQ, NQ, NW>;
  static constexpr int kLoads = LoadP::PER_WAVE + LoadQ::PER_WAVE;

  f32x16 acc[BQ][BP];
  int wave, lane, wp, wq;

  __device__ __forceinline__ Product() : wave(wave_id()), lane((int)threadIdx.x & 63) {
    wp = wave % WP;
    wq = wave / WP;
  }
  // First p and q (of the tile) of this wave.
  __device__ __forceinline__ int p0() const { return wp * (NP / WP); }
  __device__ __forceinline__ int q0() const { return wq * (NQ / WQ); }

  struct Half {
    bf16x8 p[BP], q[BQ];
  };

  // The sums over n_k k's; every wave of the workgroup.  Nothing is in flight
  // afterwards and every wave is past its last read.
  __device__ __forceinline__ void run(char *smem, LoadP lp, LoadQ lq, int n_k) {
    const Reader<LP, BP> rp(0, p0(), lane);
    const Reader<LQ, BQ> rq(kRingQ, q0(), lane);
#pragma unroll
    for (int q = 0; q < BQ; ++q)
#pragma unroll
      for (int p = 0; p < BP; ++p) acc[q][p] = f32x16{};
    int left = n_k;
    const auto load = [&](int stage) {
      lp.load(smem + (stage & 3) * kBytesP, left);
      lq.load(smem + kRingQ + (stage & 3) * kBytesQ, left);
      left -= kStep;
    };
    const auto read = [&](Half &x, int stage, int kb) {
#pragma unroll
      for (int q = 0; q < BQ; ++q) x.q[q] = rq.operand(smem, kb, q, (stage & 3) * kBytesQ);
#pragma unroll
      for (int p = 0; p < BP; ++p) x.p[p] = rp.operand(smem, kb, p, (stage & 3) * kBytesP);
    };
    const auto multiply = [&](const Half &x) {
#pragma unroll
      for (int p = 0; p < BP; ++p)
#pragma unroll
        for (int q = 0; q < BQ; ++q) acc[q][p] = mfma32x32x16(x.p[p], x.q[q], acc[q][p]);
    };
    load(0);
    load(1);
    load(2);
    wait_loads_le<kLoads>();
    stage_barrier();
    Half a, b;
    read(a, 0, 0);
    const int steps = (n_k + kStep - 1) / kStep;
    for (int t = 0; t < steps;) {
#define NSP_TILE_STEP(CUR)           \
  {                                  \
    load((CUR) + 3);                 \
    read(b, (CUR), 1);               \
    __builtin_amdgcn_sched_barrier(0); \
    multiply(a);                     \
    __builtin_amdgcn_sched_barrier(0); \
    read(a, (CUR) + 1, 0);           \
    __builtin_amdgcn_sched_barrier(0); \
    multiply(b);                     \
    wait_loads_le<kLoads>();         \
    stage_barrier();                 \
    if (++t >= steps) break;         \
  }
      NSP_TILE_STEP(0)
      NSP_TILE_STEP(1)
      NSP_TILE_STEP(2)
      NSP_TILE_STEP(3)
#undef NSP_TILE_STEP
    }
    wait_all_loads();
    stage_barrier();
  }
};

// Tile `id` of np x nq (p, q), for workgroups that go to the XCDs in turn: each
// XCD takes one run of the order, in which `group` neighbours of p pass over all q
// (its compute units then share group + some of q's operands in its L2).  False:
// there is none.
__device__ __forceinline__ bool place(int id, int np, int nq, int group, int &p, int &q) {
  const int total = np * nq, x = id % kXcdQueues, i = id / kXcdQueues;
  const int per = total / kXcdQueues, more = total % kXcdQueues;
  if (i >= per + (x < more ? 1 : 0)) return false;
  const int at = x * per + min(x, more) + i;
  const int g = at / (group * nq), in = at - g * group * nq;
  const int wide = min(group, np - g * group);
  q = in / wide;
  p = g * group + in - q * wide;
  return true;
}

}  // namespace tile
}  // namespace nsp
