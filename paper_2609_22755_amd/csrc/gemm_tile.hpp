// A tile of a matrix product on the matrix cores, for the operators that work
// on the vocabulary's weight: C^T[q][p] = sum_k P(p, k) Q(q, k), bf16 operands,
// float32 sums.  P is the matrix instruction's row side, Q its column side, so a
// lane holds one q and, of each 32 x 32 block, the p's 8 (i / 4) + 4 (lane / 32)
// + i % 4 of its 16 elements i.
//
// An operand lies in memory with k along its rows (kAlong: row p or q, elements
// k) or across them (kAcross: row k, elements p or q).  Both go through LDS by
// direct loads of 16 bytes a lane, 64 k a stage: 128 bytes of a row, since an L2
// takes a request a cycle and channel, whether of 64 bytes or 128 (with stages of
// 32 k a product of two kAlong operands kept the matrix cores busy 57 to 71% of the
// time, one of two kAcross operands 77%).  The first kind is read back a row of 8 k
// a lane, the second transposed on the way (ds_read_b64_tr_b16).  Elements outside
// the operand are zeros: their loads are out of the resource's range, which touches
// no memory.
//
// P has three stages of LDS and Q two (96 + 64 KB at 256 x 256).  A stage's four
// blocks of 16 k are multiplied while the operands of the next block are read; its
// one barrier comes when the last block's operands are in registers, so the stage is
// free from there on: Q's loads for the stage after the next go out at once, P's for
// the third after it during the next two blocks.
#pragma once

#include <type_traits>
#include <utility>

#include "device_common.hpp"

namespace nsp {
namespace tile {

constexpr int kStep = 64;      // k a stage
constexpr int kBlocks = kStep / 16;
constexpr int kRowBytes = 2 * kStep;
constexpr int kRingP = 3, kRingQ = 2;
// An offset out of every resource's range.
constexpr unsigned kOutside = 0x80000000u;

enum Lie { kAlong, kAcross };

// f(0), ..., f(N - 1), as constants.
template <int... I, class F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F f) {
  each_of(std::make_integer_sequence<int, N>(), f);
}

// One stage of an operand of N rows or columns.
template <Lie LIE, int N>
struct Stage {
  static constexpr int kBytes = N * kRowBytes;
  static constexpr int kInstr = kBytes / 1024;   // direct loads of a wave's 1 KB
  static_assert(N % 8 == 0 && (LIE == kAlong || N % 128 == 0), "whole instructions");
};

// The loads of one operand: N rows (or columns) from `first` on by the NW waves of
// a workgroup.
template <Lie LIE, int N, int NW>
struct Loader {
  static constexpr int PER_WAVE = Stage<LIE, N>::kInstr >= NW ? Stage<LIE, N>::kInstr / NW : 1;
  static_assert(Stage<LIE, N>::kInstr % NW == 0 || NW % Stage<LIE, N>::kInstr == 0, "the loads split evenly");
  const char *base;            // of the stage that is loaded next (uniform)
  int64_t step_bytes;
  int left;                    // k's from its first on
  unsigned voff[PER_WAVE];
  int kk[PER_WAVE];            // the k (of the stage) that a lane's 16 bytes lie at
  int lds;                     // of the wave's first load in a stage

  // kAlong: rows first .. first + N - 1 of `data` (row stride `stride` elements),
  // those from `end` on outside; kAcross: the same of columns.  k's k0 .. k0 + n_k - 1.
  __device__ __forceinline__ Loader(const void *data, int64_t stride, int64_t first, int64_t end, int64_t k0, int n_k, int wave, int lane)
      : left(n_k) {
    constexpr int I = Stage<LIE, N>::kInstr;
    const int w = I >= NW ? wave * PER_WAVE : wave % I;   // (with fewer loads than waves some waves load the same)
    lds = w * 1024;
    if constexpr (LIE == kAlong) {
      base = (const char *)data + 2 * (first * stride + k0);
      step_bytes = 2 * kStep;
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        const int r = (w + i) * 8 + lane / 8;
        kk[i] = 8 * ((lane % 8) ^ swz<64>(r));
        voff[i] = first + r < end ? (unsigned)(2 * (r * (int)stride + kk[i])) : kOutside;
      }
    } else {
      base = (const char *)data + 2 * (k0 * stride + first);
      step_bytes = 2 * kStep * stride;
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        const int r = (w + i) % 16 * 4 + lane / 16;       // 4 rows of a part of 128 columns
        const int c = 128 * ((w + i) / 16) + 8 * ((lane % 16) ^ swz<128>(r));
        kk[i] = r;
        voff[i] = first + c < end ? (unsigned)(2 * (r * (int)stride + c)) : kOutside;
      }
    }
  }
  // Loads FROM .. TO - 1 of the next stage into `stage`; the last of them end it.
  template <int FROM, int TO>
  __device__ __forceinline__ void load(char *stage) {
    if constexpr (FROM < TO) {
      const uint64_t at = (uint64_t)base;
      const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, 0x7fffffff, 0x00020000);
#pragma unroll
      for (int i = FROM; i < TO; ++i) load_lds_untracked<16>(rs, kk[i] < left ? voff[i] : kOutside, stage + lds + i * 1024);
      if constexpr (TO == PER_WAVE) {
        base += step_bytes;
        left -= kStep;
      }
    }
  }
};

// Addresses (bytes, in LDS) of a wave's operands of stage 0: blocks of 32 rows or
// columns from `first` on.
template <Lie LIE, int BLOCKS>
struct Reader {
  unsigned at[LIE == kAlong ? kBlocks : 2 * BLOCKS];
  __device__ __forceinline__ Reader(unsigned ring, int first, int lane) {
    const int l32 = lane & 31, h = lane >> 5, g = lane >> 4, j = lane & 15;
    if constexpr (LIE == kAlong) {
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) {
        at[kb] = ring + 2u * (unsigned)tile_off<64>(first + l32, 16 * kb + 8 * h);
        asm volatile("" : "+v"(at[kb]));
      }
    } else {
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int c = first + 32 * b + 16 * (g & 1) + 4 * (j & 3), r = 8 * h + 4 * hi + (j >> 2);
          at[2 * b + hi] = ring + (unsigned)((c / 128) * 128 * kRowBytes + 2 * tile_off<128>(r, c % 128));
          asm volatile("" : "+v"(at[2 * b + hi]));
        }
    }
  }
  // Operand of block b, k's 16 kb + 8 (lane / 32) .. + 7, of the stage `off` bytes on.
  __device__ __forceinline__ bf16x8 operand(const char *smem, int kb, int b, unsigned off) const {
    if constexpr (LIE == kAlong) {
      return *(const bf16x8 *)(smem + at[kb] + off + 32 * kRowBytes * b);
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
  static constexpr unsigned kAtQ = kRingP * kBytesP;
  static constexpr int kLds = kAtQ + kRingQ * kBytesQ;
  using LoadP = Loader<LP, NP, NW>;
  using LoadQ = Loader<LQ, NQ, NW>;

  f32x16 acc[BQ][BP];
  int wave, lane, wp, wq;

  __device__ __forceinline__ Product() : wave(wave_id()), lane((int)threadIdx.x & 63) {
    wp = wave % WP;
    wq = wave / WP;
  }
  // First p and q (of the tile) of this wave.
  __device__ __forceinline__ int p0() const { return wp * (NP / WP); }
  __device__ __forceinline__ int q0() const { return wq * (NQ / WQ); }

  struct Operands {
    bf16x8 p[BP], q[BQ];
  };

  // The sums over n_k k's; every wave of the workgroup.  Nothing is in flight
  // afterwards and every wave is past its last read.
  __device__ __forceinline__ void run(char *smem, LoadP lp, LoadQ lq, int n_k) {
    clear();
    add(smem, lp, lq, n_k);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < BQ; ++q)
#pragma unroll
      for (int p = 0; p < BP; ++p) acc[q][p] = f32x16{};
  }
  // The same, added to what is there.
  __device__ __forceinline__ void add(char *smem, LoadP lp, LoadQ lq, int n_k) {
    constexpr int IP = LoadP::PER_WAVE, IQ = LoadQ::PER_WAVE;
    const Reader<LP, BP> rp(0, p0(), lane);
    const Reader<LQ, BQ> rq(kAtQ, q0(), lane);
    const auto at_p = [&](int stage) { return smem + stage % kRingP * kBytesP; };
    const auto at_q = [&](int stage) { return smem + kAtQ + stage % kRingQ * kBytesQ; };
    const auto read_q = [&](Operands &x, int stage, int kb) {
#pragma unroll
      for (int q = 0; q < BQ; ++q) x.q[q] = rq.operand(smem, kb, q, stage % kRingQ * kBytesQ);
    };
    const auto read_p = [&](Operands &x, int stage, int kb) {
#pragma unroll
      for (int p = 0; p < BP; ++p) x.p[p] = rp.operand(smem, kb, p, stage % kRingP * kBytesP);
    };
    // The products of x, with the next block's operands (block kb of `stage`) read
    // into `next` behind the first of them and `loads` direct loads, one behind each of
    // the following: what they take to issue hides behind a product.
    const auto block = [&](const Operands &x, Operands &next, int stage, int kb, auto loads, auto load) {
#pragma unroll
      for (int p = 0; p < BP; ++p)
#pragma unroll
        for (int q = 0; q < BQ; ++q) {
          constexpr int kProducts = BP * BQ, kLoads = decltype(loads)::value;
          const int i = p * BQ + q;
          acc[q][p] = mfma32x32x16(x.p[p], x.q[q], acc[q][p]);
          if (i == 0) {
            read_q(next, stage, kb);
            read_p(next, stage, kb);
            __builtin_amdgcn_s_setprio(1);       // (over the other wave's reads: 1%)
          }
          if (i == BP * BQ - 1) __builtin_amdgcn_s_setprio(0);
          if constexpr (kLoads > 0) {
            if (i > 0 || kProducts == 1) {
              // loads j with 1 + j * (kProducts - 1) / kLoads == i, or all of them
              static_for<kLoads>([&](auto j) {
                constexpr int J = decltype(j)::value;
                if ((kProducts == 1 ? 0 : 1 + J * (kProducts - 1) / kLoads) == i) load(j);
              });
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    };
    lp.template load<0, IP>(at_p(0));
    lq.template load<0, IQ>(at_q(0));
    lp.template load<0, IP>(at_p(1));
    lq.template load<0, IQ>(at_q(1));
    wait_loads_le<IP + IQ>();
    stage_barrier();
    Operands a, b;
    read_q(a, 0, 0);
    read_p(a, 0, 0);
    const int stages = (n_k + kStep - 1) / kStep;
    const auto none = [](auto) {};
    const auto stage = [&](auto cur) {
      constexpr int CUR = decltype(cur)::value;
      block(a, b, CUR, 1, std::integral_constant<int, IP / 2>(), [&](auto j) { lp.template load<j, j + 1>(at_p(CUR + 2)); });
      block(b, a, CUR, 2, std::integral_constant<int, IP - IP / 2>(),
            [&](auto j) { lp.template load<IP / 2 + j, IP / 2 + j + 1>(at_p(CUR + 2)); });
      block(a, b, CUR, 3, std::integral_constant<int, 0>(), none);
      // the next stage is in LDS (P's after it may be on its way), and the last
      // operands of this one in registers
      wait_loads_le<IP>();
      stage_barrier();
      block(b, a, CUR + 1, 0, std::integral_constant<int, IQ>(), [&](auto j) { lq.template load<j, j + 1>(at_q(CUR + 2)); });
    };
    for (int t = 0; t < stages;) {
#define NSP_TILE_STAGE(CUR)                       \
  stage(std::integral_constant<int, CUR>());      \
  if (++t >= stages) break;
      NSP_TILE_STAGE(0)
      NSP_TILE_STAGE(1)
      NSP_TILE_STAGE(2)
      NSP_TILE_STAGE(3)
      NSP_TILE_STAGE(4)
      NSP_TILE_STAGE(5)
#undef NSP_TILE_STAGE
    }
    wait_all_loads();
    stage_barrier();
  }
};

// Tile `id` of np x nq (p, q) in `parts` parts, for workgroups that go to the XCDs in
// turn: each XCD takes one run of the order, part after part, in which `group`
// neighbours of p pass over all q (its compute units then share group + some of q's
// operands in its L2).  False: there is none.
struct Place {
  int p, q, part;
  __device__ __forceinline__ bool find(int id, int np, int nq, int parts, int group) {
    const int tiles = np * nq, total = tiles * parts, x = id % kXcdQueues, i = id / kXcdQueues;
    const int per = total / kXcdQueues, more = total % kXcdQueues;
    if (i >= per + (x < more ? 1 : 0)) return false;
    int at = x * per + min(x, more) + i;
    part = parts > 1 ? at / tiles : 0;
    at -= part * tiles;
    const int g = at / (group * nq), in = at - g * group * nq;
    const int wide = min(group, np - g * group);
    q = in / wide;
    p = g * group + in - q * wide;
    return true;
  }
};

}  // namespace tile
}  // namespace nsp
