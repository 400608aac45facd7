// Device building blocks of the row operators: vectors of 16 bytes at any
// element's address, conversions, and sums over groups of lanes.
//
// Rows start wherever a caller's tensor puts them, so a lane's 16 bytes are
// aligned to an element only.  gfx950 loads and stores those in one
// instruction as well (unaligned accesses are on); only the last, incomplete
// vector of a row goes element by element.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nsp {

typedef __bf16 bf16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Elements of 16 bytes.
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Every element is read once: a non-temporal load (a read of 2 GiB reaches 7.1
// TB/s with it, 6.3 without, a copy 5.7 instead of 5.5).
__device__ __forceinline__ u32x4 load16(const void *p) { return __builtin_nontemporal_load((const u32x4_any *)p); }
__device__ __forceinline__ void store16(void *p, u32x4 v) { __builtin_nontemporal_store(v, (u32x4_any *)p); }

// The same of 16-bit elements at an address of no whole words, from the words
// that hold them: such vectors read where they start come at 4.7 TB/s, those at
// whole words at 5.8.
__device__ __forceinline__ u32x4 load16_odd(const void *p) {
  typedef uint32_t u32x4_word __attribute__((ext_vector_type(4), aligned(4)));
  const u32x4 w = __builtin_nontemporal_load((const u32x4_word *)((const char *)p - 2));
  const uint32_t last = *(const uint32_t *)((const char *)p + 14);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i + 1] : last, w[i], 16);
  return r;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) {
  return __uint_as_float((uint32_t)__builtin_bit_cast(unsigned short, x) << 16);
}

template <class T>
__device__ __forceinline__ void unpack(u32x4 w, float (&x)[kVec<T>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __uint_as_float(w[i]);
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// One rounding, to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(bf16)a, (bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

template <class T>
__device__ __forceinline__ u32x4 pack(const float (&x)[kVec<T>]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
    else w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  }
  return w;
}

// `cnt` (< a vector's) elements at p, the others `fill`.
template <class T>
__device__ __forceinline__ void load_some(const T *p, int cnt, float fill, float (&x)[kVec<T>]) {
#pragma unroll
  for (int e = 0; e < kVec<T>; ++e) x[e] = e < cnt ? to_f32(p[e]) : fill;
}

template <class T>
__device__ __forceinline__ void store_some(T *p, int cnt, const float (&x)[kVec<T>]) {
#pragma unroll
  for (int e = 0; e < kVec<T>; ++e)
    if (e < cnt) p[e] = (T)x[e];
}

template <class T>
__device__ __forceinline__ void load_vec(const T *p, int cnt, float fill, float (&x)[kVec<T>]) {
  if (cnt >= kVec<T>) unpack<T>(load16(p), x);
  else load_some(p, cnt, fill, x);
}

// The same of what other workgroups read too.
template <class T>
__device__ __forceinline__ void load_vec_kept(const T *p, int cnt, float fill, float (&x)[kVec<T>]) {
  if (cnt >= kVec<T>) unpack<T>(*(const u32x4_any *)p, x);
  else load_some(p, cnt, fill, x);
}

template <class T>
__device__ __forceinline__ void store_vec(T *p, int cnt, const float (&x)[kVec<T>]) {
  if (cnt >= kVec<T>) store16(p, pack<T>(x));
  else store_some(p, cnt, x);
}

// Each lane's x beside the x of the lane N further in its row of 16 (around),
// and over the rows: pairs of rows, then pairs of half waves.
template <int N>
__device__ __forceinline__ float row_turn(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + N, 0xf, 0xf, false));
}

// op over each aligned group of G (16 or 64) lanes, in every lane of it, the
// same bits in each: every step joins two values that both lanes hold, and op
// is commutative.
template <int G, class Op>
__device__ __forceinline__ float group_join(float x, Op op) {
  x = op(x, row_turn<8>(x));
  x = op(x, row_turn<4>(x));
  x = op(x, row_turn<2>(x));
  x = op(x, row_turn<1>(x));
  if constexpr (G == 64) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(b[0]), __uint_as_float(b[1]));
  }
  return x;
}

template <int G>
__device__ __forceinline__ float group_sum(float x) {
  // (not fused with a product that made x: one lane's would be rounded, its neighbour's not)
  return group_join<G>(x, [](float a, float b) {
#pragma clang fp contract(off)
    return a + b;
  });
}

__device__ __forceinline__ float wave_max(float x) {
  return group_join<64>(x, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace nsp
