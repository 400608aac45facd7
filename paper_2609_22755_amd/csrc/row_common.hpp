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

struct __attribute__((packed)) Bytes16 {
  u32x4 v;
};

__device__ __forceinline__ u32x4 load16(const void *p) { return ((const Bytes16 *)p)->v; }
__device__ __forceinline__ void store16(void *p, u32x4 v) { ((Bytes16 *)p)->v = v; }

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

template <class T>
__device__ __forceinline__ u32x4 pack(const float (&x)[kVec<T>]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(x[i]);
    } else {
      const bf16 a = (bf16)x[2 * i], b = (bf16)x[2 * i + 1];   // one rounding, to nearest even
      w[i] = (uint32_t)__builtin_bit_cast(unsigned short, a) |
             ((uint32_t)__builtin_bit_cast(unsigned short, b) << 16);
    }
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

template <class T>
__device__ __forceinline__ void store_vec(T *p, int cnt, const float (&x)[kVec<T>]) {
  if (cnt >= kVec<T>) store16(p, pack<T>(x));
  else store_some(p, cnt, x);
}

// Sum over each aligned group of G lanes (a power of two up to 64), in every
// lane of it; the same order in every lane.
template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int m = 1; m < G; m <<= 1) x += __shfl_xor(x, m);
  return x;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

}  // namespace nsp
