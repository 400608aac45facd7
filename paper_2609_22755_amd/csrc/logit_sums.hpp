// Device building blocks of the passes over rows of logits: the masked range, and
// running sums of exponentials with a lazily moved reference.
#pragma once

#include "row_common.hpp"

namespace nsp {
namespace logits {

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

}  // namespace logits
}  // namespace nsp
