// Rounding helpers shared by the elementwise kernels of libff (device code).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ff {

typedef float ff_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 ff_bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// two floats to a packed bf16 pair, nearest even (v_cvt_pk_bf16_f32)
__device__ inline uint32_t pack_bf16_rne(float a, float b) {
  ff_f32x2 f = {a, b};
  ff_bf16x2 h = __builtin_convertvector(f, ff_bf16x2);
  return __builtin_bit_cast(uint32_t, h);
}

// float64 -> float32 rounded to odd: truncate toward zero and set the last
// bit when inexact.  Rounding that result to bf16 (8 significant bits, far
// fewer than float32's 24) to nearest even equals rounding x directly.
__device__ inline float round_to_odd_f32(double x) {
  const float r = float(x);  // nearest even
  const double rd = double(r);
  if (rd == x) return r;
  uint32_t bits = __float_as_uint(r);
  if (fabs(rd) > fabs(x)) bits -= 1;  // one step toward zero
  return __uint_as_float(bits | 1u);
}

// Rotation of adjacent pairs in float64, rounded once to the storage type:
// (a, b) -> (a cos - b sin, a sin + b cos) with cs = (cos, sin); rotate_vec turns the
// pairs of one 16-byte vector of T.
__device__ inline uint32_t rotate_bf16_pair(uint32_t w, double2 cs) {
  const double a = bf16_lo(w), b = bf16_hi(w);
  const double o0 = a * cs.x - b * cs.y;
  const double o1 = a * cs.y + b * cs.x;
  return pack_bf16_rne(round_to_odd_f32(o0), round_to_odd_f32(o1));
}

template <typename T>
__device__ inline uint4 rotate_vec(uint4 w, const double2* cs) {
  if constexpr (sizeof(T) == 2) {
    w.x = rotate_bf16_pair(w.x, cs[0]);
    w.y = rotate_bf16_pair(w.y, cs[1]);
    w.z = rotate_bf16_pair(w.z, cs[2]);
    w.w = rotate_bf16_pair(w.w, cs[3]);
  } else {
    const double a0 = __uint_as_float(w.x), b0 = __uint_as_float(w.y);
    const double a1 = __uint_as_float(w.z), b1 = __uint_as_float(w.w);
    w.x = __float_as_uint(float(a0 * cs[0].x - b0 * cs[0].y));
    w.y = __float_as_uint(float(a0 * cs[0].y + b0 * cs[0].x));
    w.z = __float_as_uint(float(a1 * cs[1].x - b1 * cs[1].y));
    w.w = __float_as_uint(float(a1 * cs[1].y + b1 * cs[1].x));
  }
  return w;
}

}  // namespace ff
