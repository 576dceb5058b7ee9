// rotary.h -- the position rotation of query and key rows.
//
// Pair i of a row at position p turns by theta_i = p f_i: (x, y) becomes
// (x c - y s, y c + x s) with c = cos theta_i, s = sin theta_i.  theta is worked out
// in 64 bits (in 32, half a unit in the last place of a position of 100000 is 0.004
// rad), c and s are rounded to 32 bits once, each product and each sum to 32 bits
// (the sources that turn keys are compiled without contraction): the codes that the
// quantizer gives the turned rows are then the same wherever they are worked out.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace semkv {

struct RotaryArgs {
  const float* freqs;            // [dim / 2]
  const int32_t* positions;      // of the call's rows; null: a row's place in its sequence
  int32_t dim, interleaved;      // channels turned; pairs (2i, 2i+1), else (i, i + dim/2)
};

// cos and sin of p f, rounded to 32 bits: Cody and Waite's reduction, then Taylor's
// series.  k, the nearest whole number of quarter
// turns, comes out of an addition that leaves no bits below the point (its lowest
// bits say which quarter); the angle is reduced to [-pi/4, pi/4] by two parts of
// pi/2 (exact products in fused multiply-adds: k has at most 31 bits), then both
// series are summed as far as 64 bits reach: x^15/15! and x^16/16!, what follows is
// below 5e-17.  Some 30 operations in 64 bits, at the rate of 32-bit ones.
__device__ inline float2 turn_of(int32_t p, float f) {
  constexpr double WHOLE = 6755399441055744.0;                        // 1.5 2^52
  const double theta = double(p) * double(f);
  const double t = __builtin_fma(theta, 0.63661977236758134308, WHOLE);
  const double k = t - WHOLE;
  double r = __builtin_fma(-k, 1.5707963267948965580, theta);
  r = __builtin_fma(-k, 6.1232339957367658e-17, r);
  const double z = r * r;
  double s = -7.6471637318198164759e-13;                              // -1/15!
  s = __builtin_fma(s, z, 1.6059043836821614599e-10);                 //  1/13!
  s = __builtin_fma(s, z, -2.5052108385441718775e-8);                 // -1/11!
  s = __builtin_fma(s, z, 2.7557319223985890653e-6);                  //  1/9!
  s = __builtin_fma(s, z, -1.9841269841269841270e-4);                 // -1/7!
  s = __builtin_fma(s, z, 8.3333333333333333333e-3);                  //  1/5!
  s = __builtin_fma(s, z, -1.6666666666666666667e-1);                 // -1/3!
  s = __builtin_fma(s * z, r, r);
  double c = 4.7794773323873852974e-14;                               //  1/16!
  c = __builtin_fma(c, z, -1.1470745597729724714e-11);                // -1/14!
  c = __builtin_fma(c, z, 2.0876756987868098979e-9);                  //  1/12!
  c = __builtin_fma(c, z, -2.7557319223985890653e-7);                 // -1/10!
  c = __builtin_fma(c, z, 2.4801587301587301587e-5);                  //  1/8!
  c = __builtin_fma(c, z, -1.3888888888888888889e-3);                 // -1/6!
  c = __builtin_fma(c, z, 4.1666666666666666667e-2);                  //  1/4!
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const uint32_t q = uint32_t(__builtin_bit_cast(uint64_t, t));       // quarters, modulo 4; a frequency that is not finite leaves NaN in r
  const float a = float(q & 1 ? s : c), b = float(q & 1 ? c : s);
  return make_float2((q + 1) & 2 ? -a : a, q & 2 ? -b : b);
}

// The pair (x, y) turned.
__device__ inline float turned_x(float x, float y, float2 t) {
  const float a = x * t.x, b = y * t.y;
  return a - b;
}
__device__ inline float turned_y(float x, float y, float2 t) {
  const float a = y * t.x, b = x * t.y;
  return a + b;
}

}  // namespace semkv
