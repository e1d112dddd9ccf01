// Cosines and sines of rotary angles.
//
// The angle of position p and frequency w (radians per position) is p w, formed in fp64: at a position of a million an fp32
// product is off by a sixteenth of a radian, an fp64 one by 1e-10.  It is reduced by multiples of pi / 2 held in two fp64 numbers (two fused
// multiply-adds; the multiple's last bits, which say the quadrant, are those of a number to which 1.5 x 2^52 was added) and both
// functions are their Taylor series on [-pi / 4, pi / 4], whose first terms left out are below 3e-14; results are rounded to
// fp32 once.  28 fp64 operations, without a branch; fp64 runs at the rate of fp32 here.
#pragma once

#include "lkv_common.h"

namespace lkv {

struct RotaryArgs {
  const double* inv_freq;   // [rotary_dim / 2]
  double factor;            // of cosine and sine
  int rotary_dim;
  int pairs;                // 1: channels 2i and 2i + 1 turn together; 0: i and i + rotary_dim / 2
};

__device__ __forceinline__ void rotary_cos_sin(int position, double inv_freq, double factor, float* c_out, float* s_out) {
  const double angle = (double)position * inv_freq;
  constexpr double kTwoOverPi = 0.63661977236758134308, kMagic = 6755399441055744.0;
  constexpr double kHalfPiHi = 1.57079632679489661923, kHalfPiLo = 6.12323399573676588613e-17;   // pi / 2 and what its fp64 number leaves
  const double t = fma(angle, kTwoOverPi, kMagic);
  const double k = t - kMagic;
  const uint32_t quarter = (uint32_t)__builtin_bit_cast(uint64_t, t) & 3u;
  double r = fma(-k, kHalfPiHi, angle);
  r = fma(-k, kHalfPiLo, r);
  const double z = r * r;
  // sin r = r (1 - z / 3! + z^2 / 5! - ...), cos r = 1 - z / 2! + z^2 / 4! - ...
  double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
  c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, -1.0 / 39916800.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, -0.5);
  s = fma(s * z, r, r);
  c = fma(c, z, 1.0);
  const bool swap = (quarter & 1u) != 0;
  const double cc = swap ? s : c, ss = swap ? c : s;
  *c_out = (float)((((quarter + 1u) & 2u) != 0 ? -cc : cc) * factor);
  *s_out = (float)(((quarter & 2u) != 0 ? -ss : ss) * factor);
}

// (a, b) turned by the angle; each product and sum rounded to fp32 by itself, so that the result does not hang on which of them
// a compiler fuses.
__device__ __forceinline__ void rotary_turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float y = a * c - b * s;
  const float z = b * c + a * s;
  a = y;
  b = z;
}

}  // namespace lkv
