// Sine and cosine of a row's turn, in 64 bits; plain arithmetic, so that a host compiler takes it too.
#pragma once
#include <stdint.h>

namespace ss {

// scale cos(a) and scale sin(a), a = p f.  The nearest whole quarter turn is taken off in two steps, exactly but for the last bits,
// and Taylor series to x^11 and x^12 take the rest: off by 7e-12 over an eighth of a turn either way.  How many quarters is rounded
// from a 2 / pi, itself off by 2^-6 of one below 2^48, so that the rest may be as much longer: 1.4e-11; 8e-11 at 2^50.
__device__ __forceinline__ void turn_of(double p, float f, double scale, double &c, double &s) {
  const double a = p * (double)f, n = __builtin_rint(a * 0.63661977236758134);                            // 2 / pi
  const double x = __builtin_fma(-n, 6.123233995736766e-17, __builtin_fma(-n, 1.5707963267948966, a));      // pi / 2 in two parts
  const double y = x * x;
  const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  double u = __builtin_fma(y, -1.0 / 39916800, 1.0 / 362880), v = __builtin_fma(y, 1.0 / 479001600, -1.0 / 3628800);
  u = __builtin_fma(y, u, -1.0 / 5040);
  u = __builtin_fma(y, u, 1.0 / 120);
  u = __builtin_fma(y, u, -1.0 / 6);
  v = __builtin_fma(y, v, 1.0 / 40320);
  v = __builtin_fma(y, v, -1.0 / 720);
  v = __builtin_fma(y, v, 1.0 / 24);
  v = __builtin_fma(y, v, -0.5);
  const double sx = __builtin_fma(x * y, u, x), cx = __builtin_fma(y, v, 1.0);
  const double k = q & 1 ? sx : cx, l = q & 1 ? cx : sx;
  c = scale * ((q + 1) & 2 ? -k : k);
  s = scale * (q & 2 ? -l : l);
}

}  // namespace ss
