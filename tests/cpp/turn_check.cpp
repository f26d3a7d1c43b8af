// CPU check of the rows' turn (ss_turn.h): sine and cosine against 113 bits, over angles of every size up to a limit (log2,
// the first argument).  Prints the worst error as log2 and as text.
#include <cmath>
#define __device__
#define __forceinline__ inline
#include "ss_turn.h"

#include <cstdio>
#include <cstdlib>
#include <random>

int main(int argc, char **argv) {
  const double most = argc > 1 ? std::atof(argv[1]) : 48;
  std::mt19937_64 rng(1);
  const __float128 half_pi = 1.57079632679489661923132169163975144Q;
  double worst = 0, at = 0;
  const auto check = [&](double p, float f, double scale) {
    const double a = p * (double)f;
    if (!(std::fabs(a) < std::ldexp(1.0, (int)most))) return;
    double c, s;
    ss::turn_of(p, f, scale, c, s);
    __float128 n = (__float128)a / half_pi;      // whole quarters, by the nearest
    const long long q = (long long)std::floor((double)n);
    const __float128 back = n - (__float128)q;
    const long long k = back > 0.5Q ? q + 1 : q;
    const long double x = (long double)((__float128)a - (__float128)k * half_pi);
    const long double sx = sinl(x), cx = cosl(x);
    const int r = (int)(((k % 4) + 4) % 4);
    const long double want_s = r == 0 ? sx : r == 1 ? cx : r == 2 ? -sx : -cx, want_c = r == 0 ? cx : r == 1 ? -sx : r == 2 ? -cx : sx;
    const double off = (double)hypotl((long double)c - scale * want_c, (long double)s - scale * want_s) / scale;
    if (!(off <= worst)) {
      worst = off;
      at = a;
    }
  };
  for (int i = 0; i < 4000000; ++i) {
    const double p = (double)(int32_t)(uint32_t)(rng() >> (32 + rng() % 32));                       // any position, and its negative
    const double span = most - 31;
    const float f = (float)std::ldexp((double)(rng() >> 11) / 9007199254740992.0 + 0.5, (int)(rng() % 60) - 50 + (int)span);
    check(rng() & 1 ? p : -p, f, 1.0 + (double)(rng() % 3) / 4);
  }
  // angles next to odd multiples of an eighth of a turn, where the rest is longest
  for (int e = 0; e < (int)most; ++e)
    for (int i = 0; i < 20000; ++i) {
      const double k = std::floor(std::ldexp((double)(rng() >> 11) / 9007199254740992.0, e)) * 2 + 1;
      check(1.0, (float)(k * 0.78539816339744831), 1.0);
      const double p = (double)(1u << 30) + (double)(rng() >> 35);
      check(p, (float)(k * 0.78539816339744831 / p), 1.0);
    }
  printf("worst 2^%.2f (%.3g) at %.17g\n", std::log2(worst), worst, at);
  return 0;
}
