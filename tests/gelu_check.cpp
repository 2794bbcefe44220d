// Host-side check of what GELU is made of (gated_tile.h): z^2 / 2 log2(e) with its rounding put back, and the tail of
// the normal distribution's integral over its exponential, against 64 bits over 0 <= z <= 20 (past it the integral
// is 0 in 32 bits) and, for the polynomial in 64 bits, up to 1e6.  Prints "ok" and exits 0, else the first
// mismatch.
#include <cmath>
#include <cstdio>

#include "../paper_2609_05228_amd/csrc/gated_tile.h"

// d log(t P(t)) / d log t
static double power(double t) {
  double p = ace::kTail[0], slope = 0;
  for (int k = 1; k < 10; ++k) {
    slope = slope * t + p;
    p = p * t + ace::kTail[k];
  }
  return 1 + t * slope / p;
}

int main() {
  const double step = std::ldexp(1.0, -24), half_log2e = 0.5 / std::log(2.0);
  double fit = 0;
  for (int i = 0; i <= 2000000; ++i) {
    const float z = static_cast<float>(i * 1e-5);
    const double x = z, want = -x * x * half_log2e;
    // rest is at most 2e-5 (half steps of z^2 and of e, and c_rest z^2) and a sum of three, each rounded
    const ace::HalfSquare v = ace::half_square(z);
    const double off = std::fabs(static_cast<double>(v.e) + v.rest - want);
    if (off > 3 * step * 2e-5 + 2 * std::ldexp(1.0, -53) * std::fabs(want)) {
      std::printf("z = %.9g: exponent off by %.3g\n", z, off);
      return 1;
    }
    const double tail = 0.5 * std::erfc(x * std::sqrt(0.5)) * std::exp(0.5 * x * x);
    fit = std::fmax(fit, std::fabs(ace::tail_of(1.0 / (1.0 + static_cast<double>(0.32f) * x)) / tail - 1));
    // in 32 bits: a half step of each partial sum on its way to the result, of the product with t, and of t twice over, times
    // the power of t that the value goes by there
    const double t = 1.0 / (1.0 + static_cast<double>(0.32f) * x);
    double p = ace::kTail[0], way = 0;
    for (int k = 1; k < 10; ++k) {
      p = p * t + ace::kTail[k];
      way = way * t + std::fabs(p);
    }
    const double most = 4.5e-8 + step * (way / p + 1 + 2 * power(t)), is = std::fabs(ace::tail_of(1.0f / fmaf(0.32f, z, 1.f)) / tail - 1);
    if (is > most) {
      std::printf("z = %.9g: tail off by %.3g of at most %.3g\n", z, is, most);
      return 1;
    }
  }
  // past z = 20 by the asymptotic series, whose first term left out is 105 / z^8
  for (double x = 20; x < 1e6; x *= 1.001) {
    const double q = 1 / (x * x), tail = (1 - q * (1 - 3 * q * (1 - 5 * q))) / (x * std::sqrt(2 * M_PI));
    fit = std::fmax(fit, std::fabs(ace::tail_of(1.0 / (1.0 + static_cast<double>(0.32f) * x)) / tail - 1) - 105 * q * q * q * q);
  }
  if (fit > 4.5e-8) {
    std::printf("the polynomial is off by %.3g\n", fit);
    return 1;
  }
  std::printf("ok\n");
  return 0;
}
