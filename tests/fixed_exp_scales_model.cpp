// The fixed-point weights on the host at temperatures of every size a 32-bit
// float has, the subnormal ones among them, against exp in 64 bits: prints the
// largest error beyond two roundings relative to the weight, in units of 2^-40, and
// how many weights were looked at.
#include <cmath>
#include <cstdio>
#include <random>

#include "fixed_exp.h"

constexpr uint32_t BITS = ro::WEIGHT_BITS;
static const float HI[32] = {RO_EXP_HI}, LO[32] = {RO_EXP_LO};

int main() {
  std::mt19937_64 g(2);
  std::uniform_real_distribution<double> u(0, 1);
  double worst = 0;
  long n = 0;
  for (int e = -149; e <= 127; ++e)
    for (int i = 0; i < 4000; ++i) {
      const float T = (float)std::ldexp(1.0 + u(g), e);
      if (!std::isfinite(T)) continue;
      const float top = (float)((u(g) - 0.5) * std::pow(10.0, u(g) * 3) * T);
      const float x = (float)(top - u(g) * (i % 2 ? 20.0 : 2.0) * T);
      if (!std::isfinite(top) || !std::isfinite(x) || !std::isfinite(top - x) || x > top) continue;
      const uint64_t w = ro::whole(ro::exp_weight(ro::exp_argument(top, x, ro::exp_scale(T)), std::ldexp(1.f, BITS),
                                                  [](uint32_t j) { return ro::Pair32{HI[j], LO[j]}; }),
                                   BITS);
      const double want = std::exp(((double)x - (double)top) / (double)T) * std::ldexp(1.0, BITS);
      worst = std::fmax(worst, (std::fabs((double)w - want) - 1.0) / want * std::ldexp(1.0, 40));
      ++n;
    }
  std::printf("%.3f %ld\n", worst, n);
  return 0;
}
