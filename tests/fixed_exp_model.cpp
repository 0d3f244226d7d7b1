// The fixed-point weights on the host, against exp in more bits: prints the
// largest error relative to the weight, in units of 2^-40, and whether weights
// of falling scores ever rise.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "fixed_exp.h"

static const uint64_t COARSE[32] = {RO_EXP_COARSE}, FINE[32] = {RO_EXP_FINE};

int main() {
  std::mt19937_64 g(1);
  std::uniform_real_distribution<double> u(0, 1);
  double worst = 0;
  uint64_t top_w = 0;
  long risen = 0;
  for (int i = 0; i < 2000000; ++i) {
    const double T = std::exp(std::log(0.05) + u(g) * std::log(20.0 / 0.05));
    const float Tf = (float)T, top = (float)((u(g) - 0.5) * std::pow(10.0, u(g) * 3));
    const float x = (float)(top - u(g) * 20.0 * Tf);
    if (x > top) continue;
    const double c = 1.4426950408889634074 / (double)Tf;
    const ro::ExpScale s = {(float)c, (float)(c - (float)c)};
    const uint32_t S = 46;
    const auto z = ro::exp_argument(top, x, s);
    if (z == ~0ull) continue;
    const uint64_t w = ro::exp_weight(z, S, [](uint32_t j) { return COARSE[j]; }, [](uint32_t j) { return FINE[j]; });
    const double want = std::exp(((double)x - (double)top) / (double)Tf) * std::ldexp(1.0, S);
    const double off = (std::fabs((double)w - want) - 0.5) / want * std::ldexp(1.0, 40);
    if (off > worst) worst = off;
    const auto z2 = ro::exp_argument(top, std::nextafterf(x, -INFINITY), s);
    if (z2 != ~0ull && z2 + 8 < z) ++risen;
    if (w > top_w) top_w = w;
  }
  const ro::ExpScale one = {1.442695f, 0.f};
  const uint64_t full = ro::exp_weight(ro::exp_argument(3.f, 3.f, one), 46, [](uint32_t j) { return COARSE[j]; },
                                       [](uint32_t j) { return FINE[j]; });
  std::printf("%.3f %ld %d %d\n", worst, risen, (int)(full == (1ull << 46)),
              (int)(ro::exp_argument(3.f, -INFINITY, one) == ~0ull));
  return 0;
}
