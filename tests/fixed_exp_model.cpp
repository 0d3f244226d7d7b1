// The fixed-point weights on the host, against exp in 64 bits: prints the
// largest error beyond two roundings relative to the weight, in units of 2^-40, how
// often weights of falling scores rise by more than that, whether a weight of
// the largest is one, and whether -inf weighs nothing.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "fixed_exp.h"

constexpr uint32_t BITS = ro::WEIGHT_BITS;
static const float HI[32] = {RO_EXP_HI}, LO[32] = {RO_EXP_LO};
static uint64_t weight(float top, float x, ro::ExpScale s) {
  return ro::whole(ro::exp_weight(ro::exp_argument(top, x, s), std::ldexp(1.f, BITS),
                                  [](uint32_t j) { return ro::Pair32{HI[j], LO[j]}; }),
                   BITS);
}

int main() {
  std::mt19937_64 g(1);
  std::uniform_real_distribution<double> u(0, 1);
  double worst = 0;
  long risen = 0;
  for (int i = 0; i < 2000000; ++i) {
    const double T = std::exp(std::log(0.05) + u(g) * std::log(20.0 / 0.05));
    const float Tf = (float)T, top = (float)((u(g) - 0.5) * std::pow(10.0, u(g) * 3));
    const float x = (float)(top - u(g) * (i % 2 ? 20.0 : 2.0) * Tf);
    if (x > top) continue;
    const float c = 1.44269502162933349609f / Tf;
    const ro::ExpScale s = {c, (fmaf(-c, Tf, 1.44269502162933349609f) + 1.92596299112661746887e-8f) / Tf};
    const uint64_t w = weight(top, x, s);
    const double want = std::exp(((double)x - (double)top) / (double)Tf) * std::ldexp(1.0, BITS);
    const double off = (std::fabs((double)w - want) - 1.0) / want * std::ldexp(1.0, 40);
    if (off > worst) worst = off;
    const uint64_t below = weight(top, std::nextafterf(x, -INFINITY), s);
    if (below > w && (double)(below - w) > 2 + std::ldexp((double)w, -39)) ++risen;
  }
  const ro::ExpScale one = {1.442695f, 0.f};
  std::printf("%.3f %ld %d %d\n", worst, risen, (int)(weight(3.f, 3.f, one) == (1ull << BITS)),
              (int)(weight(3.f, -INFINITY, one) == 0 && weight(INFINITY, 3.f, one) == 0 &&
                    weight(INFINITY, INFINITY, one) == (1ull << BITS)));
  return 0;
}
