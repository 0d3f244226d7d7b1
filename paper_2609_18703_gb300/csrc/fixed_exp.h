// fixed_exp.h — softmax weights in 64-bit fixed point, about 2^-40 off relative
// to the largest.  Plain C++, so that it can also be run on the host.
//
// A token is drawn by comparing u * (sum of the weights) with running sums.  In
// 32-bit floats such a sum is off by 2^-22 or so, and one row in some hundred
// would get its neighbour's token; whole numbers are summed without error in any
// order, so what is left is each weight's own error.
//
//   w = 2^B e^-((max - x) / T) = 2^(B - z),  z = (max - x) log2(e) / T,  B <= 50
//
// in pairs of 32-bit floats (the GPU's 64-bit floats are few, its 64-bit
// integers slow: a weight took 270 cycles of a warp's issue in integers, 60 in
// pairs of floats): z from the difference with its rounding error and the factor
// with its own; z = m / 32 + r, |r| <= 1 / 64, gives 2^-(m / 32) from a table and
// an exponent, and 2^-r = 1 + g + g^2 / 2 + .. with g = -r ln 2, whose first two
// terms are pairs (the fifth is below 2^-39, the sixth below 2^-48).  Every
// operation is rounded as written: a weight is the same wherever it is computed.
#pragma once

#include <cstdint>
#include <cstring>
#ifndef __CUDACC__
#include <cmath>
#endif

#ifndef RO_HD
#ifdef __CUDACC__
#define RO_HD __host__ __device__ __forceinline__
#else
#define RO_HD inline
#endif
#endif

namespace ro {

// 2^-(j/32) in two floats
#define RO_EXP_HI \
    0x1.0000000000000p+0f, 0x1.f507660000000p-1f, 0x1.ea4afa0000000p-1f, 0x1.dfc9740000000p-1f, \
    0x1.d5818e0000000p-1f, 0x1.cb720e0000000p-1f, 0x1.c199be0000000p-1f, 0x1.b7f7700000000p-1f, \
    0x1.ae89fa0000000p-1f, 0x1.a5503c0000000p-1f, 0x1.9c49180000000p-1f, 0x1.93737c0000000p-1f, \
    0x1.8ace540000000p-1f, 0x1.82589a0000000p-1f, 0x1.7a11480000000p-1f, 0x1.71f75e0000000p-1f, \
    0x1.6a09e60000000p-1f, 0x1.6247ec0000000p-1f, 0x1.5ab07e0000000p-1f, 0x1.5342b60000000p-1f, \
    0x1.4bfdae0000000p-1f, 0x1.44e0860000000p-1f, 0x1.3dea640000000p-1f, 0x1.371a740000000p-1f, \
    0x1.306fe00000000p-1f, 0x1.29e9e00000000p-1f, 0x1.2387a60000000p-1f, 0x1.1d48740000000p-1f, \
    0x1.172b840000000p-1f, 0x1.11301e0000000p-1f, 0x1.0b55860000000p-1f, 0x1.059b0e0000000p-1f
#define RO_EXP_LO \
    0x0.0p+0f, -0x1.246eb00000000p-27f, 0x1.52486c0000000p-28f, -0x1.908c940000000p-26f, \
    -0x1.822dbc0000000p-28f, -0x1.8837cc0000000p-28f, -0x1.3d56b20000000p-28f, -0x1.a094380000000p-26f, \
    -0x1.a94b140000000p-27f, -0x1.b83b540000000p-26f, 0x1.51f8480000000p-28f, -0x1.e647440000000p-26f, \
    0x1.15506e0000000p-28f, -0x1.accc7c0000000p-27f, -0x1.829fd00000000p-26f, 0x1.1d8bee0000000p-26f, \
    0x1.9fcef40000000p-27f, -0x1.f8b5500000000p-26f, -0x1.5bd5ec0000000p-28f, -0x1.2c56100000000p-26f, \
    -0x1.593abc0000000p-26f, 0x1.8624b40000000p-31f, 0x1.8246840000000p-26f, -0x1.18aac60000000p-26f, \
    0x1.4636e20000000p-26f, -0x1.5c04240000000p-26f, 0x1.ceac480000000p-26f, -0x1.d2e8ca0000000p-26f, \
    -0x1.c157420000000p-28f, -0x1.fdb4960000000p-26f, 0x1.9f31220000000p-26f, -0x1.9d4f520000000p-26f

constexpr uint32_t WEIGHT_BITS = 50;   // B at most

#ifdef __CUDA_ARCH__
#define RO_MUL(a, b) __fmul_rn(a, b)
#define RO_ADD(a, b) __fadd_rn(a, b)
#define RO_FMA(a, b, c) __fmaf_rn(a, b, c)
#else   // (compiled without contraction)
#define RO_MUL(a, b) ((a) * (b))
#define RO_ADD(a, b) ((a) + (b))
#define RO_FMA(a, b, c) fmaf(a, b, c)
#endif
RO_HD int32_t float_bits(float x) {
#ifdef __CUDA_ARCH__
  return __float_as_int(x);
#else
  int32_t i;
  memcpy(&i, &x, 4);
  return i;
#endif
}
RO_HD float bits_float(int32_t i) {
#ifdef __CUDA_ARCH__
  return __int_as_float(i);
#else
  float x;
  memcpy(&x, &i, 4);
  return x;
#endif
}

struct ExpScale {
  float hi, lo;   // log2(e) / (up T) in two floats
  // a power of two that keeps them, and what they multiply, normal numbers: 1 for
  // temperatures from 2^-64 to 2^64
  float up = 1.f;
};
RO_HD ExpScale exp_scale(float T) {
  ExpScale c;
  c.up = T < 0x1p-64f ? 0x1p64f : T > 0x1p64f ? 0x1p-64f : 1.f;
  const float t = RO_MUL(T, c.up);
  c.hi = 1.44269502162933349609f / t;   // the quotient, and its remainder's
  c.lo = RO_ADD(RO_FMA(-c.hi, t, 1.44269502162933349609f), 1.92596299112661746887e-8f) / t;
  return c;
}
struct Pair32 {
  float hi, lo;
};
// z, x <= top, neither a NaN; its higher part is 64 or more (or NaN) for weights of 0.
RO_HD Pair32 exp_argument(float top, float x, ExpScale c) {
  const float apart = x == top ? 0.f : RO_ADD(top, -x);
  const float v = RO_ADD(apart, -top);           // what its rounding lost, exactly:
  const float rest = x == top ? 0.f : RO_ADD(RO_ADD(top, -RO_ADD(apart, -v)), RO_ADD(-x, -v));
  const float d = RO_MUL(apart, c.up), lost = RO_MUL(rest, c.up);
  Pair32 z;
  z.hi = d == 0.f ? 0.f : RO_MUL(d, c.hi);
  z.lo = d == 0.f ? 0.f : RO_FMA(lost, c.hi, RO_FMA(d, c.lo, RO_FMA(d, c.hi, -z.hi)));
  return z;
}
// A weight in two whole numbers, hi 2^(B - 20) + lo (lo of either sign), and sums of a few.
struct Weight {
  int32_t hi;
  int64_t lo;
};
RO_HD uint64_t whole(Weight w, uint32_t B) { return (uint64_t)(((int64_t)w.hi << (B - 20)) + w.lo); }
RO_HD int32_t nearest(float x) {
#ifdef __CUDA_ARCH__
  return __float2int_rn(x);
#else
  return (int32_t)lrintf(x);
#endif
}
// The weight of argument z in steps of 1 / unit = 2^-B.  table(j): 2^-(j/32);
// called for every argument, by whole warps.
template <class Table>
RO_HD Weight exp_weight(Pair32 z, float unit, Table table) {
  const bool none = !(z.hi < 64.f);
  const float p = none ? 0.f : z.hi;
  const float t = RO_FMA(p, 32.f, 12582912.f);   // 1.5 2^23: the last bits are m
  const int32_t m = float_bits(t) - 0x4B400000;
  const float r0 = RO_FMA(RO_ADD(t, -12582912.f), -0.03125f, p);   // exact
  const float r = RO_ADD(r0, z.lo), rl = RO_ADD(RO_ADD(r0, -r), z.lo);
  const Pair32 T = table((uint32_t)m & 31u);
  // g = -(r + rl) ln 2, and e^g - 1 = u
  const float gh = RO_MUL(r, -0x1.62e43p-1f);
  const float gl = RO_FMA(rl, -0x1.62e43p-1f, RO_FMA(r, 0x1.05c61p-29f, RO_FMA(r, -0x1.62e43p-1f, -gh)));
  const float half = RO_MUL(gh, 0.5f), qh = RO_MUL(gh, half), ql = RO_FMA(gh, gl, RO_FMA(gh, half, -qh));
  const float more = RO_MUL(RO_MUL(gh, gh), RO_MUL(gh, RO_FMA(gh, RO_FMA(gh, 0x1.111112p-7f, 0x1.555556p-5f), 0x1.555556p-3f)));
  const float uh = RO_ADD(gh, qh), ul = RO_ADD(RO_ADD(RO_ADD(RO_ADD(gh, -uh), qh), gl), RO_ADD(ql, more));
  // T (1 + u)
  const float ph = RO_MUL(T.hi, uh), pl = RO_FMA(T.hi, uh, -ph);
  const float s0 = RO_ADD(T.hi, ph);
  const float s1 = RO_ADD(RO_ADD(RO_ADD(RO_ADD(T.hi, -s0), ph), pl), RO_FMA(T.hi, ul, RO_FMA(T.lo, uh, T.lo)));
  const float sh = RO_ADD(s0, s1), sl = RO_ADD(RO_ADD(s0, -sh), s1);
  // times 2^-(m / 32 rounded down), in steps of 2^-20, what is left in steps of 2^-B
  const float down = bits_float((127 - (m >> 5)) << 23);
  const float wh = RO_MUL(sh, down), wl = RO_MUL(sl, down);
  const float a = RO_ADD(wh, 12.f);              // 1.5 2^3: 23 bits below are 2^-20
  const float b = RO_MUL(RO_ADD(wh, -RO_ADD(a, -12.f)), unit), c = RO_MUL(wl, unit);   // at most 2^29 + 2^25
  Weight w;
  w.hi = none ? 0 : float_bits(a) - 0x41400000;
  w.lo = none ? 0 : nearest(b) + nearest(c);
  return w;
}

}  // namespace ro
