// fixed_exp.h — softmax weights in 64-bit fixed point, about 2^-40 off relative
// to the largest.  Plain C++, so that it can also be run on the host.
//
// A token is drawn by comparing u * (sum of the weights) with running sums.  In
// 32-bit floats such a sum is off by 2^-22 or so, and one row in some hundred
// would get its neighbour's token; integers are summed without error in any
// order, so what is left is each weight's own error.
//
//   w = 2^S e^-((max - x) / T) = 2^(S - z),  z = (max - x) log2(e) / T
//
// z is a product of two sums of two floats each (max - x with its rounding
// error, log2(e) / T with its own), taken to 43 bits behind the point.  Of its
// fraction ten bits choose 2^-(j/32) and 2^-(k/1024) from tables, and the rest r
// < 2^-10 enters as 1 - 2^-r = t - t^2/2 + t^3/6 with t = r ln 2 (the next term
// is below 2^-46).
#pragma once

#include <cstdint>
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

// floor(2^63 2^-(j/32)) and floor(2^63 2^-(j/1024))
#define RO_EXP_COARSE \
    0x8000000000000000ull, 0x7D41D96DB915019Dull, 0x7A92BE8A92436616ull, 0x77F25CCDEE6D7AE6ull, \
    0x75606373EE921C97ull, 0x72DC8373BE41A454ull, 0x70666F76154A7089ull, 0x6DFDDBCBED791BABull, \
    0x6BA27E656B4EB57Aull, 0x69540EC8F895722Dull, 0x6712460A8FC24072ull, 0x64DCDEC3371793D1ull, \
    0x62B39508AA836D6Full, 0x6096266533384A2Bull, 0x5E8451CFAC061B5Full, 0x5C7DD7A3B17DCF75ull, \
    0x5A827999FCEF3242ull, 0x5891FAC0E95612C8ull, 0x56AC1F752150A563ull, 0x54D0AD5A753E077Cull, \
    0x52FF6B54D8A89C75ull, 0x513821818624B40Cull, 0x4F7A993048D088D7ull, 0x4DC69CDCEAA72A9Cull, \
    0x4C1BF828C6DC54B8ull, 0x4A7A77D47F7B84B1ull, 0x48E1E9B9D588E19Bull, 0x47521CC5A2E6A9E0ull, \
    0x45CAE0F1F545EB73ull, 0x444C0740496D4294ull, 0x42D561B3E6243D8Aull, 0x4166C34C5615D0ECull
#define RO_EXP_FINE \
    0x8000000000000000ull, 0x7FE9D3A8E07BF086ull, 0x7FD3AB290E46D769ull, 0x7FBD867FDF0ACB3Bull, \
    0x7FA765ACA88F6453ull, 0x7F9148AEC0B9B7B1ull, 0x7F7B2F857D8C51E5ull, 0x7F651A30352731EEull, \
    0x7F4F08AE3DC7C426ull, 0x7F38FAFEEDC8DD26ull, 0x7F22F1219BA2B4AEull, 0x7F0CEB159DEAE091ull, \
    0x7EF6E8DA4B544F9Aull, 0x7EE0EA6EFAAF4479ull, 0x7ECAEFD302E950AFull, 0x7EB4F905BB0D4F78ull, \
    0x7E9F06067A4360BAull, 0x7E8916D497D0E3F4ull, 0x7E732B6F6B18732Aull, 0x7E5D43D64B99DDD7ull, \
    0x7E47600890F223DEull, 0x7E31800592DB7078ull, 0x7E1BA3CCA92D152Cull, 0x7E05CB5D2BDB84BEull, \
    0x7DEFF6B672F84E24ull, 0x7DDA25D7D6B2177Full, 0x7DC458C0AF549908ull, 0x7DAE8F7055489813ull, \
    0x7D98C9E62113E1FAull, 0x7D8308216B594720ull, 0x7D6D4A218CD895E5ull, 0x7D578FE5DE6E95A0ull

struct ExpScale {
  float hi, lo;   // log2(e) / T in two floats
};
RO_HD uint64_t mul_hi64(uint64_t a, uint64_t b) {
#ifdef __CUDA_ARCH__
  return __umul64hi(a, b);
#else
  return (uint64_t)(((unsigned __int128)a * b) >> 64);
#endif
}
// z = (top - x) (c.hi + c.lo) in units of 2^-43; ~0 when it is 64 or more.
// x <= top, neither a NaN; equal ones give 0.
RO_HD uint64_t exp_argument(float top, float x, ExpScale c) {
  if (x == top) return 0;
  const float d = top - x;                       // and what its rounding lost, exactly:
  const float v = d - top, lost = (top - (d - v)) + (-x - v);
  const float p = d * c.hi;
  if (!(p < 64.f)) return ~0ull;
  float e = fmaf(d, c.hi, -p);
  e = fmaf(d, c.lo, e);
  e = fmaf(lost, c.hi, e);
  const float q = p * 131072.f;                  // 2^17: below 2^23
  const int32_t whole = (int32_t)q;
  const int64_t rest = (int64_t)(int32_t)((q - (float)whole) * 67108864.f) + (int32_t)(e * 8796093022208.f);   // 2^26, 2^43
  const int64_t z = ((int64_t)whole << 26) + rest;
  return z > 0 ? (uint64_t)z : 0;
}
// 2^(S - z) for z in units of 2^-43, rounded to a whole number: S <= 46.
// coarse(j), fine(k): the tables; called for every argument, by whole warps.
template <class Coarse, class Fine>
RO_HD uint64_t exp_weight(uint64_t z, uint32_t S, Coarse coarse, Fine fine) {
  const uint32_t top = (uint32_t)(z >> 33);      // whole part and ten bits
  const uint64_t ab = mul_hi64(coarse((top >> 5) & 31u), fine(top & 31u));    // 2^62 2^-(..)
  const uint32_t r = (uint32_t)(z >> 1);         // the rest in units of 2^-42: 32 bits
#ifdef __CUDA_ARCH__
  const uint32_t t = __umulhi(r, 0xB17217F8u);   // ln 2 in 2^-32
#else
  const uint32_t t = (uint32_t)(((uint64_t)r * 0xB17217F8u) >> 32);
#endif
  const float f = (float)t * 2.2737367544323206e-13f;   // 2^-42
  const uint32_t less = (uint32_t)(f * f * (0.5f - f * 0.16666667f) * 4398046511104.f);
  const uint64_t w = ab - (((ab >> 32) * (uint64_t)(t - less)) >> 10);
  const uint32_t shift = 62u - S + (top >> 10);
  if (shift >= 64u) return 0;
  return shift == 0u ? w : (w + (1ull << (shift - 1))) >> shift;
}

}  // namespace ro
