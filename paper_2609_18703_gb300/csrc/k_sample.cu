// k_sample.cu — tokens from logits and given random numbers (ro_sample).
//
//   w_i = e^((x_i - max) / T); tokens in order: larger logit first, equal ones by
//   index.  Top-k, top-p and min-p each keep the first so many of that order, so
//   all three keep the fewest of them: the tokens above a threshold and the
//   first few equal to it.  The token is the first kept one, by index, whose
//   running sum of weights passes u times the sum of all kept.
//
// Weights and sums are 64-bit fixed point (fixed_exp.h), so no sum depends on
// its order and tokens do not depend on how a row is split.
//
// A cluster of CTAs takes a row, a slice each in shared memory, read once from
// memory.  Thresholds come from passes over the bits of the logits' keys (which
// order alike), a histogram of counts (top-k) or of weights (top-p) summed over
// the cluster in each.
#include <algorithm>

#include "fixed_exp.h"
#include "ro_step.cuh"

namespace ro {

constexpr int SM_THREADS = 512;
constexpr uint32_t SM_WARPS = SM_THREADS / 32, SM_BINS = 2048, SM_MAX_CLUSTER = 8;
// bytes of a slice that a CTA holds at most
constexpr uint32_t SM_SLICE = 192 * 1024;
constexpr uint32_t NO_TOKEN = 0xFFFFFFFFu;
constexpr uint32_t KEY_NONE = 0x007FFFFFu;   // of -inf

// larger logit, larger key; -0 as 0
__device__ __forceinline__ uint32_t logit_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
// an item of CTA `rank` of the cluster: added to, fetched and added to, written
__device__ __forceinline__ void cluster_count(const uint32_t* p, uint32_t rank) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], 1;" ::"r"(cluster_at(step_smem(p), rank)) : "memory");
}
__device__ __forceinline__ uint32_t cluster_take(const uint32_t* p, uint32_t rank, uint32_t n) {
  uint32_t v;
  asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;"
               : "=r"(v)
               : "r"(cluster_at(step_smem(p), rank)), "r"(n)
               : "memory");
  return v;
}
__device__ __forceinline__ void cluster_write(const unsigned long long* p, uint32_t rank, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_at(step_smem(p), rank)), "l"(v) : "memory");
}
template <class V>
__device__ __forceinline__ V cluster_read(const V* p, uint32_t rank) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "a word or two");
  const uint32_t a = cluster_at(step_smem(p), rank);
  if constexpr (sizeof(V) == 8) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return (V)v;
  } else {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return (V)v;
  }
}
// x * f as a whole number, rounded down or up; 0 <= f < 1, x < 2^63.  (f is a
// whole number of at most 24 bits over a power of two.)
__device__ __forceinline__ uint64_t scaled(uint64_t x, float f, bool up) {
  if (f == 0.f || x == 0) return 0;
  int e;
  const uint64_t m = (uint64_t)(frexpf(f, &e) * 16777216.f);   // f = m 2^(e - 24)
  const int shift = 24 - e;                                      // at least 24
  if (shift >= 96) return up ? 1 : 0;
  const unsigned __int128 y = (unsigned __int128)x * m;
  return (uint64_t)((y + (up ? ((unsigned __int128)1 << shift) - 1 : 0)) >> shift);
}
__device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// 16 bytes of logits as they lie, and one of them
template <typename T>
struct Logits {
  static constexpr uint32_t E = 16 / sizeof(T);
  static __device__ __forceinline__ float at(const uint4& v, uint32_t i) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    const uint32_t h = (w[i / 2] >> (i % 2 * 16)) & 0xFFFFu;
    if constexpr (std::is_same_v<T, __half>)
      return __half2float(__ushort_as_half((unsigned short)h));
    else
      return __uint_as_float(h << 16);
  }
};
template <typename T>
__device__ __forceinline__ T minus_infinity();
template <>
__device__ __forceinline__ float minus_infinity<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ __half minus_infinity<__half>() { return __ushort_as_half(0xFC00); }
template <>
__device__ __forceinline__ __nv_bfloat16 minus_infinity<__nv_bfloat16>() { return __ushort_as_bfloat16(0xFF80); }

// Sorts the first n of v, a power of two, by one CTA: falling or rising.
// (Exchanges over at most 32 places stay within a warp's 64 items.)
__device__ __forceinline__ void sort_items(unsigned long long* v, uint32_t n, bool falling) {
  const uint32_t t = threadIdx.x;
  for (uint32_t size = 2; size <= n; size *= 2)
    for (uint32_t step = size / 2; step > 0; step /= 2) {
      if (step >= 32 || size == 2)
        __syncthreads();
      else
        __syncwarp();
      for (uint32_t c = t; c < n / 2; c += SM_THREADS) {
        const uint32_t i = 2 * c - (c & (step - 1)), j = i + step;
        const unsigned long long a = v[i], b = v[j];
        if ((a < b) == (((i & size) == 0) == falling) && a != b) {
          v[i] = b;
          v[j] = a;
        }
      }
    }
  __syncthreads();
}
__device__ const unsigned long long EXP_COARSE[32] = {RO_EXP_COARSE}, EXP_FINE[32] = {RO_EXP_FINE};

// What a row's tokens have to pass: keys above `key`, and the first `ties` equal to it.
struct Threshold {
  uint32_t key, ties;
};

// A row's candidates: the few tokens that can stay, where settings leave few.
constexpr uint32_t SM_LIST = 1024;
static_assert(2 * SM_LIST <= SM_BINS, "candidates and their weights lie where the bins do");
// Tokens that the candidates are meant to hold where top-p alone decides, and at
// most; and of the threads' largest logits.
constexpr uint32_t SM_WANT = 512, SM_WANT_MOST = 704;
constexpr uint32_t SM_COARSE = 512;
// What 32-bit weights and their sum may be off, relative to the sum: the
// argument, below 64, by 2^-23 of itself, and roundings of 2^-22.
constexpr double SM_SLACK = 1.0 / (1 << 16);
enum SampleWay : uint32_t { WAY_DONE, WAY_MASS, WAY_WIDE };

struct SampleShared {
  unsigned long long mass[SM_BINS];
  uint32_t count[SM_BINS];
  unsigned long long warp_mass[SM_WARPS];
  uint32_t warp_ties[SM_WARPS], warp_count[SM_WARPS];
  unsigned long long best;                 // key and ~place of the largest logit
  uint32_t least;                          // key of the threads' smallest maximum
  uint32_t coarse[SM_COARSE];              // the threads' maxima, counted by distance from the largest
  uint32_t cut, listed, way;
  float rough;                             // the sum of all weights in 32 bits
  float warp_rough[SM_WARPS];
  unsigned long long scan[SM_WARPS];
  unsigned long long found_left;
  uint32_t found;
  uint32_t total_ties;
  float temperature, top_p, min_p, u;
  uint32_t top_k, valid;
};

template <typename T>
__global__ void __launch_bounds__(SM_THREADS) sample_kernel(const __grid_constant__ SampleArgs a) {
  constexpr uint32_t E = Logits<T>::E;
  // the low bits of a 16-bit logit's key follow from its sign
  constexpr int LOW = std::is_same_v<T, float> ? 0 : std::is_same_v<T, __half> ? 11 : 16;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ SampleShared s;
  uint4* slice = (uint4*)smem_raw;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t nc = a.cluster, rank = nc > 1 ? cluster_rank() : 0, row = blockIdx.x / nc;
  auto sync = [&] {
    if (nc > 1)
      cluster_sync();
    else
      __syncthreads();
  };
  // the row in 16-byte blocks from the boundary before it on; place = index + off
  const T* x = (const T*)a.x + row * a.stride;
  const uint32_t off = (uint32_t)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T)), end = off + a.vocab;
  const uint4* blocks = (const uint4*)(x - off);
  const uint32_t n_blocks = (end + E - 1) / E;
  const uint32_t b0 = min(n_blocks, rank * a.blocks), n = min(n_blocks, b0 + a.blocks) - b0;
  if (tid == 0) {
    s.temperature = a.temperature ? a.temperature[row] : 1.f;
    s.top_p = a.top_p ? a.top_p[row] : 1.f;
    s.min_p = a.min_p ? a.min_p[row] : 0.f;
    s.top_k = a.top_k ? a.top_k[row] : 0u;
    s.u = a.u[row];
    s.valid = s.temperature >= 0.f && s.temperature < INFINITY && s.top_p >= 0.f && s.top_p <= 1.f && s.min_p >= 0.f &&
              s.min_p <= 1.f && s.u >= 0.f && s.u < 1.f;
    if (!s.valid && rank == 0) record(a.err, ERR_INVAL);
  }
  // ---- the slice, and the largest logit (the first of equal ones) ----
  float top = -INFINITY;
  uint32_t place = 0;
#pragma unroll 4
  for (uint32_t i = tid; i < n; i += SM_THREADS) {
    const uint32_t p0 = (b0 + i) * E;
    uint4 v;
    if (p0 >= off && p0 + E <= end) {
      v = __ldcs(blocks + b0 + i);
    } else {
      __align__(16) T e[E];
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) e[k] = p0 + k >= off && p0 + k < end ? x[p0 + k - off] : minus_infinity<T>();
      v = *(const uint4*)e;
    }
    slice[i] = v;
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) {
      const float y = Logits<T>::at(v, k);
      if (y > top) {
        top = y;
        place = p0 + k;
      }
    }
  }
  {
    unsigned long long b = top == -INFINITY ? 0 : (unsigned long long)logit_key(top) << 32 | ~place;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
    if (lane == 0) s.scan[warp] = b;
    __syncthreads();
    if (warp == 0) {
      b = lane < SM_WARPS ? s.scan[lane] : 0;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
      if (lane == 0) s.best = b;
    }
    const uint32_t low = __reduce_min_sync(0xffffffffu, top == -INFINITY ? ~0u : logit_key(top));
    if (lane == 0) s.warp_count[warp] = low;
    for (uint32_t i = tid; i < SM_COARSE; i += SM_THREADS) s.coarse[i] = 0;
    if (tid == 0) s.listed = 0;
    __syncthreads();
    if (warp == 0) {
      const uint32_t all = __reduce_min_sync(0xffffffffu, lane < SM_WARPS ? s.warp_count[lane] : ~0u);
      if (lane == 0) s.least = all;
    }
  }
  const float my_top = top;
  sync();
  unsigned long long best = s.best;
  uint32_t least = s.least;
  if (nc > 1)
    for (uint32_t r = 0; r < nc; ++r) {
      best = max(best, cluster_read(&s.best, r));
      least = min(least, cluster_read(&s.least, r));
    }
  const float T_ = s.temperature, top_p = s.top_p;
  uint32_t top_k = s.top_k;
  auto finish = [&](uint32_t token, float logp, uint32_t kept) {
    a.token[row] = token;
    if (a.logp) a.logp[row] = logp;
    if (a.kept) a.kept[row] = kept;
  };
  if (!s.valid || best == 0 || T_ == 0.f || top_k == 1u || top_p == 0.f) {   // (the whole cluster)
    if (rank == 0 && tid == 0) {
      if (!s.valid || best == 0)
        finish(NO_TOKEN, -INFINITY, 0);
      else
        finish(~(uint32_t)best - off, 0.f, 1);
    }
    if (nc > 1) cluster_sync();
    return;
  }
  top = key_logit((uint32_t)(best >> 32));

  // ---- weights ----
  const double c = 1.4426950408889634074 / (double)T_;
  const ExpScale scale = {(float)c, (float)(c - (double)(float)c)};
  const unsigned long long my_coarse = EXP_COARSE[lane], my_fine = EXP_FINE[lane];
  // of a whole warp's logits; 0 where !in
  auto weight = [&](float y, bool in) -> uint64_t {
    const uint64_t z = in ? exp_argument(top, y, scale) : ~0ull;
    if (!__any_sync(0xffffffffu, z != ~0ull)) return 0;
    const uint64_t w = exp_weight(
        z, a.frac_bits, [&](uint32_t j) { return (uint64_t)__shfl_sync(0xffffffffu, my_coarse, j); },
        [&](uint32_t j) { return (uint64_t)__shfl_sync(0xffffffffu, my_fine, j); });
    return z != ~0ull ? w : 0;
  };
  auto key_of = [&](float y) -> uint32_t { return y == y ? logit_key(y) : KEY_NONE; };   // (a NaN is never drawn)

  // ---- thresholds ----
  Threshold th = {KEY_NONE, 0};
  if (s.min_p > 0.f) {   // w >= min_p; the smallest such float
    const float least_x = __double2float_ru((double)top + (double)T_ * log((double)s.min_p));
    th.key = max(KEY_NONE, logit_key(least_x) - 1u);
  }
  // Every thread's items of a pass: this CTA's blocks, a warp's side by side, all warps alike in number.
  const uint32_t rounds = (n + SM_THREADS - 1) / SM_THREADS;
  // Finds the key where the tokens above `th`, largest first, reach `want` (in
  // tokens or in weight), which they do: leaves the key and what is still wanted of it.
  auto select = [&](auto by_mass, uint64_t want, uint64_t* left) -> uint32_t {
    constexpr bool MASS = decltype(by_mass)::value;
    uint32_t prefix = 0, mask = 0;
#pragma unroll 1
    for (int pass = 0; pass < (LOW == 0 ? 3 : 2); ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? (LOW == 0 ? 10 : LOW) : 0;
      const int bits = (pass == 0 ? 32 : pass == 1 ? 21 : 10) - shift;
      const uint32_t bins = 1u << bits;
      for (uint32_t i = tid; i < bins; i += SM_THREADS) {
        s.count[i] = 0;
        s.mass[i] = 0;
      }
      if (tid == 0) s.found = 0;
      __syncthreads();
      for (uint32_t r = 0; r < rounds; ++r) {
        const uint32_t i = r * SM_THREADS + tid;
        const uint4 v = i < n ? slice[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) {
          const float y = Logits<T>::at(v, k);
          const uint32_t key = key_of(y);
          const bool in = i < n && key > th.key && (key & mask) == prefix;
          if constexpr (MASS) {
            const uint64_t w = weight(y, in);
            if (in && w) atomicAdd(&s.mass[(key >> shift) & (bins - 1)], (unsigned long long)w);
          } else {
            if (in) atomicAdd(&s.count[(key >> shift) & (bins - 1)], 1u);
          }
        }
      }
      sync();
      // a thread sums its bins over the cluster, largest keys first
      const uint32_t each = max(1u, bins / SM_THREADS);
      uint64_t mine[SM_BINS / SM_THREADS], sum = 0;
#pragma unroll
      for (uint32_t j = 0; j < SM_BINS / SM_THREADS; ++j) {
        mine[j] = 0;
        const uint32_t d = tid * each + j;
        if (j < each && d < bins) {
          const uint32_t bin = bins - 1 - d;
          for (uint32_t q = 0; q < nc; ++q) {
            if constexpr (MASS)
              mine[j] += nc > 1 ? cluster_read(&s.mass[bin], q) : s.mass[bin];
            else
              mine[j] += nc > 1 ? cluster_read(&s.count[bin], q) : s.count[bin];
          }
        }
        sum += mine[j];
      }
      uint64_t inc = warp_incl_scan(sum);
      if (lane == 31) s.scan[warp] = inc;
      __syncthreads();
      uint64_t before = 0;
      for (uint32_t q = 0; q < warp; ++q) before += s.scan[q];
      before += inc - sum;
#pragma unroll
      for (uint32_t j = 0; j < SM_BINS / SM_THREADS; ++j) {
        if (before < want && before + mine[j] >= want) {
          s.found = bins - 1 - (tid * each + j);
          s.found_left = want - before;
        }
        before += mine[j];
      }
      sync();   // every CTA has read the others' bins
      prefix |= s.found << shift;
      mask |= (bins - 1) << shift;
      want = s.found_left;
      __syncthreads();
    }
    prefix |= (prefix & 0x80000000u) ? 0u : (1u << LOW) - 1u;   // a negative logit's low bits are ones
    *left = want;
    return prefix;
  };
  // Sums of what passes the threshold: over this warp's run of the slice, then over all before it.
  const uint32_t per = (n + SM_WARPS - 1) / SM_WARPS, i0 = min(n, warp * per), i1 = min(n, i0 + per);
  struct Sums {
    uint64_t mass, before, ties_before;   // of all; before this warp: weight above the threshold, tokens on it
    uint64_t ties, count;                 // on it, above it, in all
    uint64_t own;                         // this warp's weight above it
    uint32_t own_ties;
  };
  auto sums = [&](bool with_mass) -> Sums {
    uint64_t m = 0;
    uint32_t on = 0, above = 0;
    for (uint32_t i = i0; i < i1; i += 32) {
      const bool have = i + lane < i1;
      const uint4 v = have ? slice[i + lane] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        const float y = Logits<T>::at(v, k);
        const uint32_t key = key_of(y);
        const bool in = have && key > th.key;
        if (with_mass) m += weight(y, in);
        above += in;
        on += have && key == th.key;
      }
    }
    m = warp_sum64(m);
    on = __reduce_add_sync(0xffffffffu, on);
    above = __reduce_add_sync(0xffffffffu, above);
    if (lane == 0) {
      s.warp_mass[warp] = m;
      s.warp_ties[warp] = on;
      s.warp_count[warp] = above;
    }
    sync();
    Sums t = {};
    t.own = m;
    t.own_ties = on;
    for (uint32_t q = lane; q < nc * SM_WARPS; q += 32) {
      const uint32_t r = q / SM_WARPS, w = q % SM_WARPS;
      const uint64_t wm = nc > 1 ? cluster_read(&s.warp_mass[w], r) : s.warp_mass[w];
      const uint32_t wt = nc > 1 ? cluster_read(&s.warp_ties[w], r) : s.warp_ties[w];
      const uint32_t wc = nc > 1 ? cluster_read(&s.warp_count[w], r) : s.warp_count[w];
      t.mass += wm;
      t.ties += wt;
      t.count += wc;
      if (q < rank * SM_WARPS + warp) {
        t.before += wm;
        t.ties_before += wt;
      }
    }
    t.mass = warp_sum64(t.mass);
    t.ties = warp_sum64(t.ties);
    t.count = warp_sum64(t.count);
    t.before = warp_sum64(t.before);
    t.ties_before = warp_sum64(t.ties_before);
    sync();   // read by all before it is written again
    return t;
  };

  // ---- few candidates ----
  // At least `want` tokens lie at or above the want-th largest of the threads'
  // maxima, and seldom many more.  Where top-k, top-p or min-p leaves only some
  // of those, they are gathered and sorted by the first CTA, and the rest of the
  // row is not looked at again.  The sum that top-p is a share of is first taken
  // in 32 bits; only if a border lies within what that may be off, exactly.
  const bool by_k = top_k != 0u && top_k < a.vocab, by_p = top_p < 1.f, by_min = s.min_p > 0.f;
  const uint32_t threads = nc * SM_THREADS, most = min(SM_WANT_MOST, threads * 3 / 4);
  uint32_t way = WAY_WIDE;
  if ((by_k || by_p || by_min) && top < INFINITY) {
    const uint32_t want = by_k && top_k <= most ? top_k : min(SM_WANT, most);
    const bool all_of_k = by_k && top_k <= most;   // the candidates hold the first top_k
    // maxima counted by how far they lie below the largest
    // (as far as weights go: beyond 45 T they are below 2^-64)
    const float per_bin = (float)SM_COARSE / fmaxf(fminf(top - key_logit(least), 45.f * T_), 1e-30f);
    auto bin_of = [&](float y) { return (uint32_t)fminf((top - y) * per_bin, (float)(SM_COARSE - 1)); };
    if (my_top > -INFINITY) {
      const uint32_t b = bin_of(my_top);
      if (nc > 1)
        for (uint32_t r = 0; r < nc; ++r) cluster_count(&s.coarse[b], r);
      else
        atomicAdd(&s.coarse[b], 1u);
    }
    if (by_p && !all_of_k) {
      float sum = 0.f;
      for (uint32_t i = tid; i < n; i += SM_THREADS) {
        const uint4 v = slice[i];
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) {
          const float y = Logits<T>::at(v, k);
          if (y > -INFINITY) {                      // (and no NaN)
            const float d = top - y, z = d * scale.hi, e = fmaf(d, scale.lo, fmaf(d, scale.hi, -z));
            if (z < 64.f) sum = fmaf(ex2(-z), fmaf(e, -LN2, 1.f), sum);
          }
        }
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) s.warp_rough[warp] = sum;
    }
    sync();
    // the bin at which `want` maxima are reached: its far end is the cut
    static_assert(SM_COARSE == SM_THREADS, "a bin a thread");
    if (tid == 0) {
      s.cut = SM_COARSE;
      float sum = 0.f;
      for (uint32_t w = 0; w < SM_WARPS; ++w) sum += s.warp_rough[w];
      s.rough = sum;
    }
    const uint32_t mine = s.coarse[tid], inc = warp_incl_scan(mine);
    if (lane == 31) s.warp_count[warp] = inc;
    __syncthreads();
    uint32_t before = inc - mine;
    for (uint32_t w = 0; w < warp; ++w) before += s.warp_count[w];
    if (before < want && before + mine >= want) s.cut = tid;
    __syncthreads();
    const uint32_t cut = s.cut;                      // SM_COARSE: fewer maxima than wanted, so every token
    const bool with_min = by_min && !all_of_k;       // (top-p's sum is over the first top_k, whatever min-p says)
    auto candidate = [&](float y) {
      return y > -INFINITY && (cut == SM_COARSE || bin_of(y) <= cut) && (!with_min || logit_key(y) > th.key);
    };
    if (candidate(my_top))
      for (uint32_t i = tid; i < n; i += SM_THREADS) {
        const uint4 v = slice[i];
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) {
          const float y = Logits<T>::at(v, k);
          if (!candidate(y)) continue;
          const unsigned long long item = (unsigned long long)logit_key(y) << 32 | ~((b0 + i) * E + k - off);
          if (nc > 1) {
            const uint32_t at = cluster_take(&s.listed, 0, 1u);
            if (at < SM_LIST) cluster_write(&s.mass[at], 0, item);
          } else {
            const uint32_t at = atomicAdd(&s.listed, 1u);
            if (at < SM_LIST) s.mass[at] = item;
          }
        }
      }
    sync();
    // ---- the first CTA's ----
    unsigned long long* list = s.mass;
    unsigned long long* weights = s.mass + SM_LIST;
    // Whether every token that min-p leaves is a candidate, or every token.
    const uint32_t listed = rank == 0 ? s.listed : 0;
    uint64_t own[2] = {0, 0}, ahead[2] = {0, 0};               // weights of this thread's two candidates, and of those ahead
    bool whole = false;
    double rough = 0.0;
    // how many stay, given the sum that top-p is a share of; false: not the tokens alone decide
    auto count_below = [&](uint64_t limit, uint32_t first) -> uint32_t {
      const uint32_t mine2 = (2 * tid < first && ahead[0] < limit) + (2 * tid + 1 < first && ahead[1] < limit);
      return (uint32_t)__syncthreads_count(mine2 >= 1) + (uint32_t)__syncthreads_count(mine2 >= 2);
    };
    uint32_t stay = 0, first = 0;
    if (rank == 0) {
      way = WAY_WIDE;
      if (listed > 0 && listed <= SM_LIST) {
        uint32_t size = 2;
        while (size < listed) size *= 2;
        for (uint32_t i = listed + tid; i < size; i += SM_THREADS) list[i] = 0;
        sort_items(list, size, true);
        uint64_t sum = 0;
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
          const uint32_t i = 2 * tid + j;
          own[j] = weight(key_logit((uint32_t)(list[min(i, SM_LIST - 1)] >> 32)), i < listed);
          if (i < listed) weights[i] = own[j];
          sum += own[j];
        }
        const uint64_t run = warp_incl_scan(sum);
        if (lane == 31) s.scan[warp] = run;
        __syncthreads();
        uint64_t base = run - sum;
        for (uint32_t w = 0; w < warp; ++w) base += s.scan[w];
        ahead[0] = base;
        ahead[1] = base + own[0];
        uint64_t list_mass = 0;
        for (uint32_t w = 0; w < SM_WARPS; ++w) list_mass += s.scan[w];
        // min-p's
        uint32_t by_limit = listed;
        if (by_min) {
          const uint32_t in = (2 * tid < listed && (uint32_t)(list[2 * tid] >> 32) > th.key) +
                              (2 * tid + 1 < listed && (uint32_t)(list[2 * tid + 1] >> 32) > th.key);
          by_limit = (uint32_t)__syncthreads_count(in >= 1) + (uint32_t)__syncthreads_count(in >= 2);
        }
        // every token that counts for the outcome of top-k and min-p is listed:
        // all of them, the first top_k, or all that min-p leaves
        whole = cut == SM_COARSE || all_of_k || by_limit < listed || (with_min && bin_of(key_logit(th.key + 1u)) <= cut);
        first = all_of_k ? min(top_k, listed) : listed;
        stay = min(first, by_limit);
        if (!by_p) {
          if (by_k) stay = min(stay, top_k);
          way = whole ? WAY_DONE : WAY_WIDE;
        } else if (all_of_k || (cut == SM_COARSE && !with_min && !by_k)) {   // the sum is the listed ones'
          const uint64_t sum_first = first == listed ? list_mass : [&] {
            if (tid == first / 2) s.found_left = ahead[first & 1];
            __syncthreads();
            return (uint64_t)s.found_left;
          }();
          stay = min(stay, max(1u, count_below(scaled(sum_first, top_p, true), first)));
          way = WAY_DONE;
        } else if (!by_k) {
          if (nc > 1) {
            for (uint32_t r = 0; r < nc; ++r) rough += (double)__uint_as_float(cluster_read((const uint32_t*)&s.rough, r));
          } else {
            rough = (double)s.rough;
          }
          rough *= exp2((double)a.frac_bits) * (double)top_p;
          const uint32_t lo = max(1u, count_below((uint64_t)(rough * (1.0 - SM_SLACK)), listed));
          const uint32_t hi = max(1u, count_below((uint64_t)(rough * (1.0 + SM_SLACK)) + 2, listed));
          // (hi == listed: top-p may leave tokens that are not listed)
          if (!whole && hi == listed)
            way = WAY_WIDE;
          else if (min(lo, stay) == min(hi, stay))
            way = WAY_DONE, stay = min(lo, stay);
          else
            way = WAY_MASS;
        }
      }
      if (tid < nc) {   // to every CTA's own: this one may be gone before they look
        if (nc > 1)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_at(step_smem(&s.way), tid)), "r"(way) : "memory");
        else
          s.way = way;
      }
    }
    sync();
    way = s.way;
    if (way == WAY_MASS) {
      const Threshold keep = th;
      th = {KEY_NONE, 0};
      const uint64_t sum = sums(true).mass;
      th = keep;
      if (rank == 0) stay = min(stay, max(1u, count_below(scaled(sum, top_p, true), listed)));
      way = WAY_DONE;
    }
    if (way == WAY_DONE) {
      if (rank == 0) {
        // the sum of those that stay, then where it passes the goal, by index
        if (2 * tid < stay && stay <= 2 * tid + 2) s.found_left = ahead[(stay - 1) & 1] + own[(stay - 1) & 1];
        __syncthreads();
        const uint64_t total = s.found_left, goal = scaled(total, s.u, false);
        uint32_t size = 2;
        while (size < stay) size *= 2;
        unsigned long long item[2];
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) item[j] = 2 * tid + j < stay ? list[2 * tid + j] : 0;
        __syncthreads();
        // places rise, and each remembers its candidate; keys and weights stay where they are
        unsigned long long* order = (unsigned long long*)s.count;   // 1,024 of them
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j)
          if (2 * tid + j < size)
            order[2 * tid + j] = 2 * tid + j < stay ? (unsigned long long)~(uint32_t)item[j] << 32 | (2 * tid + j) : ~0ull;
        sort_items(order, size, false);
        uint64_t w2[2], sum = 0;
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
          w2[j] = 2 * tid + j < stay ? weights[(uint32_t)order[2 * tid + j]] : 0;
          sum += w2[j];
        }
        const uint64_t run = warp_incl_scan(sum);
        if (lane == 31) s.scan[warp] = run;
        __syncthreads();
        uint64_t at = run - sum;
        for (uint32_t w = 0; w < warp; ++w) at += s.scan[w];
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
          if (goal >= at && goal < at + w2[j]) {
            const unsigned long long o = order[2 * tid + j];
            const float y = key_logit((uint32_t)(list[(uint32_t)o] >> 32));
            const double less = y == top ? 0.0 : ((double)top - (double)y) / (double)T_;
            finish((uint32_t)(o >> 32), -(float)(less + log((double)total * exp2(-(double)a.frac_bits))), stay);
          }
          at += w2[j];
        }
      }
      return;
    }
  }

  if (top_k != 0u && top_k < a.vocab) {
    if (sums(false).count > top_k) {
      uint64_t left;
      th.key = select(std::false_type(), top_k, &left);
      th.ties = (uint32_t)left;
    }
  }
  if (top_p < 1.f) {
    // the mass of the first k: with min-p's cut it is not that, so top-k's own threshold counts
    Threshold cut = th;
    Threshold k_only = {KEY_NONE, 0};
    if (s.min_p > 0.f) {
      th = k_only;
      if (top_k != 0u && top_k < a.vocab && sums(false).count > top_k) {
        uint64_t left;
        th.key = select(std::false_type(), top_k, &left);
        th.ties = (uint32_t)left;
      }
    }
    const Sums t = sums(true);
    const uint64_t tie = weight(key_logit(th.key), th.ties != 0u);
    const uint64_t want = scaled(t.mass + tie * th.ties, top_p, true);
    if (want <= t.mass) {
      uint64_t left;
      const uint32_t key = select(std::true_type(), want, &left);
      const uint64_t w = weight(key_logit(key), true);
      th.key = key;
      th.ties = (uint32_t)min((left + w - 1) / w, (uint64_t)0xFFFFFFFFu);
    } else {
      th.ties = (uint32_t)min((want - t.mass + tie - 1) / tie, (uint64_t)th.ties);
    }
    if (cut.key > th.key || (cut.key == th.key && cut.ties < th.ties)) th = cut;
  }

  // ---- the token ----
  const Sums t = sums(true);
  const uint64_t tie = weight(key_logit(th.key), th.ties != 0u);
  const uint64_t ties = min((uint64_t)th.ties, t.ties);
  const uint64_t total = t.mass + tie * ties;
  const uint64_t goal = scaled(total, s.u, false);   // the first running sum above it
  uint64_t ties_before = min(ties, t.ties_before);
  uint64_t at = t.before + tie * ties_before;
  const uint64_t own = t.own + tie * (min(ties, t.ties_before + t.own_ties) - ties_before);
  if (goal >= at && goal < at + own) {              // this warp's run has it
    for (uint32_t i = i0; i < i1; i += 32) {
      const bool have = i + lane < i1;
      const uint4 v = have ? slice[i + lane] : make_uint4(0, 0, 0, 0);
      uint64_t w[E], sum = 0;
      uint32_t on = 0;
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        const float y = Logits<T>::at(v, k);
        const uint32_t key = key_of(y);
        w[k] = weight(y, have && key > th.key);
        sum += w[k];
        on += have && key == th.key;
      }
      const uint32_t on_inc = warp_incl_scan(on);
      uint64_t rank_on = ties_before + on_inc - on;  // (counted on past `ties`, where it has no effect)
      const uint64_t kept_on = min(ties, rank_on + on) - min(ties, rank_on);
      sum += tie * kept_on;
      const uint64_t inc = warp_incl_scan(sum);
      const uint64_t all = __shfl_sync(0xffffffffu, inc, 31);
      if (goal < at + all) {
        uint64_t run = at + inc - sum;
        if (goal >= run && goal < run + sum) {
          bool done = false;
#pragma unroll
          for (uint32_t k = 0; k < E; ++k) {
            uint64_t wk = w[k];
            const float y = Logits<T>::at(v, k);
            if (have && key_of(y) == th.key) {
              if (rank_on < ties) wk = tie;
              ++rank_on;
            }
            run += wk;
            if (!done && goal < run) {
              done = true;
              const double less = y == top ? 0.0 : ((double)top - (double)y) / (double)T_;
              finish((b0 + i + lane) * E + k - off, -(float)(less + log((double)total * exp2(-(double)a.frac_bits))),
                     (uint32_t)(t.count + ties));
            }
          }
        }
        break;
      }
      at += all;
      ties_before += __shfl_sync(0xffffffffu, on_inc, 31);
    }
  }
  if (nc > 1) cluster_sync();   // no CTA leaves while another reads its shared memory
}

template <typename T>
static uint32_t sample_blocks(uint32_t vocab) { return vocab / Logits<T>::E + 2; }

template <typename T>
static void launch(const LaunchCfg& L, SampleArgs a, int sms) {
  // CTAs of a row: as many as its slices need, and more while the GPU has room
  const uint32_t blocks = sample_blocks<T>(a.vocab);
  uint32_t nc = 1;
  while (nc < SM_MAX_CLUSTER && ((uint64_t)ceil_div(blocks, nc) * 16 > SM_SLICE / 3 ||
                                 ((uint64_t)a.rows * nc * 2 <= (uint64_t)sms && blocks / (nc * 2) >= SM_THREADS)))
    nc *= 2;
  a.cluster = nc;
  a.blocks = (uint32_t)ceil_div(blocks, nc);
  // the largest sum of weights stays below 2^63
  a.frac_bits = 46;
  while (((uint64_t)a.vocab << a.frac_bits) >> 62) --a.frac_bits;
  launch_k(L, K_SAMPLE, sample_kernel<T>, a.rows * nc, SM_THREADS, (size_t)a.blocks * 16, a, dim3(nc));
}
void launch_sample(const LaunchCfg& L, const SampleArgs& a, int dtype, int sms) {
  dtype == RO_F32 ? launch<float>(L, a, sms) : dtype == RO_F16 ? launch<__half>(L, a, sms) : launch<__nv_bfloat16>(L, a, sms);
}

template <typename T>
static cudaError_t allow() {
  return cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(SM_SLICE + 64));
}
cudaError_t prepare_sample_kernels() {
  for (cudaError_t e : {allow<float>(), allow<__half>(), allow<__nv_bfloat16>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
