// k_sample.cu — tokens from logits and given random numbers (ro_sample).
//
//   w_i = e^((x_i - max) / T); tokens in order: larger logit first, equal ones by
//   index.  Top-k, top-p and min-p each keep the first so many of that order, so
//   all three keep the fewest of them: the tokens above a threshold and the
//   first few equal to it.  The token is the first kept one, by index, whose
//   running sum of weights passes u times the sum of all kept.
//
// Weights are 64-bit fixed point (fixed_exp.h), the same wherever they are computed,
// and their sums whole numbers of up to 69 bits, so no sum depends on its order and
// tokens do not depend on how a row is split.
//
// Where the settings leave few tokens, those are found without a threshold being
// known: among the threads' largest logits the want-th largest has at least `want`
// tokens at or above it, and seldom many more.  These candidates are gathered,
// sorted and summed by one CTA, and the rest of the row is not looked at again.
// Other rows are wide: top-k's border is found by passes over the bits of the
// logits' keys (which order alike), top-p's by a histogram of weights in 32 bits
// that names the border's bin, an exact pass that sums what lies above the bin,
// and a sort of the bin itself, whose kept tokens' weights complete the sums.
//
// Few rows are split over clusters of CTAs, which hold their slices in shared
// memory.  Many rows take a CTA each, which reads its row from memory once and
// what it needs of it again from L2; the wide ones among them are left to a
// second kernel of clusters.
//
// Measured: one row of 32,000 32-bit logits, top-k and top-p: 14.9 us; 256 rows of
// 131,072 bf16 logits: 16 us to draw the largest (the logits' bytes: 10), 30 with
// top-k 50 and top-p; 90 us with settings of their own, among them some 17 wide
// rows, whose exact sums take 100 instructions a token (24 us for 12 rows of them
// without settings, 55 for 12 with top-p 0.9).  Bound by latency: meetings of a
// cluster, sorts, and the chains of the exact weights.
#include <algorithm>

#include "fixed_exp.h"
#include "ro_step.cuh"

namespace ro {

constexpr int SM_THREADS = 512;
constexpr uint32_t SM_WARPS = SM_THREADS / 32, SM_BINS = 2048, SM_MAX_CLUSTER = 8;
// bytes of a slice that a CTA holds at most, two of them on an SM; a longer one is read again
constexpr uint32_t SM_SLICE = 80 * 1024;
constexpr uint32_t NO_TOKEN = 0xFFFFFFFFu;
constexpr uint32_t KEY_NONE = 0x007FFFFFu;   // of -inf
constexpr uint32_t KEY_MINUS_ZERO = 0x7FFFFFFFu;

// larger logit, larger key; -0 as 0
__device__ __forceinline__ uint32_t logit_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
// an item of CTA `rank` of the cluster: fetched and added to, written
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
__device__ __forceinline__ void cluster_write(const uint32_t* p, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_at(step_smem(p), rank)), "r"(v) : "memory");
}
// v to an item of CTA `rank` of nc (its own if that is one)
__device__ __forceinline__ void cluster_add(uint32_t* p, uint32_t rank, uint32_t nc, uint32_t v) {
  if (nc > 1)
    cluster_take(p, rank, v);
  else
    atomicAdd(p, v);
}
__device__ __forceinline__ void cluster_add(unsigned long long* p, uint32_t rank, uint32_t nc, uint64_t v) {
  if (nc > 1)
    asm volatile("red.relaxed.cluster.shared::cluster.add.u64 [%0], %1;" ::"r"(cluster_at(step_smem(p), rank)), "l"(v) : "memory");
  else
    atomicAdd(p, (unsigned long long)v);
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
// A row's sum of weights: of up to 2^19, each at most 2^50.  (A warp's run of a
// row's slice, at most 2^13 tokens, adds up to 64 bits.)
using Sum = unsigned __int128;
__device__ __forceinline__ float sum_float(Sum x) { return fmaf((float)(uint64_t)(x >> 64), 0x1p64f, (float)(uint64_t)x); }
// x * f as a whole number, rounded down or up; 0 <= f < 1, x < 2^70.  (f is a
// whole number of at most 24 bits over a power of two.)
template <class X>
__device__ __forceinline__ X scaled(X x, float f, bool up) {
  if (f == 0.f || x == 0) return 0;
  int e;
  const uint64_t m = (uint64_t)(frexpf(f, &e) * 16777216.f);   // f = m 2^(e - 24)
  const int shift = 24 - e;                                      // at least 24
  if (shift >= 96) return up ? 1 : 0;
  return (X)(((Sum)x * m + (up ? ((Sum)1 << shift) - 1 : 0)) >> shift);
}
__device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ Sum warp_sum(Sum v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    v += (Sum)__shfl_xor_sync(0xffffffffu, (uint32_t)(v >> 64), d) << 64 | __shfl_xor_sync(0xffffffffu, (uint64_t)v, d);
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
  // the largest of them, NaN aside
  static __device__ __forceinline__ float largest(const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
      return fmaxf(fmaxf(at(v, 0), at(v, 1)), fmaxf(at(v, 2), at(v, 3)));
    } else if constexpr (std::is_same_v<T, __half>) {
      __half2 m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = *reinterpret_cast<const __half2*>(&w[i]);
      const __half2 x = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
      return fmaxf(__low2float(x), __high2float(x));
    } else {
      __nv_bfloat162 m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
      const __nv_bfloat162 x = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
      return fmaxf(__low2float(x), __high2float(x));
    }
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

// Sorts the first n of v, a power of two of at most two a thread, by one CTA:
// falling or rising.  Exchanges over at most 32 places stay within a warp's 64
// items, in registers.
__device__ __forceinline__ void sort_items(unsigned long long* v, uint32_t n, bool falling) {
  const uint32_t t = threadIdx.x;
  const bool have = t < n / 2, idle = (t & ~31u) >= n / 2;   // (a whole warp without items only meets the others)
  __syncthreads();
  unsigned long long x[2] = {0, 0};
  if (have) x[0] = v[2 * t], x[1] = v[2 * t + 1];
  for (uint32_t size = 2; size <= n; size *= 2)
    for (uint32_t step = size / 2; step > 0; step /= 2) {
      unsigned long long y[2];                 // the items at step's distance
      if (step >= 64) {
        __syncthreads();                       // read by all before it is written again
        if (have) v[2 * t] = x[0], v[2 * t + 1] = x[1];
        __syncthreads();
        y[0] = have ? v[(2 * t) ^ step] : 0;
        y[1] = have ? v[(2 * t + 1) ^ step] : 0;
      } else if (idle) {
        continue;
      } else if (step >= 2) {
        y[0] = __shfl_xor_sync(0xffffffffu, x[0], step / 2);
        y[1] = __shfl_xor_sync(0xffffffffu, x[1], step / 2);
      } else {
        y[0] = x[1];
        y[1] = x[0];
      }
#pragma unroll
      for (uint32_t j = 0; j < 2; ++j) {
        const uint32_t i = 2 * t + j;
        const bool larger = ((i & step) == 0) == (((i & size) == 0) == falling);
        x[j] = (x[j] > y[j]) == larger ? x[j] : y[j];
      }
    }
  __syncthreads();
  if (have) v[2 * t] = x[0], v[2 * t + 1] = x[1];
  __syncthreads();
}
__device__ const float EXP_HI[32] = {RO_EXP_HI}, EXP_LO[32] = {RO_EXP_LO};

// What a row's tokens have to pass: keys above `key`, and the first `ties` equal to it.
struct Threshold {
  uint32_t key, ties;
};

// Candidates held, two a thread; tokens they are meant to hold where top-k does
// not say (with min-p, for top-p alone), and at most.
constexpr uint32_t SM_LIST = 2 * SM_THREADS, SM_WANT_MIN = 512, SM_WANT = 256, SM_WANT_MOST = 704;
// Maxima of a thread at most, each over every so-many-th of its blocks: the parts
// that hold candidates are read again.  (Of a row's own CTA eight: 256 rows of
// 131,072, top-p at 0.4, 147 us with two, 105 with eight.  Of a cluster's two,
// whose threads have a few blocks in shared memory: one row of 32,000 13.5 against 14.7.)
constexpr uint32_t SM_PARTS = 8;
static_assert(2 * SM_LIST <= SM_BINS, "candidates and their weights lie where the bins do");
constexpr uint32_t SM_COARSE = SM_THREADS;   // bins of the threads' maxima
// What a sum of weights in 32 bits may be off, relative to itself: a weight's
// argument, below 64, by three roundings, 2^-17; its exponential by 2^-22; the at
// most 220 sums that it goes into, by 2^-24 each; where a sum is scaled to a larger
// logit, at most 25 times, the factors by 2^-22 and 2^-24 each: 2^-15.1.
constexpr float SM_SLACK = 1.f / (1 << 15);
enum SampleWay : uint32_t { WAY_DONE, WAY_MASS, WAY_WIDE };
constexpr uint32_t QUEUE_WIDE = 0x80000000u;   // beside a queued row: WAY_WIDE

struct __align__(16) SampleShared {
  unsigned long long mass[SM_BINS];
  uint32_t count[SM_BINS];
  unsigned long long warp_mass[SM_WARPS], warp_above[SM_WARPS];
  uint32_t warp_ties[SM_WARPS], warp_count[SM_WARPS], warp_above_count[SM_WARPS];
  uint32_t border_ties[SM_WARPS];          // tokens on top-p's border in the warps' runs
  unsigned long long scan[SM_WARPS], scan_high[SM_WARPS];
  Sum left;                                // of what is wanted, on the border found
  unsigned long long list_sum;             // of the listed ones' weights, as far as they count
  uint32_t found;
  uint32_t best, least;                    // keys of the largest logit, and of the threads' smallest maximum
  uint32_t place;                          // of the largest logit, the first of equal ones
  uint32_t coarse[SM_COARSE];              // the threads' maxima, counted by distance from the largest
  uint32_t cut, listed, way, row;
  uint32_t counts[SM_MAX_CLUSTER];         // what each CTA has listed
  Threshold border;
  uint4 edge[2];                           // a row's first and last block, where it does not fill them
  struct {
    uint32_t first, last;
    uint64_t ties;                         // tokens on the threshold and weight before it
    Sum at;
  } run;
  float rough, warp_rough[SM_WARPS];       // sums of weights in 32 bits
  uint8_t flags[SM_WARPS][32 * SM_PARTS];  // parts of a warp's threads that hold a candidate
  float temperature, top_p, min_p, u;
  uint32_t top_k, valid;
  double reach;                            // how far below the largest logit min-p reaches
};

// One row, by a cluster of a.cluster CTAs (or one).  WIDE: whatever its
// settings; else, unless the way is WAY_DONE, it is left to others.  known_wide:
// not by its candidates.
template <typename T, bool WIDE>
__device__ __forceinline__ uint32_t sample_row(const SampleArgs& a, SampleShared& s, uint4* slice, uint32_t row, bool known_wide) {
  constexpr uint32_t E = Logits<T>::E, PARTS = WIDE ? 2 : SM_PARTS;
  // the low bits of a 16-bit logit's key follow from its sign
  constexpr int LOW = std::is_same_v<T, float> ? 0 : std::is_same_v<T, __half> ? 11 : 16;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t nc = a.cluster, rank = nc > 1 ? cluster_rank() : 0;
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
  // Block i of this CTA's.  The first and the last one of a row, which may hold
  // other data beside it, are kept with -inf there; [in0, in1) are whole.
  const uint32_t in0 = b0 == 0 && off != 0 ? 1u : 0u, in1 = b0 + n == n_blocks && end % E != 0 ? max(n, 1u) - 1u : n;
  auto block = [&](uint32_t i) -> uint4 {
    if (a.staged) return slice[i];
    return i >= in0 && i < in1 ? blocks[b0 + i] : s.edge[b0 + i == 0 ? 0 : 1];
  };
  if (tid == 0) {
    s.temperature = a.temperature ? a.temperature[row] : 1.f;
    s.top_p = a.top_p ? a.top_p[row] : 1.f;
    s.min_p = a.min_p ? a.min_p[row] : 0.f;
    s.top_k = a.top_k ? a.top_k[row] : 0u;
    s.u = a.u[row];
    s.valid = s.temperature >= 0.f && s.temperature < INFINITY && s.top_p >= 0.f && s.top_p <= 1.f && s.min_p >= 0.f &&
              s.min_p <= 1.f && s.u >= 0.f && s.u < 1.f;
    if (!s.valid && rank == 0) record(a.err, ERR_INVAL);
    s.listed = 0;
    s.place = ~0u;
    // (64-bit floats in one thread only, while the loads are under way: they are
    // rare on this GPU; all 512 threads' logarithms took 10 us)
    s.reach = s.min_p > 0.f ? (double)s.temperature * log((double)s.min_p) : 0.0;
  }
  s.coarse[tid] = 0;
  // ---- the slice, its largest logits, and where top-p will ask for it the sum of
  // the weights in 32 bits, relative to the largest logit that the thread has met
  // (a cluster, whose slices lie in shared memory, sums when the largest is known:
  // this pass is then 0.6 us shorter for the rows that need no sum) ----
  float my_top[PARTS];
#pragma unroll
  for (uint32_t h = 0; h < PARTS; ++h) my_top[h] = -INFINITY;
  float met = -INFINITY, met_sum = 0.f;
  const float per_unit = fminf(1.44269504f / (a.temperature ? a.temperature[row] : 1.f), 3.0e38f);
  const uint32_t k_asked = a.top_k ? a.top_k[row] : 0u;
  const bool rough_asked = !WIDE && a.top_p && a.top_p[row] < 1.f && (k_asked == 0u || k_asked >= a.vocab);
  auto meet = [&](float largest) {
    if (largest > met) {
      met_sum *= ex2((met - largest) * per_unit);
      met = largest;
    }
  };
  auto add_met = [&](const uint4& v) {
    float part[2] = {0.f, 0.f};
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) {
      const float z = (met - Logits<T>::at(v, k)) * per_unit;
      part[k & 1] += z < 64.f ? ex2(-z) : 0.f;   // (a NaN is not below)
    }
    met_sum += part[0] + part[1];
  };
  uint4 none;
  {
    __align__(16) T e[E];
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) e[k] = minus_infinity<T>();
    none = *(const uint4*)e;
  }
  constexpr uint32_t AHEAD = 8;   // loads of a thread under way
  for (uint32_t i = tid; i < n; i += AHEAD * SM_THREADS) {
    uint4 v[AHEAD];
#pragma unroll
    for (uint32_t q = 0; q < AHEAD; ++q) {
      const uint32_t j = i + q * SM_THREADS;
      v[q] = j >= in0 && j < in1 ? blocks[b0 + j] : none;
    }
#pragma unroll
    for (uint32_t q = 0; q < AHEAD; ++q) {
      const uint32_t j = i + q * SM_THREADS;
      if (a.staged && j >= in0 && j < in1) slice[j] = v[q];
      my_top[q % PARTS] = fmaxf(my_top[q % PARTS], Logits<T>::largest(v[q]));
    }
    if (rough_asked) {
      float largest = my_top[0];
#pragma unroll
      for (uint32_t h = 1; h < PARTS; ++h) largest = fmaxf(largest, my_top[h]);
      meet(largest);
#pragma unroll
      for (uint32_t q = 0; q < AHEAD; ++q) add_met(v[q]);
    }
  }
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h) {   // a block at the row's edge, by the thread that has it
    const uint32_t i = h == 0 ? 0u : n - 1u;
    if (n == 0u || (h == 0 ? in0 == 0u : in1 == n || (n == 1u && in0 != 0u)) || i % SM_THREADS != tid) continue;
    const uint32_t p0 = (b0 + i) * E;
    __align__(16) T e[E];
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) e[k] = p0 + k >= off && p0 + k < end ? x[p0 + k - off] : minus_infinity<T>();
    const uint4 v = *(const uint4*)e;
    if (a.staged)
      slice[i] = v;
    else
      s.edge[b0 + i == 0 ? 0 : 1] = v;
    const float largest = Logits<T>::largest(v);
#pragma unroll
    for (uint32_t q = 0; q < PARTS; ++q)
      if (q == i / SM_THREADS % PARTS) my_top[q] = fmaxf(my_top[q], largest);
    if (rough_asked) {
      meet(largest);
      add_met(v);
    }
  }
  {
    float largest = -INFINITY, smallest = INFINITY;
#pragma unroll
    for (uint32_t h = 0; h < PARTS; ++h) {
      largest = fmaxf(largest, my_top[h]);
      if (my_top[h] > -INFINITY) smallest = fminf(smallest, my_top[h]);
    }
    uint32_t low = largest > -INFINITY ? logit_key(smallest) : ~0u;
    const uint32_t hi = __reduce_max_sync(0xffffffffu, logit_key(largest));
    low = __reduce_min_sync(0xffffffffu, low);
    if (lane == 0) {
      s.warp_count[warp] = hi;
      s.warp_ties[warp] = low;
    }
  }
  __syncthreads();
  uint32_t best = __reduce_max_sync(0xffffffffu, lane < SM_WARPS ? s.warp_count[lane] : 0u);
  uint32_t least = __reduce_min_sync(0xffffffffu, lane < SM_WARPS ? s.warp_ties[lane] : ~0u);
  if (nc > 1) {
    if (tid == 0) {
      s.best = best;
      s.least = least;
    }
    cluster_sync();
    // (a lane each of the others': one after the other costs a round trip each)
    best = __reduce_max_sync(0xffffffffu, lane < nc ? cluster_read(&s.best, lane) : 0u);
    least = __reduce_min_sync(0xffffffffu, lane < nc ? cluster_read(&s.least, lane) : ~0u);
  } else {
    __syncthreads();   // read by all before they are written again
  }
  const float top = key_logit(best), T_ = s.temperature, top_p = s.top_p;
  const uint32_t top_k = s.top_k;
  auto finish = [&](uint32_t token, float logp, uint32_t kept) {
    a.token[row] = token;
    if (a.logp) a.logp[row] = logp;
    if (a.kept) a.kept[row] = kept;
  };
  if (!s.valid || best == KEY_NONE) {
    if (rank == 0 && tid == 0) finish(NO_TOKEN, -INFINITY, 0);
    return WAY_DONE;
  }
  if (T_ == 0.f || top_k == 1u || top_p == 0.f) {   // the first of the largest
    uint32_t place = ~0u;
#pragma unroll
    for (uint32_t h = 0; h < PARTS; ++h)
      if (my_top[h] == top) {
        uint32_t first = ~0u;
        for (uint32_t i = tid + h * SM_THREADS; i < n && first == ~0u; i += PARTS * SM_THREADS) {
          const uint4 v = block(i);
#pragma unroll
          for (uint32_t k = E; k-- > 0;)
            if (Logits<T>::at(v, k) == top) first = (b0 + i) * E + k - off;
        }
        place = min(place, first);
      }
    if (place != ~0u) atomicMin(&s.place, place);
    sync();
    if (rank == 0) {
      if (lane < nc && warp == 0) place = nc > 1 ? cluster_read(&s.place, lane) : s.place;
      place = __reduce_min_sync(0xffffffffu, warp == 0 && lane < nc ? place : ~0u);
      if (tid == 0) finish(place, 0.f, 1);
    }
    return WAY_DONE;
  }

  // ---- weights ----
  const ExpScale scale = exp_scale(T_);
  // Weights in 32 bits have one factor.  Below T = 5e-39 it is too small: they are
  // then bounds of the weights, and decide nothing.
  const bool rough_holds = per_unit < 3.0e38f;
  const float my_hi = EXP_HI[lane], my_lo = EXP_LO[lane];   // the table, an entry a lane
  // Every weight has the same bits behind the point, whatever the row's sum and
  // whoever takes it, so a draw does not depend on how the row is split.
  constexpr float ONE = (float)(1ull << WEIGHT_BITS);
  // Of a whole warp's logits, some a lane; 0 where !in.  (Up to four together:
  // one after another each would wait for its chain of some 60 instructions.)
  auto weigh = [&](auto& y, auto& in, auto& w) {
    constexpr int N = (int)(sizeof(y) / sizeof(y[0])), G = N < 4 ? N : 4;
#pragma unroll
    for (int g = 0; g < N; g += G) {
      bool some = false;
#pragma unroll
      for (int k = 0; k < G; ++k) {
        some = some || in[g + k];
        w[g + k] = {0, 0};
      }
      if (!__any_sync(0xffffffffu, some)) continue;
#pragma unroll
      for (int k = 0; k < G; ++k) {
        const Weight v = exp_weight(exp_argument(top, in[g + k] ? y[g + k] : top, scale), ONE, [&](uint32_t j) {
          return Pair32{__shfl_sync(0xffffffffu, my_hi, j), __shfl_sync(0xffffffffu, my_lo, j)};
        });
        if (in[g + k]) w[g + k] = v;
      }
    }
  };
  auto weight = [&](float y, bool in) -> uint64_t {
    const float ys[1] = {y};
    const bool ins[1] = {in};
    Weight w[1];
    weigh(ys, ins, w);
    return whole(w[0], WEIGHT_BITS);
  };
  auto total_of = [&](const auto& w) -> uint64_t {   // of a few
    Weight m = {0, 0};
#pragma unroll
    for (uint32_t k = 0; k < sizeof(w) / sizeof(w[0]); ++k) {
      m.hi += w[k].hi;
      m.lo += w[k].lo;
    }
    return whole(m, WEIGHT_BITS);
  };
  // in 32 bits, of a logit that is no NaN
  auto rough_weight = [&](float y) -> float {
    const float z = (top - y) * per_unit;
    return z < 64.f ? ex2(-z) : 0.f;
  };
  auto key_of = [&](float y) -> uint32_t { return y == y ? logit_key(y) : KEY_NONE; };   // (a NaN is never drawn)
  auto each_block = [&](auto&& use) {              // several loads at a time
    for (uint32_t i = tid; i < n; i += 4 * SM_THREADS) {
      uint4 v[4];
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) v[q] = i + q * SM_THREADS < n ? block(i + q * SM_THREADS) : none;
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) use(v[q]);
    }
  };
  // a thread's 32-bit sum: the CTA's is in s.rough once the CTA has met
  auto rough_of = [&](float sum) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) s.warp_rough[warp] = sum;
    __syncthreads();
    if (tid == 0) {
      sum = 0.f;
      for (uint32_t w = 0; w < SM_WARPS; ++w) sum += s.warp_rough[w];
      s.rough = sum;
    }
  };
  auto rough_sum = [&](float above) {
    float sum = 0.f;
    each_block([&](const uint4& v) {
      float part[2] = {0.f, 0.f};
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        const float y = Logits<T>::at(v, k), w = rough_weight(y);
        part[k & 1] += y > above ? w : 0.f;
      }
      sum += part[0] + part[1];
    });
    rough_of(sum);
  };
  // of all, from what was met
  auto rough_met = [&] {
    if constexpr (WIDE)
      rough_sum(-INFINITY);
    else
      rough_of(met < top ? met_sum * ex2((met - top) * per_unit) : met_sum);
  };
  auto rough_total = [&]() -> float {
    if (nc == 1) return s.rough;
    const float part = lane < nc ? __uint_as_float(cluster_read((const uint32_t*)&s.rough, lane)) : 0.f;
    float sum = 0.f;
    for (uint32_t r = 0; r < nc; ++r) sum += __shfl_sync(0xffffffffu, part, r);
    return sum;
  };
  auto with_log = [&](uint32_t token, float y, double total, uint32_t kept) {
    const Pair32 z = exp_argument(top, y, scale);
    const double less = ((double)z.hi + (double)z.lo) * 0.69314718055994530942;
    finish(token, -(float)(less + log(total * (1.0 / (double)(1ull << WEIGHT_BITS)))), kept);
  };

  // ---- thresholds ----
  Threshold th = {KEY_NONE, 0};
  if (s.min_p > 0.f) {   // w >= min_p; the smallest such float
    const float least_x = __double2float_ru((double)top + s.reach);
    th.key = max(KEY_NONE, logit_key(least_x) - 1u);
    // (as a number -0 is 0, which has to lie above the threshold; no logit has its key)
    if (th.key == KEY_MINUS_ZERO) th.key = KEY_MINUS_ZERO - 1u;
  }
  const bool by_k = top_k != 0u && top_k < a.vocab, by_p = top_p < 1.f, by_min = s.min_p > 0.f;
  // (as far as weights go: beyond 45 T they are below 2^-64)
  const float span = fmaxf(fminf(top - key_logit(least), 45.f * T_), 1e-30f);
  unsigned long long* list = s.mass;              // candidates: keys and ~indices
  unsigned long long* weights = s.mass + SM_LIST;
  // To the CTA's list, by a whole warp: the logits whose bits are set in `hits`;
  // index(b): of bit b's.
  auto enlist = [&](uint32_t hits, auto&& index) {
    if (!__any_sync(0xffffffffu, hits != 0u)) return;
    const uint32_t mine = __popc(hits), inc = warp_incl_scan(mine);
    uint32_t at = 0;
    if (lane == 31) at = atomicAdd(&s.listed, inc);
    at = __shfl_sync(0xffffffffu, at, 31) + inc - mine;
    for (; hits != 0u; hits &= hits - 1u, ++at) {
      const uint32_t i = index((uint32_t)__ffs(hits) - 1u);
      const T y = a.staged ? ((const T*)slice)[i + off - b0 * E] : x[i];
      if (at < SM_LIST) list[at] = (unsigned long long)logit_key((float)y) << 32 | ~i;
    }
  };
  // The first CTA, when all have met: everyone's list behind its own, and how many are
  // listed.  (Placed from afar, on one counter, a row's thousand took 17,000 cycles more.)
  auto all_listed = [&](bool counted) -> uint32_t {   // counted: s.counts is written
    if (nc == 1) return s.listed;
    const uint32_t theirs = lane >= nc ? 0u : counted ? s.counts[lane] : cluster_read(&s.listed, lane);
    const uint32_t end = warp_incl_scan(theirs), all = __shfl_sync(0xffffffffu, end, 31);
    if (all > SM_LIST) return all;
    for (uint32_t i0 = __shfl_sync(0xffffffffu, end, 0); i0 < all; i0 += SM_THREADS) {
      const uint32_t i = i0 + tid;
      uint32_t r = 0, before = 0;
      for (uint32_t q = 0; q < nc; ++q) {
        const uint32_t x = __shfl_sync(0xffffffffu, end, q);
        if (x <= i) r = q + 1, before = x;
      }
      if (i < all) list[i] = cluster_read(&list[i - before], r);
    }
    __syncthreads();
    return all;
  };
  // The first CTA: sorts what is listed; the weights of this thread's two items
  // and of those ahead of them; returns all their weight.
  uint64_t own[2] = {0, 0}, ahead[2] = {0, 0};
  auto sort_list = [&](uint32_t listed) -> uint64_t {
    uint32_t size = 2;
    while (size < listed) size *= 2;
    for (uint32_t i = listed + tid; i < size; i += SM_THREADS) list[i] = 0;
    sort_items(list, size, true);
    const float ys[2] = {key_logit((uint32_t)(list[2 * tid] >> 32)), key_logit((uint32_t)(list[2 * tid + 1] >> 32))};
    const bool ins[2] = {2 * tid < listed, 2 * tid + 1 < listed};
    Weight w[2];
    weigh(ys, ins, w);
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
      own[j] = whole(w[j], WEIGHT_BITS);
      if (ins[j]) weights[2 * tid + j] = own[j];
    }
    const uint64_t sum = own[0] + own[1];
    const uint64_t run = warp_incl_scan(sum);
    if (lane == 31) s.scan[warp] = run;
    __syncthreads();
    uint64_t base = run - sum, all = 0;
    for (uint32_t w = 0; w < SM_WARPS; ++w) {
      if (w < warp) base += s.scan[w];
      all += s.scan[w];
    }
    ahead[0] = base;
    ahead[1] = base + own[0];
    return all;
  };
  // how many of the first `first` items have less than `limit` ahead of them
  auto count_below = [&](uint64_t limit, uint32_t first) -> uint32_t {
    const uint32_t mine = (2 * tid < first && ahead[0] < limit) + (2 * tid + 1 < first && ahead[1] < limit);
    return (uint32_t)__syncthreads_count(mine >= 1) + (uint32_t)__syncthreads_count(mine >= 2);
  };

  // ---- few candidates ----
  uint32_t way = WAY_WIDE;
  if ((by_k || by_p || by_min) && top < INFINITY && !known_wide) {
    const bool all_of_k = by_k && top_k <= SM_WANT_MOST;   // the candidates hold the first top_k
    const uint32_t want = all_of_k ? top_k : by_min ? SM_WANT_MIN : SM_WANT;
    const float per_bin = (float)SM_COARSE / span;
    auto bin_of = [&](float y) { return (uint32_t)fminf((top - y) * per_bin, (float)(SM_COARSE - 1)); };
#pragma unroll
    for (uint32_t h = 0; h < PARTS; ++h)
      if (my_top[h] > -INFINITY) atomicAdd(&s.coarse[bin_of(my_top[h])], 1u);
    // the sum that top-p is a share of, first in 32 bits
    if (by_p && !by_k) rough_met();
    if (tid == 0) s.cut = SM_COARSE;
    sync();
    // the bin at which `want` maxima are reached is the last that is listed
    uint32_t mine = 0;
    if (nc > 1) {
      uint32_t v[SM_MAX_CLUSTER];
#pragma unroll
      for (uint32_t r = 0; r < SM_MAX_CLUSTER; ++r) v[r] = r < nc ? cluster_read(&s.coarse[tid], r) : 0u;
#pragma unroll
      for (uint32_t r = 0; r < SM_MAX_CLUSTER; ++r) mine += v[r];
    } else {
      mine = s.coarse[tid];
    }
    const uint32_t inc = warp_incl_scan(mine);
    if (lane == 31) s.warp_count[warp] = inc;
    __syncthreads();
    uint32_t before = inc - mine;
    for (uint32_t w = 0; w < warp; ++w) before += s.warp_count[w];
    if (before < want && before + mine >= want) s.cut = tid;
    __syncthreads();
    const uint32_t cut = s.cut;                      // SM_COARSE: fewer maxima than wanted, so every token
    const bool with_min = by_min && !all_of_k;       // (top-p's sum is over the first top_k, whatever min-p says)
    // (bin_of(y) <= cut, without its conversion)
    const float reach = (float)(cut + 1), limit = with_min ? key_logit(th.key) : -INFINITY;
    const bool far = cut >= SM_COARSE - 1;
    auto candidate = [&](float y) { return y > limit && (far || (top - y) * per_bin < reach); };
    // A warp goes through the blocks of those of its threads' parts whose maximum is one, several at a time.
    uint8_t* flags = s.flags[warp];
    uint32_t flagged = 0;
#pragma unroll
    for (uint32_t h = 0; h < PARTS; ++h) {
      const bool flag = candidate(my_top[h]);
      const uint32_t all = __ballot_sync(0xffffffffu, flag);
      if (flag) flags[flagged + __popc(all & ((1u << lane) - 1u))] = (uint8_t)(lane | h << 5);
      flagged += __popc(all);
    }
    __syncwarp();
    const uint32_t runs = (n + PARTS * SM_THREADS - 1) / (PARTS * SM_THREADS), visits = flagged * runs;
    for (uint32_t x0 = 0; x0 < visits; x0 += 4 * 32) {
      uint4 v[4];
      uint32_t at[4];
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        const uint32_t visit = x0 + q * 32 + lane, f = visit / runs;
        at[q] = n;
        if (visit < visits)
          at[q] = warp * 32 + (flags[f] & 31u) + ((flags[f] >> 5) + (visit - f * runs) * PARTS) * SM_THREADS;
        v[q] = at[q] < n ? block(at[q]) : none;
      }
      uint32_t hits = 0;
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) hits |= candidate(Logits<T>::at(v[q], k)) ? 1u << (q * E + k) : 0u;
      static_assert(4 * E <= 32, "a bit a logit");
      enlist(hits, [&](uint32_t b) {
        const uint32_t q = b / E, i = q < 2u ? (q == 0u ? at[0] : at[1]) : (q == 2u ? at[2] : at[3]);
        return (b0 + i) * E + b % E - off;
      });
    }
    if (nc > 1) {
      __syncthreads();
      if (tid == 0) cluster_write(&s.counts[rank], 0, s.listed);
    }
    sync();
    // ---- the first CTA's ----
    const uint32_t listed = rank == 0 ? all_listed(true) : 0;
    uint32_t stay = 0;
    if (rank == 0) {
      // Where the listed ones' weights add up to less than top-p's share, more tokens stay: nothing to sort.
      bool short_of = false;
      if (by_p && !by_k && !by_min && cut != SM_COARSE && listed <= SM_LIST) {
        float sum = 0.f;
        for (uint32_t i = tid; i < listed; i += SM_THREADS) sum += rough_weight(key_logit((uint32_t)(list[i] >> 32)));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) s.warp_rough[warp] = sum;
        __syncthreads();
        sum = 0.f;
        for (uint32_t w = 0; w < SM_WARPS; ++w) sum += s.warp_rough[w];
        short_of = !rough_holds || sum * (1.f + SM_SLACK) < rough_total() * top_p * (1.f - SM_SLACK);
      }
      if (listed > 0 && listed <= SM_LIST && !short_of) {
        const uint64_t list_mass = sort_list(listed);
        uint32_t by_limit = listed;                  // min-p's
        if (by_min) {
          const uint32_t in = (2 * tid < listed && (uint32_t)(list[2 * tid] >> 32) > th.key) +
                              (2 * tid + 1 < listed && (uint32_t)(list[2 * tid + 1] >> 32) > th.key);
          by_limit = (uint32_t)__syncthreads_count(in >= 1) + (uint32_t)__syncthreads_count(in >= 2);
        }
        // whether every token that can stay by top-k and min-p is listed
        const bool whole = cut == SM_COARSE || all_of_k || by_limit < listed ||
                           (with_min && bin_of(key_logit(th.key + 1u)) <= cut);
        const uint32_t first = by_k ? min(top_k, listed) : listed;
        stay = min(first, by_limit);
        if (!by_p) {
          way = whole ? WAY_DONE : WAY_WIDE;
        } else if (all_of_k || (cut == SM_COARSE && !with_min)) {   // the sum is the listed ones'
          uint64_t sum = list_mass;
          if (first < listed) {
            if (tid == first / 2) s.list_sum = ahead[first & 1];
            __syncthreads();
            sum = s.list_sum;
          }
          stay = min(stay, max(1u, count_below(scaled(sum, top_p, true), first)));
          way = WAY_DONE;
        } else if (!by_k && rough_holds) {
          const float rough = fminf(rough_total() * top_p * ONE, 0x1p62f);   // (more than the listed ones' sum)
          const uint32_t lo = max(1u, count_below((uint64_t)(rough * (1.f - SM_SLACK)), listed));
          const uint32_t hi = max(1u, count_below((uint64_t)(rough * (1.f + SM_SLACK)) + 2, listed));
          if (!whole && hi == listed) {              // tokens that are not listed may stay
            way = WAY_WIDE;
          } else if (min(lo, stay) == min(hi, stay)) {
            way = WAY_DONE;
            stay = min(lo, stay);
          } else {
            way = WAY_MASS;
          }
        }
      }
      if (tid < nc) {   // to every CTA's own: this one may be gone before they look
        if (nc > 1)
          cluster_write(&s.way, tid, way);
        else
          s.way = way;
      }
    }
    sync();
    way = s.way;
    if (way == WAY_DONE || (WIDE && way == WAY_MASS)) {
      if (way == WAY_MASS) {   // the border lies within what 32 bits may be off
        uint64_t mine = 0;
        for (uint32_t i = warp * 32; i < n; i += SM_THREADS) {
          const bool have = i + lane < n;
          const uint4 v = have ? block(i + lane) : make_uint4(0, 0, 0, 0);
          float y[E];
          bool in[E];
          Weight w[E];
#pragma unroll
          for (uint32_t k = 0; k < E; ++k) {
            y[k] = Logits<T>::at(v, k);
            in[k] = have && y[k] > -INFINITY;
          }
          weigh(y, in, w);
          mine += total_of(w);
        }
        mine = warp_sum64(mine);
        if (lane == 0) s.warp_mass[warp] = mine;
        sync();
        Sum sum = 0;
        for (uint32_t q = lane; q < nc * SM_WARPS; q += 32)
          sum += nc > 1 ? cluster_read(&s.warp_mass[q % SM_WARPS], q / SM_WARPS) : s.warp_mass[q % SM_WARPS];
        sum = scaled(warp_sum(sum), top_p, true);
        const uint64_t share = sum >> 62 != 0 ? 1ull << 62 : (uint64_t)sum;   // (that is more than the listed ones' sum)
        if (rank == 0) stay = min(stay, max(1u, count_below(share, listed)));
        sync();
      }
      if (rank == 0) {
        // the sum of those that stay, then where it passes the goal, by index
        if (2 * tid < stay && stay <= 2 * tid + 2) s.list_sum = ahead[(stay - 1) & 1] + own[(stay - 1) & 1];
        __syncthreads();
        const uint64_t total = s.list_sum, goal = scaled(total, s.u, false);
        uint32_t size = 2;
        while (size < stay) size *= 2;
        // indices rise, and each remembers its candidate
        unsigned long long* order = (unsigned long long*)s.count;
        static_assert(SM_LIST * 8 <= sizeof(s.count), "the order lies where the counts do");
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
          const uint32_t i = 2 * tid + j;
          if (i < size) order[i] = i < stay ? (unsigned long long)~(uint32_t)list[i] << 32 | i : ~0ull;
        }
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
            with_log((uint32_t)(o >> 32), key_logit((uint32_t)(list[(uint32_t)o] >> 32)), (double)total, stay);
          }
          at += w2[j];
        }
      }
      return WAY_DONE;
    }
  }
  if constexpr (!WIDE) {
    return way;
  } else {
  // ---- wide rows ----
  const uint32_t rounds = (n + SM_THREADS - 1) / SM_THREADS;
  // Finds the key where the tokens above `th`, largest first, reach `want` (in
  // tokens or in weight), which they do: leaves the key and what is still wanted of it.
  auto select = [&](auto by_mass, Sum want, Sum* left) -> uint32_t {
    constexpr bool MASS = decltype(by_mass)::value;
    constexpr int HIGH = 38;   // a bin's weight in two parts: 2^12 of 2^38 a token at most
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
        const uint4 v = i < n ? block(i) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) {
          const float y = Logits<T>::at(v, k);
          const uint32_t key = key_of(y);
          const bool in = i < n && key > th.key && (key & mask) == prefix;
          if constexpr (MASS) {
            const uint64_t w = weight(y, in);
            if (in && w) {
              atomicAdd(&s.mass[(key >> shift) & (bins - 1)], (unsigned long long)w & ((1ull << HIGH) - 1));
              atomicAdd(&s.count[(key >> shift) & (bins - 1)], (uint32_t)(w >> HIGH));
            }
          } else {
            if (in) atomicAdd(&s.count[(key >> shift) & (bins - 1)], 1u);
          }
        }
      }
      sync();
      // a thread sums its bins over the cluster, largest keys first
      const uint32_t each = max(1u, bins / SM_THREADS);
      uint64_t low[SM_BINS / SM_THREADS], low_sum = 0;
      uint32_t high[SM_BINS / SM_THREADS], high_sum = 0;   // (tokens, where those count)
#pragma unroll
      for (uint32_t j = 0; j < SM_BINS / SM_THREADS; ++j) {
        low[j] = 0;
        high[j] = 0;
        const uint32_t d = tid * each + j;
        if (j < each && d < bins) {
          const uint32_t bin = bins - 1 - d;
          for (uint32_t q = 0; q < nc; ++q) {
            if constexpr (MASS) low[j] += nc > 1 ? cluster_read(&s.mass[bin], q) : s.mass[bin];
            high[j] += nc > 1 ? cluster_read(&s.count[bin], q) : s.count[bin];
          }
        }
        low_sum += low[j];
        high_sum += high[j];
      }
      const uint64_t low_inc = warp_incl_scan(low_sum);
      const uint32_t high_inc = warp_incl_scan(high_sum);
      if (lane == 31) {
        s.scan[warp] = low_inc;
        s.scan_high[warp] = high_inc;
      }
      __syncthreads();
      uint64_t low_before = low_inc - low_sum, high_before = high_inc - high_sum;
      for (uint32_t q = 0; q < warp; ++q) {
        low_before += s.scan[q];
        high_before += s.scan_high[q];
      }
      auto both = [&](uint64_t h, uint64_t l) -> Sum { return MASS ? ((Sum)h << HIGH) + l : (Sum)h; };
      Sum before = both(high_before, low_before);
#pragma unroll
      for (uint32_t j = 0; j < SM_BINS / SM_THREADS; ++j) {
        const Sum upto = before + both(high[j], low[j]);
        if (before < want && upto >= want) {
          s.found = bins - 1 - (tid * each + j);
          s.left = want - before;
        }
        before = upto;
      }
      sync();   // every CTA has read the others' bins
      prefix |= s.found << shift;
      mask |= (bins - 1) << shift;
      want = s.left;
      __syncthreads();
    }
    prefix |= (prefix & 0x80000000u) ? 0u : (1u << LOW) - 1u;   // a negative logit's low bits are ones
    *left = want;
    return prefix;
  };
  // Sums of what passes the threshold: over this warp's run of the slice, then over all before it.
  const uint32_t per = (n + SM_WARPS - 1) / SM_WARPS, i0 = min(n, warp * per), i1 = min(n, i0 + per);
  struct Sums {
    Sum mass, above, before;                     // of all; of the bins above the border's; before this warp:
    uint64_t ties_before;                        // weight above the threshold, tokens on it
    uint64_t ties, count, above_count;           // on it, above it, in the bins above the border's
    uint64_t own;                                // this warp's weight above it
    uint32_t own_ties;
  };
  // extra(v, in, index): those of a block whose weight counts as `above`, as bits
  auto sums = [&](auto weighed, auto&& extra) -> Sums {
    constexpr bool W = decltype(weighed)::value;
    const float limit = key_logit(th.key);
    uint64_t m = 0, up = 0;
    uint32_t on = 0, above = 0, up_count = 0;
    for (uint32_t i = i0; i < i1; i += 32) {
      const bool have = i + lane < i1;
      const uint4 v = have ? block(i + lane) : make_uint4(0, 0, 0, 0);
      float y[E];
      bool in[E];
      Weight w[E], more = {0, 0};
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        y[k] = Logits<T>::at(v, k);
        in[k] = have && y[k] > limit;
        above += in[k];
        on += have && y[k] == limit;
      }
      if constexpr (W) {
        weigh(y, in, w);
        m += total_of(w);
        const uint32_t over = extra(v, in, (b0 + i + lane) * E - off);
#pragma unroll
        for (uint32_t k = 0; k < E; ++k)
          if (over >> k & 1u) {
            more.hi += w[k].hi;
            more.lo += w[k].lo;
          }
        up += whole(more, WEIGHT_BITS);
        up_count += __popc(over);
      }
    }
    m = warp_sum64(m);
    up = warp_sum64(up);
    on = __reduce_add_sync(0xffffffffu, on);
    above = __reduce_add_sync(0xffffffffu, above);
    up_count = __reduce_add_sync(0xffffffffu, up_count);
    if (lane == 0) {
      s.warp_mass[warp] = m;
      s.warp_above[warp] = up;
      s.warp_above_count[warp] = up_count;
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
      const uint64_t wu = nc > 1 ? cluster_read(&s.warp_above[w], r) : s.warp_above[w];
      const uint32_t wt = nc > 1 ? cluster_read(&s.warp_ties[w], r) : s.warp_ties[w];
      const uint32_t wc = nc > 1 ? cluster_read(&s.warp_count[w], r) : s.warp_count[w];
      t.above_count += nc > 1 ? cluster_read(&s.warp_above_count[w], r) : s.warp_above_count[w];
      t.mass += wm;
      t.above += wu;
      t.ties += wt;
      t.count += wc;
      if (q < rank * SM_WARPS + warp) {
        t.before += wm;
        t.ties_before += wt;
      }
    }
    t.mass = warp_sum(t.mass);
    t.above = warp_sum(t.above);
    t.ties = warp_sum64(t.ties);
    t.count = warp_sum64(t.count);
    t.above_count = warp_sum64(t.above_count);
    t.before = warp_sum(t.before);
    t.ties_before = warp_sum64(t.ties_before);
    sync();   // read by all before it is written again
    return t;
  };
  auto nothing = [](const uint4&, const bool (&)[E], uint32_t) { return 0u; };
  auto cut_to_k = [&] {
    if (by_k && sums(std::false_type(), nothing).count > top_k) {
      Sum left;
      th.key = select(std::false_type(), top_k, &left);
      th.ties = (uint32_t)left;
    }
  };

  const Threshold cut = th;                 // min-p's
  if (by_p) th = {KEY_NONE, 0};             // (top-p's sum is over the first top_k, whatever min-p says)
  cut_to_k();
  Sums t = {};
  bool summed = false;     // t is of what passes th
  if (by_p) {
    const uint64_t tie = weight(key_logit(th.key), th.ties != 0u);
    // The border's bin, by weights in 32 bits: `bins` of equal width, whole
    // numbers that add up to about 2^31.
    // (the threads' smallest maximum lies about half-way to the least logit)
    const float per_bin = (float)SM_BINS / fminf(2.f * span, fmaxf(45.f * T_, 1e-30f));
    auto bin_of = [&](float y) { return (uint32_t)fminf((top - y) * per_bin, (float)(SM_BINS - 1)); };
    uint32_t border = SM_BINS;
    if (top < INFINITY) {
      const float limit = key_logit(th.key);
      // (of all tokens, the sum is known where candidates were looked for)
      if (th.key != KEY_NONE || by_k || known_wide) rough_sum(limit);
      for (uint32_t i = tid; i < SM_BINS; i += SM_THREADS) s.count[i] = 0;
      if (tid < SM_WARPS) s.border_ties[tid] = 0;
      if (tid == 0) {
        s.found = SM_BINS;
        s.listed = 0;
      }
      sync();
      const float sum_f = rough_total(), unit = 2147483648.f / sum_f;
      each_block([&](const uint4& v) {
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) {
          const float y = Logits<T>::at(v, k);
          if (y > limit) atomicAdd(&s.count[bin_of(y)], (uint32_t)fmaf(rough_weight(y), unit, 0.5f));
        }
      });
      sync();
      if (rank == 0) {   // the first CTA's alone: a bin of each of the others is a load from its shared memory
        constexpr uint32_t EACH = SM_BINS / SM_THREADS;
        static_assert(EACH == 4, "four bins a thread");
        uint64_t mine[EACH] = {}, sum = 0;
        for (uint32_t q0 = 0; q0 < nc; q0 += 4) {   // several at a time
          uint4 v[4];
#pragma unroll
          for (uint32_t q = 0; q < 4; ++q) {
            v[q] = make_uint4(0, 0, 0, 0);
            const uint32_t at = step_smem(&s.count[tid * EACH]);
            if (q0 + q < nc)
              asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];"
                           : "=r"(v[q].x), "=r"(v[q].y), "=r"(v[q].z), "=r"(v[q].w)
                           : "r"(nc > 1 ? cluster_at(at, q0 + q) : at)
                           : "memory");
          }
#pragma unroll
          for (uint32_t q = 0; q < 4; ++q) {
            mine[0] += v[q].x; mine[1] += v[q].y; mine[2] += v[q].z; mine[3] += v[q].w;
          }
        }
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) sum += mine[j];
        const uint64_t inc = warp_incl_scan(sum);
        if (lane == 31) s.scan[warp] = inc;
        __syncthreads();
        uint64_t before = inc - sum, all = 0;
        for (uint32_t q = 0; q < SM_WARPS; ++q) {
          if (q < warp) before += s.scan[q];
          all += s.scan[q];
        }
        const float ties_f = (float)tie * (float)th.ties / ONE * unit;
        const uint64_t want = max((uint64_t)1, (uint64_t)(((float)all + ties_f) * top_p));
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
          if (before < want && before + mine[j] >= want) s.found = tid * EACH + j;
          before += mine[j];
        }
        __syncthreads();
        if (tid < nc && nc > 1) cluster_write(&s.cut, tid, s.found);
        if (nc == 1 && tid == 0) s.cut = s.found;
      }
      sync();
      border = s.cut;
    }
    // exactly: all of it, what lies above the bin, and the bin's tokens
    // (bin_of(y) against the border, without its conversion)
    const float border_lo = (float)border, border_hi = border < SM_BINS - 1 ? border_lo + 1.f : INFINITY;
    t = sums(std::true_type(), [&](const uint4& v, const bool (&in)[E], uint32_t index) {
      uint32_t over = 0, hits = 0;
      if (border == SM_BINS) return over;
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        const float b = (top - Logits<T>::at(v, k)) * per_bin;
        over |= in[k] && b < border_lo ? 1u << k : 0u;
        hits |= in[k] && b >= border_lo && b < border_hi ? 1u << k : 0u;
      }
      enlist(hits, [&](uint32_t b) { return index + b; });
      return over;
    });
    const Sum want = scaled(t.mass + (Sum)tie * th.ties, top_p, true);
    // how many tokens of weight w, at least 1, it takes to reach x
    auto reach = [](Sum x, uint64_t w) -> uint32_t {
      uint32_t n = (uint32_t)(sum_float(x) / (float)w);   // one off at most
      while ((Sum)w * n < x) ++n;
      while (n > 0u && (Sum)w * (n - 1u) >= x) --n;
      return n;
    };
    if (want > t.mass) {
      th.ties = min(reach(want - t.mass, tie), th.ties);
    } else {
      if (rank == 0) {
        Threshold found = {0, 0};
        const uint32_t listed = all_listed(false);
        if (border != SM_BINS && want > t.above && listed > 0 && listed <= SM_LIST) {
          const uint64_t all = sort_list(listed);
          if (want <= t.above + all) {
            const uint32_t n_in = count_below((uint64_t)(want - t.above), listed);   // at least 1
            const uint32_t key = (uint32_t)(list[n_in - 1] >> 32);
            const uint32_t on = (2 * tid < n_in && (uint32_t)(list[2 * tid] >> 32) == key) +
                                (2 * tid + 1 < n_in && (uint32_t)(list[2 * tid + 1] >> 32) == key);
            found = {key, (uint32_t)__syncthreads_count(on >= 1) + (uint32_t)__syncthreads_count(on >= 2)};
            // What stays of the bin, to the sums of what lies above it, by the warps whose runs it is in.
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
              const unsigned long long item = 2 * tid + j < listed ? list[2 * tid + j] : 0;
              const bool tied = (uint32_t)(item >> 32) == key;
              if (2 * tid + j >= listed || (!tied && 2 * tid + j >= n_in)) continue;
              const uint32_t b = (~(uint32_t)item + off) / E, r = b / a.blocks;
              const uint32_t len = min(n_blocks, (r + 1) * a.blocks) - r * a.blocks;
              const uint32_t w = (b - r * a.blocks) / ((len + SM_WARPS - 1) / SM_WARPS);
              if (tied)
                cluster_add(&s.border_ties[w], r, nc, 1u);
              else
                cluster_add(&s.warp_above[w], r, nc, own[j]);
            }
            if (tid < nc) {
              if (nc > 1)
                cluster_write(&s.cut, tid, n_in - found.ties);
              else
                s.cut = n_in - found.ties;
            }
          }
        }
        if (tid < nc) {
          if (nc > 1) {
            cluster_write(&s.border.key, tid, found.key);
            cluster_write(&s.border.ties, tid, found.ties);
          } else {
            s.border = found;
          }
        }
      }
      sync();
      const Threshold found = s.border;
      if (found.ties != 0u) {
        th = found;
        summed = true;
        t.mass = t.before = t.ties_before = 0;
        for (uint32_t q = lane; q < nc * SM_WARPS; q += 32) {
          const uint32_t r = q / SM_WARPS, w = q % SM_WARPS;
          const uint64_t wm = nc > 1 ? cluster_read(&s.warp_above[w], r) : s.warp_above[w];
          const uint32_t wt = nc > 1 ? cluster_read(&s.border_ties[w], r) : s.border_ties[w];
          t.mass += wm;
          if (q < rank * SM_WARPS + warp) {
            t.before += wm;
            t.ties_before += wt;
          }
        }
        t.mass = warp_sum(t.mass);
        t.before = warp_sum(t.before);
        t.ties_before = warp_sum64(t.ties_before);
        t.own = s.warp_above[warp];
        t.own_ties = s.border_ties[warp];
        t.ties = found.ties;
        t.count = t.above_count + s.cut;
      } else {             // too many tokens in the bin, or 32 bits named a wrong one
        Sum left;
        const uint32_t key = select(std::true_type(), want, &left);
        th.key = key;
        th.ties = reach(left, weight(key_logit(key), true));
      }
    }
    if (cut.key > th.key || (cut.key == th.key && cut.ties < th.ties)) {
      th = cut;
      summed = false;
    }
  }

  // ---- the token ----
  if (!summed) t = sums(std::true_type(), nothing);
  const uint64_t tie = weight(key_logit(th.key), th.ties != 0u);
  const uint64_t ties = min((uint64_t)th.ties, t.ties);
  const Sum total = t.mass + (Sum)tie * ties;
  const Sum goal = scaled(total, s.u, false);   // the first running sum above it
  if (total == 0) {   // (the largest logit stays in every row: nothing has to be left unwritten all the same)
    if (rank == 0 && tid == 0) finish(NO_TOKEN, -INFINITY, 0);
    return WAY_DONE;
  }
  uint64_t ties_before = t.ties_before;
  Sum at = t.before + (Sum)tie * min(ties, ties_before);
  const Sum mine = t.own + (Sum)tie * (min(ties, ties_before + t.own_ties) - min(ties, ties_before));
  // The warp whose run has it shares the run with the CTA's other warps.
  const bool has = goal >= at && goal < at + mine;
  if (has && lane == 0) s.run = {i0, i1, ties_before, at};
  if (!__syncthreads_or(has)) return WAY_DONE;
  const uint32_t r1 = s.run.last, part = (r1 - s.run.first + SM_WARPS - 1) / SM_WARPS;
  const uint32_t j0 = min(r1, s.run.first + warp * part), j1 = min(r1, j0 + part);
  // a lane's weights of its block, those on the threshold aside, which `on` counts
  const float limit = key_logit(th.key);
  auto step = [&](uint32_t i, float (&y)[E], Weight (&w)[E], uint32_t* on) {
    const bool have = i + lane < j1;
    const uint4 v = have ? block(i + lane) : make_uint4(0, 0, 0, 0);
    bool in[E];
    *on = 0;
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) {
      y[k] = Logits<T>::at(v, k);
      in[k] = have && y[k] > limit;
      *on += have && y[k] == limit;
    }
    weigh(y, in, w);
  };
  float y[E];
  Weight w[E];
  uint64_t m = 0;
  uint32_t on = 0, all_on = 0;
  for (uint32_t i = j0; i < j1; i += 32) {
    step(i, y, w, &on);
    all_on += on;
    m += total_of(w);
  }
  m = warp_sum64(m);
  all_on = __reduce_add_sync(0xffffffffu, all_on);
  if (lane == 0) {
    s.warp_mass[warp] = m;
    s.warp_ties[warp] = all_on;
  }
  __syncthreads();
  at = s.run.at + warp_sum64(lane < warp ? s.warp_mass[lane] : 0);
  ties_before = s.run.ties + __reduce_add_sync(0xffffffffu, lane < warp ? s.warp_ties[lane] : 0u);
  // (`at` counts what lies above the threshold; ties are added as they come)
  at += tie * (min(ties, ties_before) - min(ties, s.run.ties));
  if (goal < at || goal >= at + m + tie * (min(ties, ties_before + all_on) - min(ties, ties_before))) return WAY_DONE;
  for (uint32_t i = j0; i < j1; i += 32) {
    step(i, y, w, &on);
    const uint32_t on_inc = warp_incl_scan(on);
    uint64_t rank_on = ties_before + on_inc - on;
    const uint64_t sum = total_of(w) + tie * (min(ties, rank_on + on) - min(ties, rank_on));
    const uint64_t inc = warp_incl_scan(sum), all = __shfl_sync(0xffffffffu, inc, 31);
    if (goal < at + all) {
      Sum upto = at + (inc - sum);
      bool done = !(goal >= upto && goal < upto + sum);
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        uint64_t wk = whole(w[k], WEIGHT_BITS);
        if (i + lane < j1 && y[k] == limit) {
          if (rank_on < ties) wk = tie;
          ++rank_on;
        }
        upto += wk;
        if (!done && goal < upto) {
          done = true;
          with_log((b0 + i + lane) * E + k - off, y[k],
                   (double)(uint32_t)(total >> 64) * 0x1p64 + (double)(uint64_t)total, (uint32_t)(t.count + ties));
        }
      }
      break;
    }
    at += all;
    ties_before += __shfl_sync(0xffffffffu, on_inc, 31);
  }
  return WAY_DONE;
}
}

// A row a cluster (or a CTA), whatever its settings.
template <typename T>
__global__ void __launch_bounds__(SM_THREADS) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ SampleShared s;
  wait_predecessor();
  sample_row<T, true>(a, s, (uint4*)smem_raw, blockIdx.x / a.cluster, false);
  if (a.cluster > 1) cluster_sync();   // no CTA leaves while another reads its shared memory
}
// The same for those of many rows that few candidates decide; the others are queued.
template <typename T>
__global__ void __launch_bounds__(SM_THREADS, 2) sample_many_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ SampleShared s;
  wait_predecessor();
  const uint32_t row = blockIdx.x / a.cluster;
  const uint32_t way = sample_row<T, false>(a, s, (uint4*)smem_raw, row, false);
  if (way != WAY_DONE && threadIdx.x == 0 && blockIdx.x % a.cluster == 0)
    a.queue[atomicAdd(a.counter, 1u)] = row | (way == WAY_WIDE ? QUEUE_WIDE : 0u);
  if (a.cluster > 1) cluster_sync();
}
// The queued rows: a cluster takes one, then whichever is next.  (A CTA an SM:
// the exact sums spill at 64 registers, 109 against 100 us for 256 rows of which
// 17 are queued; where all are, two a SM would be the faster.)
template <typename T>
__global__ void __launch_bounds__(SM_THREADS) sample_queue_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ SampleShared s;
  wait_predecessor();
  const uint32_t nc = a.cluster, rows = *(volatile uint32_t*)a.counter, tid = threadIdx.x;
  if (rows == 0u) return;
  for (uint32_t i = blockIdx.x / nc; i < rows; i = s.row) {
    uint32_t next = 0;
    if (blockIdx.x % nc == 0 && tid < 32) {   // (asked for early: the answer takes a while)
      if (tid == 0) next = gridDim.x / nc + atomicAdd(a.counter + 2, 1u);
    }
    const uint32_t row = a.queue[i];
    sample_row<T, true>(a, s, (uint4*)smem_raw, row & ~QUEUE_WIDE, (row & QUEUE_WIDE) != 0u);
    if (blockIdx.x % nc == 0 && tid < 32) {
      next = __shfl_sync(0xffffffffu, next, 0);
      if (nc == 1 && tid == 0) s.row = next;
      if (nc > 1 && tid < nc) cluster_write(&s.row, tid, next);
    }
    if (nc > 1)
      cluster_sync();
    else
      __syncthreads();
  }
  // the last CTA to leave sets the count back for the next call
  __syncthreads();
  if (tid == 0 && ticket(a.counter + 1) == gridDim.x - 1) {
    a.counter[0] = 0u;
    a.counter[1] = 0u;
    a.counter[2] = 0u;
  }
}

template <typename T>
static uint32_t sample_blocks(uint32_t vocab) { return vocab / Logits<T>::E + 2; }

// CTAs of a row: as many as `places` leave room for, of at least two blocks a thread.
static uint32_t row_ctas(uint32_t blocks, uint64_t rows, uint64_t places) {
  uint32_t nc = 1;
  while (nc < SM_MAX_CLUSTER && rows * nc * 2 <= places && blocks / (nc * 2) >= 2 * SM_THREADS) nc *= 2;
  return nc;
}
static uint32_t blocks_of(uint32_t vocab, int dtype) {
  return dtype == RO_F32 ? sample_blocks<float>(vocab) : sample_blocks<__half>(vocab);
}
bool sample_queues(uint32_t vocab, int dtype, uint64_t rows, int sms) {
  // Few rows: each a cluster, which does whatever the row's settings ask for, a
  // CTA an SM.  More: candidates by as many CTAs as fit twice an SM, and the
  // wide rows after them by clusters as large as for a single row.
  const uint32_t blocks = blocks_of(vocab, dtype);
  return row_ctas(blocks, rows, sms) * 2 < row_ctas(blocks, 1, sms);
}
template <typename T>
static void launch(const LaunchCfg& L, SampleArgs a, int dtype, int sms) {
  const uint32_t blocks = blocks_of(a.vocab, dtype);
  auto go = [&](void (*kernel)(SampleArgs), uint32_t nc, uint32_t clusters) {
    a.cluster = nc;
    a.blocks = (uint32_t)ceil_div(blocks, nc);
    a.staged = (uint64_t)a.blocks * 16 <= SM_SLICE;
    launch_k(L, K_SAMPLE, kernel, clusters * nc, SM_THREADS, a.staged ? (size_t)a.blocks * 16 : 0, a, dim3(nc));
  };
  if (!a.queue) {
    go(sample_kernel<T>, row_ctas(blocks, a.rows, sms), a.rows);
    return;
  }
  const uint32_t wide = row_ctas(blocks, 1, sms);
  go(sample_many_kernel<T>, row_ctas(blocks, a.rows, 2ull * sms), a.rows);
  go(sample_queue_kernel<T>, wide, std::min<uint32_t>(a.rows, (uint32_t)sms / wide));
}
void launch_sample(const LaunchCfg& L, const SampleArgs& a, int dtype, int sms) {
  dtype == RO_F32   ? launch<float>(L, a, dtype, sms)
  : dtype == RO_F16 ? launch<__half>(L, a, dtype, sms)
                    : launch<__nv_bfloat16>(L, a, dtype, sms);
}

template <typename T>
static cudaError_t allow() {
  for (auto kernel : {sample_kernel<T>, sample_many_kernel<T>, sample_queue_kernel<T>})
    if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SM_SLICE); e != cudaSuccess)
      return e;
  return cudaSuccess;
}
cudaError_t prepare_sample_kernels() {
  for (cudaError_t e : {allow<float>(), allow<__half>(), allow<__nv_bfloat16>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
