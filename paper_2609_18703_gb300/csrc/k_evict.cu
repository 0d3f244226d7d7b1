// k_evict.cu — cut a cache back to its heaviest tokens (ro_cache_evict).
//
// evict_select  A cluster of 1 to 8 CTAs per sequence and cache head, a run of
//               slots each.  Of the slots between the sinks and the recent ones
//               the k largest scores stay: scores map to 32-bit keys that order
//               alike (NaN lowest, -0 as 0), read once into shared memory where
//               they fit; three passes of 11, 11 and 10 bits find the k-th
//               largest key T (histograms summed over the cluster), and a last
//               pass in slot order writes the slots with a key above T and the
//               first ones equal to it.  Bound by the latency of its steps.
//               One sequence of 100,000 slots, 4 heads: 12 us with 8 CTAs a head
//               (one CTA, from L2: 181 us).
// evict_move    Kept rows of K and V to the new pages: bound by reading and
//               writing them once; 16 bytes a thread.  64 sequences of up to
//               8,192 slots, 8 heads of 128, to 2,048: 120 us, 6.1 TB/s (two or
//               four rows a thread in flight: 128 and 135 us; moved by the
//               selecting CTAs themselves: no faster in all).
#include <algorithm>

#include "ro_step.cuh"

namespace ro {

// larger score, larger key; NaN lowest
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t cached(const EvictArgs& a, uint32_t s, bool first) {
  const uint64_t p0 = a.c.page_base[s], p1 = a.c.page_base[s + 1], end = a.c.page_base[a.c.n_seqs];
  uint32_t len = a.len[s];
  if (p1 < p0 || p1 > end || len >= 0x80000000u) {
    if (first) record(a.err, ERR_INVAL);
    return 0;
  }
  uint64_t cap = (p1 - p0) * a.c.page_size;
  if (cap > a.score_cap) cap = a.score_cap;
  if (len > cap) {
    if (first) record(a.err, ERR_CAPACITY);
    len = (uint32_t)cap;
  }
  return len;
}

// ---- clusters ------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_load(const uint32_t* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_at(step_smem(p), rank)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_add(const uint32_t* p, uint32_t rank, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(cluster_at(step_smem(p), rank)), "r"(v) : "memory");
}
// Exclusive prefix of one value per thread over 1,024 threads, and the total;
// one barrier (every warp scans the warps' totals for itself).  smem: 32 words
// that no earlier call of this kernel used.
template <class T>
__device__ __forceinline__ T select_scan(T v, T* smem, T* total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const T inc = warp_incl_scan(v);
  if (lane == 31) smem[wid] = inc;
  __syncthreads();
  const T all = warp_incl_scan(smem[lane]);
  const T before = __shfl_sync(0xffffffffu, all, wid > 0 ? wid - 1 : 0);
  *total = __shfl_sync(0xffffffffu, all, 31);
  return (wid > 0 ? before : T(0)) + inc - v;
}

constexpr uint32_t ES_BINS = 2048;

__global__ void __launch_bounds__(ES_THREADS) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ uint32_t s_keys[];          // [cached]
  __shared__ uint32_t s_hist[ES_BINS];          // this CTA's counts of a pass
  __shared__ uint32_t s_sum[3][ES_BINS];        // the cluster's, a pass each
  __shared__ uint32_t s_scan[3][32];
  __shared__ unsigned long long s_scan2[32];
  __shared__ uint32_t s_digit[3], s_left[3], s_total[2];
  wait_predecessor();
  const uint32_t tid = threadIdx.x, nc = a.cluster, rank = nc > 1 ? cluster_rank() : 0;
  const uint32_t unit = blockIdx.x / nc;
  const uint32_t s = unit / a.c.n_heads, h = unit - s * a.c.n_heads;
  const uint32_t len = cached(a, s, tid == 0 && h == 0 && rank == 0);
  const uint64_t row = (uint64_t)unit * a.score_cap;
  const float* score = a.score + row;
  uint32_t* keep = a.keep + (uint64_t)unit * a.budget;
  float* out = a.score_out ? a.score_out + row : nullptr;
  const uint32_t t0 = rank * ES_THREADS + tid, step = nc * ES_THREADS;   // this thread among the cluster's
  if (len <= a.budget) {                        // (the whole cluster)
    for (uint32_t j = t0; j < len; j += step) {
      keep[j] = j;
      if (out) out[j] = score[j];
    }
    return;
  }
  const uint32_t lo = a.sinks, hi = len - a.recent;
  for (uint32_t j = t0; j < a.sinks; j += step) {
    keep[j] = j;
    if (out) out[j] = score[j];
  }
  for (uint32_t j = t0; j < a.recent; j += step) {
    const uint32_t at = a.budget - a.recent + j;
    keep[at] = hi + j;
    if (out) out[at] = score[hi + j];
  }
  // this CTA's run of the slots between, [j0, j0 + n)
  const uint32_t each = (hi - lo + nc - 1) / nc, j0 = min(hi, lo + rank * each), n = min(each, hi - j0);
  const uint32_t held = min(n, a.cached);       // of them in shared memory, the rest read again
#pragma unroll 4
  for (uint32_t i = tid; i < held; i += ES_THREADS) s_keys[i] = score_key(score[j0 + i]);
  for (uint32_t i = tid; i < ES_BINS; i += ES_THREADS) s_hist[i] = s_sum[0][i] = s_sum[1][i] = s_sum[2][i] = 0;
  if (tid < 3) {                                // nothing to choose: a threshold above every key
    s_digit[tid] = tid == 2 ? 1023u : ES_BINS - 1;
    s_left[tid] = 0;
  }
  if (nc > 1)
    cluster_sync();                             // every CTA's sums are zero
  else
    __syncthreads();
  auto key = [&](uint32_t i) { return i < held ? s_keys[i] : score_key(score[j0 + i]); };
  uint32_t left = a.budget - a.sinks - a.recent;   // still to choose among equal prefixes
  uint32_t prefix = 0, mask = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass == 2 ? 10 : 11, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t bins = 1u << bits;
    uint32_t* hist = nc > 1 ? s_hist : s_sum[pass];
    for (uint32_t i = tid; i < n; i += ES_THREADS) {
      const uint32_t k = key(i);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
    }
    if (nc > 1) {                               // bins that hold something go to every CTA's sums
      __syncthreads();
      for (uint32_t i = tid; i < bins; i += ES_THREADS) {
        const uint32_t c = s_hist[i];
        if (c == 0) continue;
        for (uint32_t r = 0; r < nc; ++r) cluster_add(&s_sum[pass][i], r, c);
        s_hist[i] = 0;
      }
      cluster_sync();
    } else {
      __syncthreads();
    }
    // the digit whose keys, counted from the largest, reach `left`: two bins a thread, largest first
    const uint32_t b1 = bins - 1 - 2 * tid, b0 = b1 - 1;
    uint32_t c1 = 0, c0 = 0, total;
    if (2 * tid < bins) {
      c1 = s_sum[pass][b1];
      c0 = s_sum[pass][b0];
    }
    const uint32_t above = select_scan(c1 + c0, s_scan[pass], &total);
    if (left > 0 && above < left && above + c1 + c0 >= left) {
      const bool first = above + c1 >= left;
      s_digit[pass] = first ? b1 : b0;
      s_left[pass] = left - above - (first ? 0 : c1);
    }
    __syncthreads();
    prefix |= s_digit[pass] << shift;
    mask |= (bins - 1) << shift;
    left = s_left[pass];
  }
  // Keys above prefix, and the first `left` equal to it, in slot order: a
  // thread takes neighbouring slots, an odd number of them (the banks of
  // shared memory), and counts before it writes.
  const uint32_t own = ((n + ES_THREADS - 1) / ES_THREADS) | 1u, f0 = min(n, tid * own), f1 = min(n, f0 + own);
  uint32_t gt = 0, eq = 0;
  for (uint32_t i = f0; i < f1; ++i) {
    const uint32_t k = key(i);
    gt += k > prefix;
    eq += k == prefix;
  }
  unsigned long long all;                       // counts of both kinds in one scan
  const unsigned long long before = select_scan(((unsigned long long)eq << 32) | gt, s_scan2, &all);
  uint32_t gt_before = (uint32_t)before, eq_before = (uint32_t)(before >> 32);
  if (nc > 1) {
    if (tid == 0) {
      s_total[0] = (uint32_t)all;
      s_total[1] = (uint32_t)(all >> 32);
    }
    cluster_sync();
    for (uint32_t r = 0; r < rank; ++r) {
      gt_before += cluster_load(s_total, r);
      eq_before += cluster_load(s_total + 1, r);
    }
  }
  for (uint32_t i = f0; i < f1; ++i) {
    const uint32_t k = key(i);
    const bool tie = k == prefix;
    if (k > prefix || (tie && eq_before < left)) {
      const uint32_t at = a.sinks + gt_before + min(eq_before, left);
      keep[at] = j0 + i;
      // a key gives its score back, but for NaN and the sign of 0
      if (out)
        out[at] = k == 0u || k == 0x80000000u ? score[j0 + i]
                                              : __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
    }
    gt_before += k > prefix;
    eq_before += tie;
  }
  if (nc > 1) cluster_sync();   // no CTA leaves while another reads its shared memory
}

constexpr int EM_THREADS = 256;
// `parts` CTAs for each (sequence, head)
__global__ void __launch_bounds__(EM_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs a) {
  wait_predecessor();
  const uint32_t unit = blockIdx.x / a.parts, part = blockIdx.x - unit * a.parts;
  const uint32_t s = unit / a.c.n_heads, h = unit - s * a.c.n_heads;
  const uint32_t len = cached(a, s, false);
  const uint32_t kept = min(len, a.budget);
  // Written here and not by the CTAs that select: len_out may be len, and those
  // have to read what the sequence held.  Whoever reads a length here after it is
  // cut keeps as much: a cut of a cut length changes nothing.
  if (h == 0 && part == 0 && threadIdx.x == 0) a.len_out[s] = kept;
  const uint64_t b0 = a.dst_base[s], b1 = a.dst_base[s + 1], end = a.dst_base[a.c.n_seqs], p0 = a.c.page_base[s];
  const bool in_list = b0 <= b1 && b1 <= end;
  const uint64_t room = in_list ? (b1 - b0) * a.c.page_size : 0;
  const uint32_t n = (uint32_t)min((uint64_t)kept, room);
  if (n < kept && part == 0 && threadIdx.x == 0) record(a.err, in_list ? ERR_CAPACITY : ERR_INVAL);
  const uint32_t per = a.c.head_dim / 8;                 // 16-byte pieces of a row
  const uint32_t* keep = a.keep + (uint64_t)unit * a.budget;
  const uint64_t items = (uint64_t)n * per, stride = (uint64_t)a.parts * EM_THREADS;
  for (uint64_t i = (uint64_t)part * EM_THREADS + threadIdx.x; i < items; i += stride) {
    const uint32_t d = (uint32_t)(i / per), p = (uint32_t)(i - (uint64_t)d * per);
    uint32_t pi, slot;
    split_slot(a.c, keep[d], &pi, &slot);
    const uint32_t src = a.c.pages[p0 + pi];
    const uint64_t from = src * a.c.page_stride + h * a.c.head_stride + slot * a.c.slot_stride + p * 8;
    split_slot(a.c, d, &pi, &slot);
    const uint32_t dst = a.dst_pages[b0 + pi];
    const uint64_t to = dst * a.c.page_stride + h * a.c.head_stride + slot * a.c.slot_stride + p * 8;
    if (src >= a.c.n_pages || dst >= a.c.n_pages) {
      record(a.err, ERR_INVAL);
      continue;
    }
    const uint4 k = *(const uint4*)((const uint16_t*)a.c.k + from), v = *(const uint4*)((const uint16_t*)a.c.v + from);
    *(uint4*)((uint16_t*)a.c.k + to) = k;
    *(uint4*)((uint16_t*)a.c.v + to) = v;
  }
}

void launch_evict(const LaunchCfg& L, const EvictArgs& in, int sms) {
  EvictArgs a = in;
  const unsigned units = a.c.n_seqs * a.c.n_heads;
  // CTAs of a unit: up to 8 while that gives each at least 1,024 slots and the
  // GPU has places (4 units of 16,000 slots, moved too: 16 us with 8 CTAs, 18 with
  // 2, 21 with 1; of 100,000: 42 and 315 us with 8 and 1)
  a.cluster = 1;
  while (a.cluster < 8 && (uint64_t)units * a.cluster * 2 <= (uint64_t)sms * 2 && a.score_cap / (a.cluster * 2) >= 1024)
    a.cluster *= 2;
  // keys in shared memory: a run's, as far as two CTAs an SM have room for them
  a.cached = (uint32_t)std::min<uint64_t>(ceil_div(a.score_cap, a.cluster), ES_CACHED);
  launch_k(L, K_EVICT_SELECT, evict_select_kernel, units * a.cluster, ES_THREADS, a.cached * sizeof(uint32_t), a,
           dim3(a.cluster));
  // eight CTAs an SM over all units, at most one per 4 items of a thread
  const uint64_t most = ceil_div((uint64_t)a.budget * (a.c.head_dim / 8), EM_THREADS * 4);
  a.parts = (uint32_t)std::max<uint64_t>(1, std::min(most, ceil_div((uint64_t)sms * 8, units)));
  launch_k(L, K_EVICT_MOVE, evict_move_kernel, a.parts * units, EM_THREADS, 0, a);
}

cudaError_t prepare_evict_kernels() {
  return cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)(ES_CACHED * sizeof(uint32_t)));
}

}  // namespace ro
