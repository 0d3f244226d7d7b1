// k_evict.cu — cut a cache back to its heaviest tokens (ro_cache_evict).
//
// evict_select  One CTA per sequence and cache head.  Of the slots between the
//               sinks and the recent ones the k largest scores stay: scores map
//               to 32-bit keys that order alike (NaN lowest, -0 as 0), four
//               passes of 8 bits find the k-th largest key T, and a last pass
//               in slot order writes the slots with a key above T and the first
//               ones equal to it.  Reads each score five times, from L2.
// evict_move    Kept rows of K and V to the new pages: bound by reading and
//               writing them once; 16 bytes a thread.
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
  const uint64_t p0 = a.c.page_base[s], p1 = a.c.page_base[s + 1];
  uint32_t len = a.len[s];
  if (p1 < p0 || len >= 0x80000000u) {
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

__global__ void __launch_bounds__(ES_THREADS) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ uint32_t s_hist[256];
  __shared__ uint32_t s_scan[33];
  __shared__ uint32_t s_digit, s_left;
  wait_predecessor();
  const uint32_t tid = threadIdx.x;
  const uint32_t s = blockIdx.x / a.c.n_heads, h = blockIdx.x - s * a.c.n_heads;
  const uint32_t len = cached(a, s, tid == 0 && h == 0);
  const uint64_t row = (uint64_t)blockIdx.x * a.score_cap;
  const float* score = a.score + row;
  uint32_t* keep = a.keep + (uint64_t)blockIdx.x * a.budget;
  float* out = a.score_out ? a.score_out + row : nullptr;
  const uint32_t kept = min(len, a.budget);
  if (h == 0 && tid == 0) a.len_out[s] = kept;
  if (len <= a.budget) {
    for (uint32_t j = tid; j < len; j += ES_THREADS) {
      keep[j] = j;
      if (out) out[j] = score[j];
    }
    return;
  }
  const uint32_t lo = a.sinks, hi = len - a.recent;
  uint32_t left = a.budget - a.sinks - a.recent;   // still to choose among equal prefixes
  uint32_t prefix = 0, mask = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (uint32_t j = lo + tid; j < hi; j += ES_THREADS) {
      const uint32_t k = score_key(score[j]);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    // the digit whose keys, counted from the largest, reach `left`
    uint32_t c = 0, total;
    if (tid < 256) c = s_hist[255 - tid];
    const uint32_t above = block_excl_scan(c, s_scan, &total);
    if (left > 0 && tid < 256 && above < left && above + c >= left) {
      s_digit = 255 - tid;
      s_left = left - above;
    }
    if (left == 0 && tid == 0) {   // nothing to choose: a threshold above every key
      s_digit = 255;
      s_left = 0;
    }
    __syncthreads();
    prefix |= s_digit << shift;
    mask |= 255u << shift;
    left = s_left;
    __syncthreads();
  }
  // keys above prefix, and the first `left` equal to it, in slot order
  for (uint32_t j = tid; j < a.sinks; j += ES_THREADS) {
    keep[j] = j;
    if (out) out[j] = score[j];
  }
  uint32_t done = 0, ties = 0;
  for (uint32_t j0 = lo; j0 < hi; j0 += ES_THREADS) {
    const uint32_t j = j0 + tid;
    uint32_t gt = 0, eq = 0;
    float x = 0.f;
    if (j < hi) {
      x = score[j];
      const uint32_t k = score_key(x);
      gt = k > prefix;
      eq = k == prefix;
    }
    uint32_t total;
    // both counts in one scan: at most 1,024 each
    const uint32_t e = block_excl_scan(gt | (eq << 16), s_scan, &total);
    const uint32_t eq_before = ties + (e >> 16), gt_before = done + (e & 0xFFFFu);
    const uint32_t eq_taken = min(eq_before, left);
    if (gt || (eq && eq_before < left)) {
      const uint32_t at = a.sinks + gt_before + eq_taken;
      keep[at] = j;
      if (out) out[at] = x;
    }
    done += total & 0xFFFFu;
    ties += total >> 16;
  }
  for (uint32_t j = tid; j < a.recent; j += ES_THREADS) {
    const uint32_t at = a.budget - a.recent + j;
    keep[at] = hi + j;
    if (out) out[at] = score[hi + j];
  }
}

constexpr int EM_THREADS = 256;
// `parts` CTAs for each (sequence, head)
__global__ void __launch_bounds__(EM_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs a) {
  wait_predecessor();
  const uint32_t unit = blockIdx.x / a.parts, part = blockIdx.x - unit * a.parts;
  const uint32_t s = unit / a.c.n_heads, h = unit - s * a.c.n_heads;
  const uint32_t len = cached(a, s, false);
  const uint32_t kept = min(len, a.budget);
  const uint64_t b0 = a.dst_base[s], b1 = a.dst_base[s + 1], p0 = a.c.page_base[s];
  const uint64_t room = b1 > b0 ? (b1 - b0) * a.c.page_size : 0;
  const uint32_t n = (uint32_t)min((uint64_t)kept, room);
  if (n < kept && part == 0 && threadIdx.x == 0) record(a.err, b1 < b0 ? ERR_INVAL : ERR_CAPACITY);
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
  launch_k(L, K_EVICT_SELECT, evict_select_kernel, units, ES_THREADS, 0, a);
  // eight CTAs an SM over all units, at most one per 4 items of a thread
  const uint64_t most = ceil_div((uint64_t)a.budget * (a.c.head_dim / 8), EM_THREADS * 4);
  a.parts = (uint32_t)std::max<uint64_t>(1, std::min(most, ceil_div((uint64_t)sms * 8, units)));
  launch_k(L, K_EVICT_MOVE, evict_move_kernel, a.parts * units, EM_THREADS, 0, a);
}

}  // namespace ro
