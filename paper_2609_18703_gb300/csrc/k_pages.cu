// k_pages.cu — pages of a cache: forked, released, moved together, copied
// (ro_cache_fork, ro_cache_compact, ro_cache_copy).
//
// The plan of a fork: entry e of the new lists, page i of continuation c of
// sequence p, is the parent's page i if that is full of tokens, or if c is p's
// first continuation and the page its own; else the k-th free page, k the number
// of such entries before e.  The plan of a compaction: with U pages in use, the
// k-th used page at or above U goes to the k-th free page below U.  Both are
// ranks among flags, taken over the whole list and the whole pool:
//   *_count   every warp counts its run of the lists and of the pool's counts,
//             whose flags it keeps as bits;
//   *_list    the ranks of pages: every warp adds up what is counted before it;
//   *_assign  entries, counts and copies.
// Bound by latency: each phase is a chain of dependent look-ups.  A plan of at
// most 32,768 entries and pages is one launch of a cluster, whose CTAs meet
// between the phases; a larger one is three launches of up to a CTA an SM.
// Measured: 128 sequences into their branches, 5,000 pages: a pass with the copies
// of two layers 20.4 us, in three launches 26.8; one prompt of 6,251 pages into 64
// samples, 400,000 entries, in three launches: 22 us.
// page_copy moves the copied pages' slots, 4 KB a warp at a time, bound by
// reading and writing them once (compacting 20,000 pages of 32 KB a side, 4,970 of
// them moved: 111 us in all, 5.9 TB/s).
#include <algorithm>

#include "ro_step.cuh"

namespace ro {

constexpr uint32_t FRESH = 0xFFFFFFFEu;   // an entry that is to get a free page

// [first, last) of n items, this warp's among all warps of the grid
__device__ __forceinline__ void warp_run(uint64_t n, uint64_t* first, uint64_t* last) {
  const uint64_t w = (uint64_t)blockIdx.x * PG_WARPS + (threadIdx.x >> 5), W = (uint64_t)gridDim.x * PG_WARPS;
  *first = n * w / W;
  *last = n * (w + 1) / W;
}
// What is counted before this warp, and in all.
__device__ __forceinline__ PageCounts counted_before(const PagesArgs& a, PageCounts* total) {
  __shared__ PageCounts s_sum[2][PG_WARPS];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, W = gridDim.x * PG_WARPS;
  const uint32_t first = blockIdx.x * PG_WARPS;
  PageCounts b = {}, t = {};
  for (uint32_t i = threadIdx.x; i < W; i += PG_THREADS) {
    const uint4 v = __ldcg((const uint4*)a.counts + i);
    t.fresh += v.x; t.moves += v.y; t.free += v.z;
    if (i < first) b.fresh += v.x, b.moves += v.y, b.free += v.z;
  }
  auto sum = [](PageCounts x) {
    x.fresh = __reduce_add_sync(0xffffffffu, x.fresh);
    x.moves = __reduce_add_sync(0xffffffffu, x.moves);
    x.free = __reduce_add_sync(0xffffffffu, x.free);
    return x;
  };
  b = sum(b);
  t = sum(t);
  if (lane == 0) {
    s_sum[0][warp] = b;
    s_sum[1][warp] = t;
  }
  __syncthreads();
  *total = sum(s_sum[1][lane]);
  PageCounts mine = sum(s_sum[0][lane]);
  __syncthreads();   // read by all before a later phase writes it
  // the CTA's own warps before this one
  const uint4 v = __ldcg((const uint4*)a.counts + first + lane);
  PageCounts own = {};
  if (lane < warp) own.fresh = v.x, own.moves = v.y, own.free = v.z;
  own = sum(own);
  mine.fresh += own.fresh;
  mine.moves += own.moves;
  mine.free += own.free;
  return mine;
}
// The pool's flags: bit set, page free.  Words of 32 pages, behind the list.
__device__ __forceinline__ uint32_t* free_bits(const PagesArgs& a) { return a.list + a.c.n_pages; }
__device__ __forceinline__ uint32_t count_free(const PagesArgs& a) {
  uint64_t w0, w1;
  const uint32_t words = (a.c.n_pages + 31) / 32, lane = threadIdx.x & 31;
  warp_run(words, &w0, &w1);
  uint32_t n = 0;
#pragma unroll 4
  for (uint64_t w = w0; w < w1; ++w) {
    const uint32_t i = (uint32_t)w * 32 + lane;
    const uint32_t r = i < a.c.n_pages ? a.refs[i] : 1u;
    if (a.refs_out != a.refs && i < a.c.n_pages) a.refs_out[i] = r;
    const uint32_t bits = __ballot_sync(0xffffffffu, r == 0u);
    if (lane == 0) free_bits(a)[w] = bits;
    n += __popc(bits);
  }
  return n;
}

// An output that shares memory with the page list, whose length the host does not know.
__device__ __forceinline__ void record_shared(const PagesArgs& a, uint64_t n, const void* p, uint64_t count) {
  const char *list = (const char*)a.c.pages, *out = (const char*)p;
  if (out < list + n * 4 && list < out + count * 4) record(a.err, ERR_INVAL);
}
__device__ __forceinline__ void record_shared_moves(const PagesArgs& a, uint64_t n) {
  record_shared(a, n, a.m.from, a.m.cap);
  record_shared(a, n, a.m.to, a.m.cap);
  record_shared(a, n, a.m.slots, a.m.cap);
  record_shared(a, n, a.m.n, 1);
  record_shared(a, n, a.refs_out, a.c.n_pages);
}

// ---- fork --------------------------------------------------------------------------------
// An entry of the new lists: where it lies in its continuation, what the parent holds.
struct ForkEntry {
  bool ok, oldest;
  uint64_t at, held, list;   // place in the list, pages of the parent, where its list starts
  uint32_t full, rest;       // its full pages, slots of the open one
};
__device__ __forceinline__ ForkEntry fork_entry(const PagesArgs& a, uint64_t e) {
  ForkEntry f = {};
  const uint32_t c = a.dst_seq[e];
  if (c >= a.n_children) return f;
  const uint64_t b0 = a.dst_base[c], b1 = a.dst_base[c + 1];
  const uint32_t p = a.child_parent[c];
  if (e < b0 || e >= b1 || b1 > a.n_dst || p >= a.c.n_seqs) return f;
  const uint64_t p0 = a.c.page_base[p], p1 = a.c.page_base[p + 1], end = a.c.page_base[a.c.n_seqs];
  const uint32_t len = a.len[p];
  if (p0 > p1 || p1 > end || len >= 0x80000000u) return f;
  f.ok = true;
  f.oldest = a.child_base[p] == c;
  f.at = e - b0;
  f.held = p1 - p0;
  f.list = p0;
  const uint32_t n = (uint32_t)min((uint64_t)len, f.held * a.c.page_size);
  f.full = page_index(a.c, n);
  f.rest = n - f.full * a.c.page_size;
  return f;
}
__device__ __forceinline__ bool fork_copies(const ForkEntry& f) { return f.ok && f.at == f.full && f.rest > 0u && f.at < f.held; }

__device__ __forceinline__ void fork_count(const PagesArgs& a) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  PageCounts n = {};
  uint64_t e0, e1;
  warp_run(a.n_dst, &e0, &e1);
#pragma unroll 4
  for (uint64_t x = e0; x < e1; x += 32) {
    const uint64_t e = x + lane;
    bool fresh = false, copies = false;
    if (e < e1) {
      const ForkEntry f = fork_entry(a, e);
      uint32_t page = RO_NO_PAGE;
      if (!f.ok) {
        record(a.err, ERR_INVAL);
      } else {
        fresh = true;
        if (f.at < f.held && (f.at < f.full || f.oldest)) {
          const uint32_t old = a.c.pages[f.list + f.at];
          if (old >= a.c.n_pages) {
            record(a.err, ERR_INVAL);
            fresh = false;
          } else if (f.at < f.full || a.refs[old] == 1u) {
            page = old;
            fresh = false;
          }
        }
        copies = fresh && fork_copies(f);
      }
      a.dst_pages[e] = fresh ? FRESH : page;
    }
    n.fresh += __popc(__ballot_sync(0xffffffffu, fresh));
    n.moves += __popc(__ballot_sync(0xffffffffu, copies));
  }
  n.free = count_free(a);
  if (lane == 0) a.counts[blockIdx.x * PG_WARPS + warp] = n;
  for (uint64_t c = (uint64_t)blockIdx.x * PG_THREADS + threadIdx.x; c < a.n_children;
       c += (uint64_t)gridDim.x * PG_THREADS) {
    const uint32_t p = a.child_parent[c];
    const uint64_t b0 = a.dst_base[c], b1 = a.dst_base[c + 1];
    uint32_t out = 0;
    bool ok = p < a.c.n_seqs && b0 <= b1 && b1 <= a.n_dst;
    if (ok) {
      const uint64_t p0 = a.c.page_base[p], p1 = a.c.page_base[p + 1];
      const uint32_t len = a.len[p];
      ok = p0 <= p1 && p1 <= a.c.page_base[a.c.n_seqs] && len < 0x80000000u;
      if (ok) {
        const uint64_t room = min(b1 - b0, p1 - p0) * a.c.page_size;
        out = (uint32_t)min((uint64_t)len, room);
        if (out < len) record(a.err, ERR_CAPACITY);
      }
    }
    if (!ok) record(a.err, ERR_INVAL);
    a.len_out[c] = out;
  }
}

__device__ __forceinline__ void fork_list(const PagesArgs& a) {
  PageCounts total;
  const PageCounts before = counted_before(a, &total);
  const uint32_t lane = threadIdx.x & 31;
  uint64_t w0, w1;
  warp_run((a.c.n_pages + 31) / 32, &w0, &w1);
  uint32_t rank = before.free;
  for (uint64_t w = w0; w < w1 && rank < total.fresh; ++w) {
    const uint32_t bits = free_bits(a)[w];
    const uint32_t mine = rank + __popc(bits & ((1u << lane) - 1u));
    if ((bits >> lane & 1u) && mine < total.fresh) a.list[mine] = (uint32_t)w * 32 + lane;
    rank += __popc(bits);
  }
  // the old lists' entries off the counts, before any new one is added
  const uint64_t n = a.c.page_base[a.c.n_seqs];
  for (uint64_t e = (uint64_t)blockIdx.x * PG_THREADS + threadIdx.x; e < n; e += (uint64_t)gridDim.x * PG_THREADS) {
    const uint32_t page = a.c.pages[e];
    if (page >= a.c.n_pages) {
      if (page != RO_NO_PAGE) record(a.err, ERR_INVAL);
    } else if (atomicAdd(a.refs_out + page, 0xFFFFFFFFu) == 0u) {
      atomicAdd(a.refs_out + page, 1u);
      record(a.err, ERR_INVAL);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.m.n = 0;
    record_shared_moves(a, n);
    record_shared(a, n, a.dst_pages, a.n_dst);
    record_shared(a, n, a.len_out, a.n_children);
  }
}

__device__ __forceinline__ void fork_assign(const PagesArgs& a) {
  PageCounts total;
  const PageCounts before = counted_before(a, &total);
  const uint32_t lane = threadIdx.x & 31, below = (1u << lane) - 1u;
  uint32_t rank = before.fresh, move = before.moves;
  uint64_t e0, e1;
  warp_run(a.n_dst, &e0, &e1);
#pragma unroll 4
  for (uint64_t x = e0; x < e1; x += 32) {
    const uint64_t e = x + lane;
    uint32_t page = e < e1 ? a.dst_pages[e] : RO_NO_PAGE;
    const bool fresh = page == FRESH;
    const uint32_t all = __ballot_sync(0xffffffffu, fresh);
    ForkEntry f = {};
    if (fresh) f = fork_entry(a, e);
    const bool copies = fresh && fork_copies(f);
    const uint32_t moves = __ballot_sync(0xffffffffu, copies);
    if (fresh) {
      const uint32_t r = rank + __popc(all & below);
      page = r < total.free ? a.list[r] : RO_NO_PAGE;
      if (page == RO_NO_PAGE) record(a.err, ERR_CAPACITY);
      a.dst_pages[e] = page;
      const uint32_t k = move + __popc(moves & below);
      if (copies && page != RO_NO_PAGE && k < a.m.cap) {
        a.m.from[k] = a.c.pages[f.list + f.at];
        a.m.to[k] = page;
        a.m.slots[k] = f.rest;
        atomicMax(a.m.n, k + 1);   // (entries without a page are the last ones)
      }
    }
    if (page < a.c.n_pages) atomicAdd(a.refs_out + page, 1u);
    rank += __popc(all);
    move += __popc(moves);
  }
}

// ---- compact -------------------------------------------------------------------------------
__device__ __forceinline__ void compact_count(const PagesArgs& a) {
  PageCounts n = {};
  n.free = count_free(a);
  if ((threadIdx.x & 31) == 0) a.counts[blockIdx.x * PG_WARPS + (threadIdx.x >> 5)] = n;
}

// The moves, and each moved page's rank.
__device__ __forceinline__ void compact_list(const PagesArgs& a) {
  PageCounts total;
  const PageCounts before = counted_before(a, &total);
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t used = a.c.n_pages - total.free, words = (a.c.n_pages + 31) / 32, W = gridDim.x * PG_WARPS;
  __shared__ uint32_t s_holes;   // free pages below `used`: the moves
  {
    // those counted by the warps whose runs end below, and what the run that holds it has before it
    const uint32_t at = used / 32;
    uint32_t n = 0;
    __shared__ uint32_t s_part[PG_WARPS];
    for (uint32_t i = threadIdx.x; i < W; i += PG_THREADS) {
      const uint64_t w0 = (uint64_t)words * i / W, w1 = (uint64_t)words * (i + 1) / W;
      if (w1 <= at) {
        n += __ldcg(&a.counts[i].free);
      } else if (w0 <= at) {
        for (uint64_t w = w0; w < at; ++w) n += __popc(free_bits(a)[w]);
        if (at < words) n += __popc(free_bits(a)[at] & ((1u << (used % 32)) - 1u));
      }
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) s_part[warp] = n;
    __syncthreads();
    if (warp == 0) {
      n = __reduce_add_sync(0xffffffffu, s_part[lane]);
      if (lane == 0) s_holes = n;
    }
    __syncthreads();
  }
  const uint32_t holes = s_holes;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.n_used = used;
    *a.m.n = holes;
  }
  uint64_t w0, w1;
  warp_run(words, &w0, &w1);
  uint32_t rank = before.free;
  for (uint64_t w = w0; w < w1; ++w) {
    const uint32_t bits = free_bits(a)[w], i = (uint32_t)w * 32 + lane;
    const uint32_t free_before = rank + __popc(bits & ((1u << lane) - 1u));
    const bool free = bits >> lane & 1u;
    if (i < used) {
      if (free && free_before < a.m.cap) a.m.to[free_before] = i;
    } else if (i < a.c.n_pages) {
      const uint32_t k = (i - free_before) - (used - holes);   // used pages before it, less those below `used`
      a.list[i] = free ? RO_NO_PAGE : k;
      if (!free && k < a.m.cap) {
        a.m.from[k] = i;
        a.m.slots[k] = a.c.page_size;
      }
    }
    rank += __popc(bits);
  }
}

__device__ __forceinline__ void compact_assign(const PagesArgs& a) {
  const uint64_t t = (uint64_t)blockIdx.x * PG_THREADS + threadIdx.x, step = (uint64_t)gridDim.x * PG_THREADS;
  const uint32_t used = *a.n_used, holes = *a.m.n;
  for (uint64_t k = t; k < holes && k < a.m.cap; k += step) {
    const uint32_t from = a.m.from[k], to = a.m.to[k];
    const uint32_t r = a.refs_out[from];   // (as counted: the copies of refs are made)
    a.refs_out[to] = r;
    a.refs_out[from] = 0;
  }
  const uint64_t n = a.c.page_base[a.c.n_seqs];
  if (t == 0) {
    if (n > a.n_list) record(a.err, ERR_CAPACITY);
    record_shared_moves(a, n);
    record_shared(a, n, a.n_used, 1);
    if (a.pages_out != a.c.pages) record_shared(a, n, a.pages_out, a.n_list);
  }
  for (uint64_t e = t; e < n && e < a.n_list; e += step) {
    uint32_t page = a.c.pages[e];
    if (page >= a.c.n_pages) {
      if (page != RO_NO_PAGE) record(a.err, ERR_INVAL);
    } else if (page >= used) {
      const uint32_t k = a.list[page];
      if (k < holes && k < a.m.cap)
        page = a.m.to[k];
      else
        record(a.err, ERR_INVAL);
    } else if (free_bits(a)[page / 32] >> (page % 32) & 1u) {
      record(a.err, ERR_INVAL);
    }
    a.pages_out[e] = page;
  }
}

// The three phases: one cluster's, or a launch each.
template <int PHASE>
__global__ void __launch_bounds__(PG_THREADS) fork_kernel(const __grid_constant__ PagesArgs a) {
  wait_predecessor();
  if (PHASE == 0 || PHASE == 1) fork_count(a);
  if (PHASE == 0) cluster_sync();
  if (PHASE == 0 || PHASE == 2) fork_list(a);
  if (PHASE == 0) cluster_sync();
  if (PHASE == 0 || PHASE == 3) fork_assign(a);
}
template <int PHASE>
__global__ void __launch_bounds__(PG_THREADS) compact_kernel(const __grid_constant__ PagesArgs a) {
  wait_predecessor();
  if (PHASE == 0 || PHASE == 1) compact_count(a);
  if (PHASE == 0) cluster_sync();
  if (PHASE == 0 || PHASE == 2) compact_list(a);
  if (PHASE == 0) cluster_sync();
  if (PHASE == 0 || PHASE == 3) compact_assign(a);
}

// ---- copies --------------------------------------------------------------------------------
constexpr int PC_THREADS = 256;
constexpr uint32_t PC_PIECE = 256;   // 16-byte vectors of a piece
__global__ void __launch_bounds__(PC_THREADS) page_copy_kernel(const __grid_constant__ PageCopyArgs a) {
  wait_predecessor();
  const uint32_t lane = threadIdx.x & 31, per = a.c.head_dim / 8;
  const uint64_t warps = (uint64_t)gridDim.x * (PC_THREADS / 32);
  const uint32_t n = *a.m.n;
  if (n > a.m.cap && blockIdx.x == 0 && threadIdx.x == 0) record(a.err, ERR_CAPACITY);
  const uint64_t items = min((uint64_t)n, a.m.cap) * a.c.n_heads * 2 * a.pieces;
  for (uint64_t x = (uint64_t)blockIdx.x * (PC_THREADS / 32) + (threadIdx.x >> 5); x < items; x += warps) {
    const uint64_t u = x / a.pieces;
    const uint32_t piece = (uint32_t)(x - u * a.pieces), kv = (uint32_t)(u & 1);
    const uint64_t mh = u >> 1, m = mh / a.c.n_heads;
    const uint32_t h = (uint32_t)(mh - m * a.c.n_heads);
    const uint32_t from = a.m.from[m], to = a.m.to[m], slots = a.m.slots[m];
    if (from >= a.c.n_pages || to >= a.c.n_pages || slots > a.c.page_size) {
      if (lane == 0) record(a.err, ERR_INVAL);
      continue;
    }
    uint16_t* pool = (uint16_t*)(kv ? a.c.v : a.c.k) + h * a.c.head_stride;
    const uint16_t* src = pool + from * a.c.page_stride;
    uint16_t* dst = pool + to * a.c.page_stride;
    const uint64_t v0 = (uint64_t)piece * PC_PIECE + lane, v1 = min((uint64_t)(piece + 1) * PC_PIECE, (uint64_t)slots * per);
    uint4 v[PC_PIECE / 32];
    uint64_t at[PC_PIECE / 32];
#pragma unroll
    for (uint32_t i = 0; i < PC_PIECE / 32; ++i) {
      const uint64_t y = v0 + i * 32, slot = a.dense ? 0 : y / per;
      at[i] = a.dense ? y * 8 : slot * a.c.slot_stride + (y - slot * per) * 8;
      if (y < v1) v[i] = __ldcs((const uint4*)(src + at[i]));
    }
#pragma unroll
    for (uint32_t i = 0; i < PC_PIECE / 32; ++i)
      if (v0 + i * 32 < v1) __stcs((uint4*)(dst + at[i]), v[i]);
  }
}

// ---- host ------------------------------------------------------------------------------------
// CTAs of a plan: four entries or pages a thread; up to eight are a cluster.
constexpr uint32_t PG_CLUSTER = 8;
uint32_t pages_ctas(uint64_t items, int sms) {
  const uint64_t n = std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(items, 4 * PG_THREADS), (uint64_t)sms));
  uint32_t pow2 = 1;
  while (pow2 < n) pow2 *= 2;
  return n <= PG_CLUSTER ? std::min(PG_CLUSTER, 4 * pow2) : (uint32_t)n;   // (short chains before few CTAs)
}
template <class K>
static void launch_phases(const LaunchCfg& L, const PagesArgs& a, uint32_t ctas, K whole, K count, K list, K assign) {
  if (ctas <= PG_CLUSTER) {
    launch_k(L, K_PAGES, whole, ctas, PG_THREADS, 0, a, dim3(ctas));
    return;
  }
  for (K phase : {count, list, assign}) launch_k(L, K_PAGES, phase, ctas, PG_THREADS, 0, a);
}
void launch_fork(const LaunchCfg& L, const PagesArgs& a, uint32_t ctas) {
  launch_phases(L, a, ctas, fork_kernel<0>, fork_kernel<1>, fork_kernel<2>, fork_kernel<3>);
}
void launch_compact(const LaunchCfg& L, const PagesArgs& a, uint32_t ctas) {
  launch_phases(L, a, ctas, compact_kernel<0>, compact_kernel<1>, compact_kernel<2>, compact_kernel<3>);
}
void launch_page_copy(const LaunchCfg& L, const PagedArgs& c, const MoveArgs& m, uint32_t* err, int sms) {
  PageCopyArgs a;
  a.c = c;
  a.m = m;
  a.err = err;
  a.dense = c.slot_stride == c.head_dim;
  a.pieces = (uint32_t)ceil_div((uint64_t)c.page_size * (c.head_dim / 8), PC_PIECE);
  const uint64_t items = m.cap * c.n_heads * 2 * a.pieces;
  const uint64_t ctas = std::min<uint64_t>(ceil_div(items, PC_THREADS / 32), (uint64_t)sms * 4);
  if (ctas) launch_k(L, K_PAGES, page_copy_kernel, (unsigned)ctas, PC_THREADS, 0, a);
}

}  // namespace ro
