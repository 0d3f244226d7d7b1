// k_attend_tiles.cu — attention of chunks over a paged cache (ro_cache_attend)
// on the fifth-generation tensor cores.
//
//   S = Q K^T, P = exp2(scale log2(e) S - m), O = P V, l = row sums of P,
// per 128-row tile of (token, head of the group) and 128 slots at a time, with
// a running m.  Bound by the tensor cores: 4 D operations for each pair of a
// row and a slot it sees.
//
// A CTA holds two row tiles, so that one tile's exponentials run while the
// tensor cores work for the other: a warp of TMA loads (page by page, swizzled)
// into a ring of key and value tiles, a warp that issues the products, and for
// each row tile four warps of softmax, a thread a row.  S and O live in TMEM;
// P replaces S there and is the left operand of the second product.  m only
// moves when a row's maximum grew by more than 2^8 (f16: 2^4), so O is seldom
// rescaled.
// Slots that no row of the CTA sees are never loaded or are zeroed in shared
// memory first (a weight of 0 does not silence a NaN in a matrix product).
// A CTA stays on its SM and takes pairs of row tiles as it gets free, heavy ones
// first: the next pair's queries, keys and first products are under way while
// the last one's output is written.  When there are fewer pairs than places,
// the slots are split into runs, whose (m, l, O) a second kernel joins in order.
//
// Measured: 8 ragged chunks of up to 2,048 tokens over up to 16,384 slots, 32
// heads on 8 of 128: 420 us, 1.54 PFLOP/s (cuBLAS's burst: 1.95); 512 tokens over
// 64,000 slots 307 us, 1.74 PFLOP/s.  A pair of products takes 2,050 cycles at the
// tensor cores' rate; a pair's cycle takes about 2,800, of which its softmax
// is 1,400 (the maxima 500, the exponentials 900, 512 of them the XU's).
#include <algorithm>

#include "ro_tcgen05.cuh"

namespace ro {

constexpr int AT_THREADS = 384, AT_ROWS = 128, AT_KEYS = 128;
constexpr int AT_SOFTMAX = 256;     // threads 0 .. 255: softmax; then a warp each of products, loads, work
// Registers: 168 a thread at launch (3 warps in each quarter of the SM); the
// last warpgroup gives up what the softmax threads need, 2 x 216 + 72 = 3 x 168.
#define AT_REGS_SOFTMAX 216
#define AT_REGS_OTHERS 72
constexpr uint32_t AT_TMEM_COLS = 512;
// log2 of what a row's maximum may grow before O is rescaled; f16 weights, at
// most 2^15, have to hold it beside the bits they are held higher by
template <typename T>
constexpr int AT_SLACK = 8;
template <>
constexpr int AT_SLACK<__half> = 4;

template <int DP>
struct TileShape {
  static constexpr uint32_t BLOCKS = DP / 64;                    // 64-column blocks of a row
  static constexpr uint32_t BLOCK_BYTES = 128 * 128;             // 128 rows of 128 bytes
  static constexpr uint32_t TILE_BYTES = BLOCKS * BLOCK_BYTES;
  static constexpr uint32_t SLOTS = DP == 128 ? 5 : 8;           // key / value tiles in the ring
  static constexpr uint32_t SMEM = 1024 + (2 + SLOTS) * TILE_BYTES;
};

// A piece of work: a pair of row tiles of one sequence and head, and a run of
// the slots they see.
struct TileItem {
  uint64_t tok0, page0;
  int64_t first;             // slot of the chunk's first token
  KeySpan span;
  uint32_t i0, i1;           // the chunk's tokens in the row tiles
  uint32_t kh, unit;         // head; (tile, head)
  uint32_t c0, n;            // the run's slot tiles
  uint32_t run, n_runs;
  uint32_t last;             // no work: the end
};
// A pair of row tiles for the join: its first token, its tokens, its runs.
struct JoinItem {
  uint64_t tok;
  uint32_t n, runs;
};
constexpr uint32_t AT_ITEMS = 2;
// The next item is taken this many slot tiles before the loads of the present
// one end: early enough to decode it, late enough not to hold work that a CTA
// which runs dry could do.
constexpr uint32_t AT_AHEAD = 8;

template <typename T, int DP>
__global__ void __launch_bounds__(AT_THREADS, 1) attend_tiles_kernel(const __grid_constant__ AttendTileArgs g) {
  using S = TileShape<DP>;
  const AttendArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[2 + 2 * S::SLOTS + 10 + 2 * AT_ITEMS + 1];
  __shared__ TileItem s_item[AT_ITEMS];
  __shared__ uint32_t s_tmem, s_gave_up;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t G = a.r.group;
  const uint32_t sm = (step_smem(smem_raw) + 1023u) & ~1023u;
  const uint32_t sm_ring = sm + 2 * S::TILE_BYTES;
  // full / empty: queries, the ring, S, P, O, items
  const uint32_t b_q = step_smem(s_bar), b_qe = b_q + 8, b_full = b_qe + 8, b_empty = b_full + 8 * S::SLOTS,
                 b_s = b_empty + 8 * S::SLOTS, b_p = b_s + 16, b_o = b_p + 32, b_oe = b_o + 16, b_item = b_oe + 16,
                 b_item_free = b_item + 8 * AT_ITEMS, b_want = b_item_free + 8 * AT_ITEMS;
  if (tid == 0) {
    s_gave_up = 0;
    bar_init(b_q, 1);
    bar_init(b_qe, 1);
    bar_init(b_want, 1);
    for (uint32_t i = 0; i < S::SLOTS; ++i) {
      bar_init(b_full + 8 * i, 1);
      bar_init(b_empty + 8 * i, 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      bar_init(b_s + 8 * i, 1);
      bar_init(b_p + 16 * i, 4);       // P in two halves of 64 slots
      bar_init(b_p + 16 * i + 8, 4);
      bar_init(b_o + 8 * i, 1);
      bar_init(b_oe + 8 * i, 4);
    }
    for (uint32_t i = 0; i < AT_ITEMS; ++i) {
      bar_init(b_item + 8 * i, 1);
      bar_init(b_item_free + 8 * i, 10);   // 8 warps of softmax, loads, products
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 8) tmem_alloc(step_smem(&s_tmem), AT_TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = __shfl_sync(0xffffffffu, s_tmem, 0);
  const uint32_t tm_s = tm, tm_o = tm + 256;   // 128 columns for each row tile

  if (warp >= AT_SOFTMAX / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(AT_REGS_OTHERS));
    // the k-th item, to a whole warp; released once its reader is done with it
    auto item = [&](uint32_t k) -> const TileItem& {
      bar_wait(b_item + 8 * (k % AT_ITEMS), (k / AT_ITEMS) & 1, &s_gave_up, a.err);
      return s_item[k % AT_ITEMS];
    };
    auto release = [&](uint32_t k) {
      __syncwarp();
      if (lane == 0) bar_arrive(b_item_free + 8 * (k % AT_ITEMS));
    };
    if (warp == 10) {
      // ---- work ----
      // The first item by the CTA's number, the others as they are asked for;
      // items are in falling order of work where that is known.
      const uint32_t items = a.tiles * a.c.n_heads * a.max_chunks;
      uint32_t k = 0;
      for (uint32_t id = blockIdx.x;;) {
        TileItem it = {};
        it.last = id >= items;
        bool some = true;
        if (!it.last) {
          // Unsplit: the heads of a pair of row tiles together, heavy pairs
          // first.  Split: the pairs that read the same slots together, so
          // that those come from L2 (one sequence of 64,000 slots, 512 new
          // tokens: its cache is twice L2).
          uint32_t tile;
          if (a.max_chunks == 1) {
            tile = id / a.c.n_heads;
            it.kh = id - tile * a.c.n_heads;
          } else {
            const uint32_t x = id / a.tiles;
            tile = id - x * a.tiles;
            it.run = x / a.c.n_heads;
            it.kh = x - it.run * a.c.n_heads;
          }
          it.unit = tile * a.c.n_heads + it.kh;
          uint32_t s = 0, p = 0;
          some = a.r.window == 0u && a.c.n_seqs <= 32 * FT_SEQS && a.r.max_new > 2 * g.toks
                     ? find_tile_heavy(a.r, a.c.n_seqs, tile, 2 * g.toks, &s, &p, a.err)
                     : find_tile(a.r, a.c.n_seqs, tile, 2 * g.toks, &s, &p, a.err);
          if (some) {
            const SeqInfo q = seq_info(a.c, a.r, s, a.err);
            it.tok0 = q.tok0;
            it.page0 = q.page0;
            it.first = q.first;
            it.i0 = p * 2 * g.toks;
            it.i1 = min(q.n, it.i0 + 2 * g.toks);
            some = it.i0 < it.i1;
            it.span = key_span(q, a.r, it.i0, max(it.i1, it.i0));
            const uint32_t n = SlotTiles<AT_KEYS>(it.span, g.box).n;
            const uint32_t per = max(a.chunk, n / a.max_chunks + 1);   // slot tiles of a run
            it.n_runs = max(1u, (n + per - 1) / per);
            it.c0 = it.run * per;
            it.n = min(per, n - min(n, it.c0));
            some = some && it.run < it.n_runs;
          }
        }
        if (!it.last && a.max_chunks > 1 && it.run == 0 && lane == 0)   // for the join of the runs
          ((JoinItem*)a.join)[it.unit] = {it.tok0 + it.i0, some ? it.i1 - it.i0 : 0u, some ? it.n_runs : 0u};
        if (some) {
          const uint32_t slot = k % AT_ITEMS;
          if (k >= AT_ITEMS) bar_wait_idle(b_item_free + 8 * slot, (k / AT_ITEMS - 1) & 1, &s_gave_up, a.err);
          if (lane == 0) s_item[slot] = it;
          __syncwarp();
          if (lane == 0) bar_arrive(b_item + 8 * slot);
          if (!it.last) bar_wait_idle(b_want, k & 1, &s_gave_up, a.err);
          ++k;
        }
        if (it.last || has_given_up(&s_gave_up)) break;
        if (lane == 0) id = gridDim.x + atomicAdd(a.counter, 1u);
        id = __shfl_sync(0xffffffffu, id, 0);
      }
      // the last CTA to leave sets the count back for the next call
      if (lane == 0 && ticket(a.counter + 1) == gridDim.x - 1) {
        a.counter[0] = 0u;
        a.counter[1] = 0u;
      }
    } else if (warp == 9) {
      // ---- loads ----
      const uint32_t boxes = AT_KEYS / g.box;
      uint32_t slot = 0, parity = 1, uses = 0, qi = 0;   // parity of the ring's round before
      for (uint32_t k = 0;; ++k) {
        const TileItem& it = item(k);
        if (it.last || has_given_up(&s_gave_up)) break;
        const uint32_t n = it.n, c0 = it.c0, kh = it.kh;
        const uint64_t page0 = it.page0;
        const SlotTiles<AT_KEYS> slots(it.span, g.box);
        if (n > 0) {
          if (qi > 0) bar_wait(b_qe, (qi - 1) & 1, &s_gave_up, a.err);
          if (lane == 0) {
            bar_expect(b_q, 2 * S::BLOCKS * g.toks * G * 128);
            for (uint32_t w = 0; w < 2; ++w)
              for (uint32_t b = 0; b < S::BLOCKS; ++b)
                tma3(sm + w * S::TILE_BYTES + b * S::BLOCK_BYTES, &g.q, b * 64, kh * G,
                     (int)(it.tok0 + it.i0 + w * g.toks), b_q);
          }
          __syncwarp();
          ++qi;
        }
        // boxes without a slot that counts are not loaded
        auto has_box = [&](const SlotTile& st) {
          const uint32_t j = st.t0 + lane * g.box;
          return lane < boxes && j < st.hi && j + g.box > st.lo;
        };
        // The page of this lane's box of a tile, looked up two tiles ahead and
        // not touched before then, so that a tile's loads never wait for it.
        auto page_of = [&](uint32_t t) -> uint32_t {
          if (t >= n) return 0u;
          const SlotTile st = slots.at(c0 + t);
          return has_box(st) ? a.c.pages[page0 + page_index(a.c, st.t0 + lane * g.box)] : 0u;
        };
        uint32_t page = page_of(0), next = page_of(1);
        const uint32_t want = n > AT_AHEAD ? n - AT_AHEAD : 0;
        if (n == 0 && lane == 0) bar_arrive(b_want);
        for (uint32_t t = 0; t < n; ++t) {
          if (t == want && lane == 0) bar_arrive(b_want);
          const uint32_t after = page_of(t + 2);
          const SlotTile st = slots.at(c0 + t);
          const uint32_t j = st.t0 + lane * g.box, y = j - page_index(a.c, j) * a.c.page_size;
          bool load = has_box(st);
          if (load && page >= a.c.n_pages) {
            record(a.err, ERR_INVAL);
            load = false;
          }
          const uint32_t loaded = __popc(__ballot_sync(0xffffffffu, load));
#pragma unroll
          for (uint32_t kv = 0; kv < 2; ++kv) {
            if (uses >= S::SLOTS) bar_wait(b_empty + 8 * slot, parity, &s_gave_up, a.err);
            if (has_given_up(&s_gave_up)) break;
            const uint32_t full = b_full + 8 * slot, dst = sm_ring + slot * S::TILE_BYTES + lane * g.box * 128;
            if (lane == 0) bar_expect(full, loaded * S::BLOCKS * g.box * 128);
            __syncwarp();
            if (load)
              for (uint32_t b = 0; b < S::BLOCKS; ++b)
                tma4(dst + b * S::BLOCK_BYTES, kv ? &g.v : &g.k, b * 64, (int)y, (int)kh, (int)page, full);
            uses = min(uses + 1, S::SLOTS);
            if (++slot == S::SLOTS) slot = 0, parity ^= 1;
          }
          page = next;
          next = after;
          if (has_given_up(&s_gave_up)) break;
        }
        release(k);
      }
    } else if (warp == 8) {
      // ---- products ----
      const uint32_t shape_s = mma_shape<T>(AT_KEYS, false), shape_o = mma_shape<T>(DP, true);
      const uint32_t one = elect_lane();
      const uint32_t q_lo = operand_lo(sm, 16), k_lo = operand_lo(sm_ring, 16), v_lo = operand_lo(sm_ring, S::BLOCK_BYTES);
      auto product_s = [&](uint32_t w, uint32_t slot) {
        const uint32_t qa = q_lo + w * (S::TILE_BYTES / 16), ka = k_lo + slot * (S::TILE_BYTES / 16);
#pragma unroll
        for (uint32_t k = 0; k < DP / 16; ++k) {
          const uint32_t off = ((k / 4) * S::BLOCK_BYTES + (k % 4) * 32) / 16;
          mma_ss(one, tm_s + w * 128, qa + off, ka + off, shape_s, k > 0);
        }
        tc_commit(one, b_s + 8 * w);
      };
      auto product_o = [&](uint32_t w, uint32_t half, uint32_t slot, bool add) {
        const uint32_t va = v_lo + slot * (S::TILE_BYTES / 16);
#pragma unroll
        for (uint32_t k = half * (AT_KEYS / 32); k < (half + 1) * (AT_KEYS / 32); ++k)
          mma_ts(one, tm_o + w * 128, tm_s + w * 128 + k * 8, va + k * (2048 / 16), shape_o, add || k > 0);
      };
      uint32_t slot = 0, parity = 0, tiles = 0, qi = 0;   // place in the ring of the next tile used, its round's parity
      auto advance = [&] {
        if (++slot == S::SLOTS) slot = 0, parity ^= 1;
      };
      for (uint32_t k = 0;; ++k) {
        const TileItem& it = item(k);
        if (it.last || has_given_up(&s_gave_up)) break;
        const uint32_t n = it.n;
        release(k);
        if (n == 0) continue;
        bar_wait(b_q, qi & 1, &s_gave_up, a.err);
        bar_wait(b_full + 8 * slot, parity, &s_gave_up, a.err);
        tc_fence_after();
        product_s(0, slot);
        product_s(1, slot);
        tc_commit(one, b_empty + 8 * slot);
        if (n == 1) tc_commit(one, b_qe);
        advance();
        for (uint32_t t = 0; t < n; ++t, ++tiles) {
          const bool more = t + 1 < n;
          const uint32_t vs = slot;
          bar_wait(b_full + 8 * vs, parity, &s_gave_up, a.err);
          advance();
#pragma unroll
          for (uint32_t w = 0; w < 2; ++w) {
            bar_wait(b_p + 16 * w, tiles & 1, &s_gave_up, a.err);
            if (t == 0 && qi > 0) bar_wait(b_oe + 8 * w, (qi - 1) & 1, &s_gave_up, a.err);   // the last item's O is read
            tc_fence_after();
            product_o(w, 0, vs, t > 0);
            bar_wait(b_p + 16 * w + 8, tiles & 1, &s_gave_up, a.err);
            tc_fence_after();
            product_o(w, 1, vs, true);
            if (w == 1) tc_commit(one, b_empty + 8 * vs);
            if (more) {
              if (w == 0) bar_wait(b_full + 8 * slot, parity, &s_gave_up, a.err);
              product_s(w, slot);
              if (w == 1) {
                tc_commit(one, b_empty + 8 * slot);
                if (t + 2 == n) tc_commit(one, b_qe);
              }
            } else {
              tc_commit(one, b_o + 8 * w);
            }
          }
          if (more) advance();
          if (has_given_up(&s_gave_up)) break;
        }
        ++qi;
      }
    }
    __syncwarp();
    asm volatile("bar.sync 0;" ::: "memory");   // every product is read
    if (*(volatile uint32_t*)&s_gave_up) __nanosleep(1000000);   // copies and products in flight end by themselves
    if (warp == 8) {
      tc_fence_after();
      tmem_free(tm, AT_TMEM_COLS);
    }
    return;
  }
  // ---- softmax: a thread a row ----
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(AT_REGS_SOFTMAX));
  const uint32_t w = warp >> 2, row = tid & 127;
  const uint32_t lanes = (warp & 3) << 21;                 // this warp's TMEM lanes
  const uint32_t ts = tm_s + w * 128 + lanes, to = tm_o + w * 128 + lanes;
  const float scale = a.r.scale_log2;
  uint32_t tiles = 0, vslot = 1, vpar = 0, done = 0;       // tiles so far; the ring's place of V; items with slots so far
  for (uint32_t k = 0;; ++k) {
    bar_wait(b_item + 8 * (k % AT_ITEMS), (k / AT_ITEMS) & 1, &s_gave_up, a.err);
    const TileItem& it = s_item[k % AT_ITEMS];
    if (it.last || has_given_up(&s_gave_up)) break;
    const uint32_t n = it.n, c0 = it.c0, i1 = it.i1, n_runs = it.n_runs;
    const SlotTiles<AT_KEYS> slots(it.span, g.box);
    const uint32_t j0 = it.i0 + w * g.toks, j1 = min(i1, j0 + g.toks);   // the row tile's tokens
    const bool live = j0 < i1;
    const uint32_t tok = j0 + row / G, head = it.kh * G + row % G;
    const bool mine = row < g.toks * G && tok < j1;
    const int64_t pos = it.first + tok;                    // the row's slot
    // The run's tiles whose every slot every row of this row tile sees: those
    // of the sinks before `sinks_all`, and [all_from, all_to).
    uint32_t sinks_all, all_from, all_to;
    {
      const int64_t a_lo = it.first + j0, a_hi = it.first + (live ? j1 : j0 + 1) - 1;
      const int64_t from = max((int64_t)slots.lo, a.r.window ? a_hi - (int64_t)a.r.window + 1 : (int64_t)0);
      const int64_t to = min((int64_t)slots.hi, a_lo + 1);
      auto tile_of = [&](int64_t x) { return x <= (int64_t)slots.first ? 0u : (uint32_t)(x - slots.first) / AT_KEYS; };
      sinks_all = slots.s_hi / AT_KEYS;
      all_from = slots.sink_tiles + tile_of(from + AT_KEYS - 1);
      all_to = slots.sink_tiles + tile_of(to);
      sinks_all = sinks_all > c0 ? sinks_all - c0 : 0;
      all_from = all_from > c0 ? all_from - c0 : 0;
      all_to = all_to > c0 ? all_to - c0 : 0;
    }
    const uint64_t out_at = (it.tok0 + tok) * a.out_tok + (uint64_t)head * a.out_head;
    const uint64_t lse_at = (it.tok0 + tok) * a.n_q_heads + head;
    const uint32_t unit = it.unit, run = it.run;
    __syncwarp();
    if (lane == 0) bar_arrive(b_item_free + 8 * (k % AT_ITEMS));
    float m = -INFINITY, l = 0.f;
    for (uint32_t t = 0; t < n; ++t, ++tiles) {
      bar_wait(b_s + 8 * w, tiles & 1, &s_gave_up, a.err);
      tc_fence_after();
      uint32_t x[AT_KEYS];
#pragma unroll
      for (int i = 0; i < 4; ++i) tc_ld32(ts + i * 32, x + i * 32);
      tc_wait_ld(x);
      const bool all = t < sinks_all || (t >= all_from && t < all_to);
      if (!all) {
        const SlotTile st = slots.at(c0 + t);
        // columns [b, e) count; of those the ones below `sinks` or from the window's first on
        const int64_t t0 = st.t0;
        const int e = (int)max((int64_t)0, min((int64_t)st.hi, pos + 1) - t0), b = (int)(st.lo - st.t0);
        int s_end = AT_KEYS, w_from = 0;
        if (a.r.window != 0u && !st.sink) {
          s_end = (int)max((int64_t)0, min((int64_t)AT_KEYS, (int64_t)a.r.sinks - t0));
          w_from = (int)max((int64_t)0, min((int64_t)AT_KEYS, pos - (int64_t)a.r.window + 1 - t0));
        }
#pragma unroll
        for (int i = 0; i < AT_KEYS; ++i) {
          const bool in = i >= b && i < e && (i < s_end || i >= w_from);
          if (!in) x[i] = 0xff800000u;
        }
        // Values no row sees must not reach the product: zero them where the
        // tile is not whole (the products of both row tiles come after this).
        if (w == 0 && (st.lo != st.t0 || st.hi != st.t0 + AT_KEYS)) {
          bar_wait(b_full + 8 * vslot, vpar, &s_gave_up, a.err);
          const uint32_t j = st.t0 + row;
          if (j < st.lo || j >= st.hi) {
#pragma unroll
            for (uint32_t i = 0; i < S::BLOCKS; ++i)
#pragma unroll
              for (uint32_t z = 0; z < 8; ++z)
                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(sm_ring + vslot * S::TILE_BYTES +
                                                                          i * S::BLOCK_BYTES + row * 128 + z * 16),
                             "r"(0u)
                             : "memory");
          }
          fence_async_smem();
        }
      }
      float mx[8];   // eight chains: one of 128 would cost its latency 128 times
#pragma unroll
      for (int i = 0; i < 8; ++i) mx[i] = fmaxf(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
#pragma unroll
      for (int i = 16; i < AT_KEYS; i += 2)
        mx[(i / 2) & 7] = fmaxf(fmaxf(mx[(i / 2) & 7], __uint_as_float(x[i])), __uint_as_float(x[i + 1]));
      const float mn = fmaxf(m, fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])),
                                      fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7]))) * scale);
      if (__any_sync(0xffffffffu, mine && mn > m + AT_SLACK<T>)) {
        // The maximum moves for the whole warp: rescale what was summed so far.
        // (Rows that are no token's have no say: theirs may hold whatever an
        // earlier kernel left, and would decide how the others are rounded.)
        const float f = mn == -INFINITY ? 1.f : ex2(m - mn);
        m = mn;
        l *= f;
        if (t > 0) {
          uint32_t o[16];
#pragma unroll 1
          for (int i = 0; i < DP / 16; ++i) {
            tc_ld16(to + i * 16, o);
            tc_wait_ld(o);
#pragma unroll
            for (int z = 0; z < 16; ++z) o[z] = __float_as_uint(__uint_as_float(o[z]) * f);
            tc_st16(to + i * 16, o);
          }
        }
      }
      const float sub = (m == -INFINITY ? 0.f : m) - WEIGHT_UP<T, AT_SLACK<T>>;   // -inf: a row that has seen nothing yet
      const uint64_t scale2 = pair(scale, scale), sub2 = pair(-sub, -sub);
      uint64_t sum[4] = {0, 0, 0, 0};   // pairs of 32-bit sums
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t p[16];
#pragma unroll
        for (int z = 0; z < 16; ++z) {
          const uint64_t y = fma_pair(pair_bits(x[i * 32 + 2 * z], x[i * 32 + 2 * z + 1]), scale2, sub2);
          const float e0 = ex2(pair_lo(y)), e1 = ex2(pair_hi(y));
          sum[z & 3] = add_pair(sum[z & 3], pair(e0, e1));
          p[z] = pack2<T>(e0, e1);   // rounded to the cache's type for the product; l sums what is not
        }
        tc_st16(ts + i * 16, p);
        if (i & 1) {   // the product of a half starts while the other's exponentials run
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(b_p + 16 * w + (i / 2) * 8);
        }
      }
      const uint64_t all4 = add_pair(add_pair(sum[0], sum[1]), add_pair(sum[2], sum[3]));
      l += pair_lo(all4) + pair_hi(all4);
      vslot += 2;
      if (vslot >= S::SLOTS) vslot -= S::SLOTS, vpar ^= 1;
    }   // (a wait that gave up ends the others at once)
    // ---- to the output, or to this run's partial result ----
    uint32_t o[DP];
    if (n > 0) {
      bar_wait(b_o + 8 * w, done & 1, &s_gave_up, a.err);
      tc_fence_after();
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) tc_ld32(to + i * 32, o + i * 32);
      tc_wait_ld(o);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(b_oe + 8 * w);
      ++done;
    } else {
#pragma unroll
      for (int i = 0; i < DP; ++i) o[i] = 0u;
    }
    const uint32_t prow = w * AT_ROWS + row;               // the row among the pair's 256
    constexpr uint32_t STEP = 2 * AT_ROWS;                 // rows of a run
    // four columns of a row together, rows next to one another: a warp's
    // accesses are whole lines
    float4* part = (float4*)a.partial + (uint64_t)unit * a.max_chunks * (DP / 4) * STEP + prow;
    float2* ml = (float2*)(a.partial + (uint64_t)a.pairs * a.max_chunks * STEP * DP) +
                 (uint64_t)unit * a.max_chunks * STEP + prow;
    if (n_runs > 1) {   // joined by attend_join_kernel
      if (mine) {
#pragma unroll
        for (int i = 0; i < DP / 4; ++i)
          __stcg(part + ((uint64_t)run * (DP / 4) + i) * STEP,
                 make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]),
                             __uint_as_float(o[4 * i + 3])));
        __stcg(ml + run * STEP, make_float2(m, l));
      }
      continue;
    }
    if (!mine) continue;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    T* out = (T*)a.out + out_at;
    uint32_t y[DP / 2];
#pragma unroll
    for (int i = 0; i < DP / 2; ++i) y[i] = pack2<T>(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
    // Each row is its thread's: 32 bytes a store where rows are aligned to
    // them, half as many stores to as many lines.
    if (g.wide) {
#pragma unroll
      for (int i = 0; i < DP / 2; i += 8)
        if ((uint32_t)i * 2 < a.c.head_dim)
          asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(out + 2 * i), "r"(y[i]), "r"(y[i + 1]),
                       "r"(y[i + 2]), "r"(y[i + 3]), "r"(y[i + 4]), "r"(y[i + 5]), "r"(y[i + 6]), "r"(y[i + 7])
                       : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < DP / 2; i += 4)
        if ((uint32_t)i * 2 < a.c.head_dim) *(uint4*)(out + 2 * i) = make_uint4(y[i], y[i + 1], y[i + 2], y[i + 3]);
    }
    if (a.lse) a.lse[lse_at] = row_lse<T, AT_SLACK<T>>(m, l);
  }
  __syncwarp();
  tc_fence_before();
  asm volatile("bar.sync 0;" ::: "memory");
}

// Joins the runs of split pairs of row tiles, in order: a thread takes four
// columns of a row, a CTA the 256 rows of a pair.  (A second launch: the last
// CTA of a pair would have to read all of its runs at one SM's rate, 2 us a run.)
template <typename T, int DP>
__global__ void __launch_bounds__(2 * AT_ROWS) attend_join_kernel(const __grid_constant__ AttendTileArgs g) {
  wait_predecessor();
  const AttendArgs& a = g.a;
  constexpr uint32_t STEP = 2 * AT_ROWS;
  const uint32_t unit = blockIdx.x / (DP / 4), c = blockIdx.x - unit * (DP / 4), prow = threadIdx.x;
  const JoinItem it = ((const JoinItem*)a.join)[unit];
  const uint32_t runs = it.runs, w = prow / AT_ROWS, row = prow % AT_ROWS;
  const uint32_t i = w * g.toks + row / a.r.group, head = (unit % a.c.n_heads) * a.r.group + row % a.r.group;
  if (runs < 2 || runs > a.max_chunks || row >= g.toks * a.r.group || i >= it.n || it.tok + i >= a.r.n_tokens) return;
  const float4* part = (const float4*)a.partial + ((uint64_t)unit * a.max_chunks * (DP / 4) + c) * STEP + prow;
  const float2* ml = (const float2*)(a.partial + (uint64_t)a.pairs * a.max_chunks * STEP * DP) +
                     (uint64_t)unit * a.max_chunks * STEP + prow;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (uint32_t r = 0; r < runs; ++r) {
    const float2 z = ml[r * STEP];
    const float4 v = part[(uint64_t)r * (DP / 4) * STEP];
    const float nm = fmaxf(m, z.x), sub = nm == -INFINITY ? 0.f : nm;
    const float f = ex2(m - sub), e = ex2(z.x - sub);
    m = nm;
    l = l * f + z.y * e;
    o.x = o.x * f + v.x * e;
    o.y = o.y * f + v.y * e;
    o.z = o.z * f + v.z * e;
    o.w = o.w * f + v.w * e;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  const uint64_t t = it.tok + i;
  if (c * 4 < a.c.head_dim)
    *(uint2*)((T*)a.out + t * a.out_tok + (uint64_t)head * a.out_head + c * 4) =
        make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
  if (c == 0 && a.lse) a.lse[t * a.n_q_heads + head] = row_lse<T, AT_SLACK<T>>(m, l);
}

// ---- host ------------------------------------------------------------------------------------
bool attend_tiles_fits(const AttendArgs& a) {
  return page_box(a.c.page_size, AT_KEYS) >= MIN_BOX && a.r.group <= AT_ROWS && a.r.scale_log2 > 0.f;
}
uint32_t attend_tile_tokens(uint32_t group) { return 2 * (AT_ROWS / group); }
size_t attend_tiles_join(const AttendArgs& a) { return (size_t)a.tiles * a.c.n_heads * sizeof(JoinItem); }
size_t attend_tiles_partial(const AttendArgs& a) {
  const size_t dp = a.c.head_dim <= 64 ? 64 : 128;
  return (size_t)a.pairs * a.max_chunks * 2 * AT_ROWS * (dp + 2) * sizeof(float);
}

template <typename T, int DP>
static void launch_tiles(const LaunchCfg& L, const AttendTileArgs& g, int sms) {
  const uint64_t items = (uint64_t)g.a.tiles * g.a.c.n_heads * g.a.max_chunks;
  launch_k(L, K_ATTEND_TILES, attend_tiles_kernel<T, DP>, (unsigned)std::min<uint64_t>(items, (uint64_t)sms), AT_THREADS,
           TileShape<DP>::SMEM, g);
  if (g.a.max_chunks > 1)
    launch_k(L, K_ATTEND_JOIN, attend_join_kernel<T, DP>, g.a.tiles * g.a.c.n_heads * (DP / 4), 2 * AT_ROWS, 0, g);
}
bool launch_attend_tiles(const LaunchCfg& L, const AttendArgs& a, int dtype, int sms) {
  AttendTileArgs g;
  g.a = a;
  g.toks = AT_ROWS / a.r.group;
  g.box = page_box(a.c.page_size, AT_KEYS);
  g.wide = a.c.head_dim % 16 == 0 && a.out_tok % 16 == 0 && a.out_head % 16 == 0 &&
           reinterpret_cast<uintptr_t>(a.out) % 32 == 0;
  if (!rows_map(&g.q, a.r, a.c.head_dim, a.n_q_heads, dtype, a.r.group, g.toks) || !pool_map(&g.k, a.c, a.c.k, dtype, g.box) ||
      !pool_map(&g.v, a.c, a.c.v, dtype, g.box))
    return false;
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == RO_BF16)
    narrow ? launch_tiles<__nv_bfloat16, 64>(L, g, sms) : launch_tiles<__nv_bfloat16, 128>(L, g, sms);
  else
    narrow ? launch_tiles<__half, 64>(L, g, sms) : launch_tiles<__half, 128>(L, g, sms);
  return true;
}

template <typename T, int DP>
static cudaError_t allow() {
  return cudaFuncSetAttribute(attend_tiles_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)TileShape<DP>::SMEM);
}
cudaError_t prepare_attend_tiles_kernels() {
  for (cudaError_t e : {allow<__nv_bfloat16, 64>(), allow<__nv_bfloat16, 128>(), allow<__half, 64>(), allow<__half, 128>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
