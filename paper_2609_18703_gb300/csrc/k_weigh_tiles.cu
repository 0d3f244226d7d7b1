// k_weigh_tiles.cu — the attention weight cached tokens gathered
// (ro_cache_weigh) from chunks of rows, on the fifth-generation tensor cores.
//
//   S^T = K Q^T,  score_j = decay past_j + sum_r exp2(scale log2(e) S_jr - lse_r log2(e))
//
// Bound by the exponentials (one a pair of a row and a slot it sees; for heads
// of 64 dimensions the products take half their time).  An item is 128 slots of
// one head of one sequence and the row tiles that can see one of them: slots are
// the rows of the product, so a thread owns a slot and adds up its columns, in
// order, without talking to anyone.  A warp finds work, a warp of TMA loads, a
// warp of products and two groups of four warps that take the row tiles in
// turn; two CTAs share an SM, so that some warps always have exponentials.
// CTAs stay and take items as they get free: an item of 16 row tiles has 11 us
// of work, and started and ended by a CTA of its own it took 2 us more, in which
// its half of the SM had nothing to do.
//
// Measured: 6 chunks of up to 1,024 tokens over up to 16,384 slots, 16 heads on
// 4 of 64: 87 us (a CTA an item: 103; mma.sync: 358).  Beside the exponentials
// (the XU needs 50 us for them) the broadcast of the rows' lse from shared memory
// costs about 10 us and the products' and barriers' latencies the rest.  Row tiles
// of 64 (with a second S a group, a third group or two slots a thread), S freed in
// halves, polynomials for a part of the exponentials and the lse subtracted by a
// product measured slower; more registers for deeper loads of S gave 2 %.
#include <algorithm>

#include "ro_tcgen05.cuh"

namespace ro {

constexpr int WT_THREADS = 352, WT_ROWS = 128;
constexpr uint32_t WT_TMEM_COLS = 256;

template <int DP>
struct WeighShape {
  static constexpr uint32_t BLOCKS = DP / 64, BLOCK_BYTES = 128 * 128, TILE_BYTES = BLOCKS * BLOCK_BYTES;
  static constexpr uint32_t KEYS = DP == 64 ? 2 : 1;       // key tiles: two where half of an SM's shared memory holds them
  static constexpr uint32_t STAGES = DP == 64 ? 4 : 2;     // row tiles in the ring
  static constexpr uint32_t SMEM = 1024 + (KEYS + STAGES) * TILE_BYTES;
};

// A piece of work: 128 slots of one sequence and head, and the tokens that see
// one of them.
struct WeighItem {
  uint64_t tok0, at;         // the sequence's first token; the first slot's score
  int64_t first;             // slot of that token
  uint32_t i0, i1, n;        // tokens, row tiles
  uint32_t j_lo, j_hi, kh;
  uint32_t last;             // no work: the end
  uint32_t page[32];         // of each box of slots
};
constexpr uint32_t WT_ITEMS = 2;
constexpr uint32_t WT_AHEAD = 4;   // the next item is taken this many row tiles before the loads of the present one end

// Of a sequence whose tokens have a window: the tiles [0, sinks) of the sinks,
// then from tile `window` on; those between are seen by no token.
struct SeenTiles {
  uint32_t sinks, window;
};
__device__ __forceinline__ SeenTiles seen_tiles(const SeqInfo& q, const RowsArgs& r) {
  const int64_t lo = q.first - (int64_t)r.window + 1;   // the first slot of the first token's window
  SeenTiles s;
  s.window = lo > 0 ? (uint32_t)(lo / WT_KEYS) : 0u;
  s.sinks = min((r.sinks + WT_KEYS - 1) / WT_KEYS, s.window);
  return s;
}
__device__ __forceinline__ uint32_t scored(const WeighArgs& a, const SeqInfo& q, bool first) {
  if (q.len > a.score_cap) {
    if (first) record(a.err, ERR_CAPACITY);
    return (uint32_t)a.score_cap;
  }
  return q.len;
}

// decay * past for the slots that no token sees
constexpr int WP_THREADS = 256;
__global__ void __launch_bounds__(WP_THREADS) weigh_past_kernel(const __grid_constant__ WeighArgs a) {
  wait_predecessor();
  const uint32_t unit = blockIdx.x / a.chunk, part = blockIdx.x - unit * a.chunk;   // a.chunk CTAs for each
  const SeqInfo q = seq_info(a.c, a.r, unit / a.c.n_heads, a.err);
  const SeenTiles st = seen_tiles(q, a.r);
  const uint32_t from = st.sinks * WT_KEYS, to = min(scored(a, q, false), st.window * WT_KEYS);
  if (from >= to) return;
  const uint32_t per = ((to - from + a.chunk - 1) / a.chunk + 3) & ~3u, lo = from + min(to - from, part * per);
  decay_past<WP_THREADS>(a, (uint64_t)unit * a.score_cap, lo, min(to, lo + per), threadIdx.x);   // (no new slot among them)
}

template <typename T, int DP>
__global__ void __launch_bounds__(WT_THREADS, 2) weigh_tiles_kernel(const __grid_constant__ WeighTileArgs g) {
  using S = WeighShape<DP>;
  const WeighArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[2 * S::KEYS + 2 * S::STAGES + 8 + 2 * WT_ITEMS + 1];
  __shared__ __align__(16) float s_lse[2][2][WT_ROWS];   // minus lse log2(e), by group and turn
  __shared__ int32_t s_tok[2][2][WT_ROWS];               // the row's token
  __shared__ float s_sum[WT_ITEMS][WT_KEYS];
  __shared__ WeighItem s_item[WT_ITEMS];
  __shared__ uint32_t s_tmem, s_gave_up;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t G = a.r.group;
  const uint32_t sm = (step_smem(smem_raw) + 1023u) & ~1023u, sm_q = sm + S::KEYS * S::TILE_BYTES;
  // full / empty: keys, rows; of each group S, its lse; sums, items
  const uint32_t b_k = step_smem(s_bar), b_ke = b_k + 8 * S::KEYS, b_full = b_ke + 8 * S::KEYS,
                 b_empty = b_full + 8 * S::STAGES, b_s = b_empty + 8 * S::STAGES, b_free = b_s + 16, b_z = b_free + 16,
                 b_sum = b_z + 16, b_item = b_sum + 16, b_item_free = b_item + 8 * WT_ITEMS,
                 b_want = b_item_free + 8 * WT_ITEMS;
  if (tid == 0) {
    s_gave_up = 0;
    bar_init(b_want, 1);
    for (uint32_t i = 0; i < S::KEYS; ++i) {
      bar_init(b_k + 8 * i, 1);
      bar_init(b_ke + 8 * i, 1);
    }
    for (uint32_t i = 0; i < S::STAGES; ++i) {
      bar_init(b_full + 8 * i, 1);
      bar_init(b_empty + 8 * i, 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      bar_init(b_s + 8 * i, 1);
      bar_init(b_free + 8 * i, 4);
      bar_init(b_z + 8 * i, 4);
      bar_init(b_sum + 8 * i, 4);
    }
    for (uint32_t i = 0; i < WT_ITEMS; ++i) {
      bar_init(b_item + 8 * i, 1);
      bar_init(b_item_free + 8 * i, 10);   // 8 warps of exponentials, loads, products
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 8) tmem_alloc(step_smem(&s_tmem), WT_TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = __shfl_sync(0xffffffffu, s_tmem, 0);   // 128 columns for each group

  // the k-th item, to a whole warp; released once its reader is done with it
  auto item = [&](uint32_t k) -> const WeighItem& {
    bar_wait(b_item + 8 * (k % WT_ITEMS), (k / WT_ITEMS) & 1, &s_gave_up, a.err);
    return s_item[k % WT_ITEMS];
  };
  auto release = [&](uint32_t k) {
    __syncwarp();
    if (lane == 0) bar_arrive(b_item_free + 8 * (k % WT_ITEMS));
  };
  if (warp == 10) {
    // ---- work ----
    // The sequences' tiles of slots in order, the heads of a tile together: the
    // first item by the CTA's number, the others as they are asked for.  Numbers
    // only grow, so each lane walks the list once, 32 sequences at a time.
    uint32_t s0 = 0, mine = 0, upto = 0, k = 0;   // the lane's sequence's tiles, those of the lanes up to it
    uint64_t before = 0;                          // tiles of the sequences before s0
    SeqInfo q = {};
    auto walk = [&] {
      const uint32_t s = s0 + lane;
      mine = 0;
      if (s < a.c.n_seqs) {
        q = seq_info(a.c, a.r, s, a.err);
        if (!q.ok)
          record(a.err, ERR_INVAL);
        else if (q.len != a.r.len[s])
          record(a.err, ERR_CAPACITY);
        mine = (scored(a, q, true) + WT_KEYS - 1) / WT_KEYS;
        if (a.unseen) {
          const SeenTiles st = seen_tiles(q, a.r);
          mine = mine > st.window ? mine - (st.window - st.sinks) : min(mine, st.sinks);
        }
      }
      upto = warp_incl_scan(mine);
    };
    walk();
    for (uint32_t id = blockIdx.x;;) {
      const uint32_t rank = id / a.c.n_heads;
      WeighItem it = {};
      it.kh = id - rank * a.c.n_heads;
      while (s0 < a.c.n_seqs && rank >= before + __shfl_sync(0xffffffffu, upto, 31)) {
        before += __shfl_sync(0xffffffffu, upto, 31);
        s0 += 32;
        if (s0 < a.c.n_seqs) walk();
      }
      it.last = s0 >= a.c.n_seqs;
      it.n = 0;
      uint32_t page = 0;
      if (!it.last) {
        const uint32_t want = (uint32_t)(rank - before);
        const int l = __ffs(__ballot_sync(0xffffffffu, upto > want)) - 1;
        uint32_t tile = want - __shfl_sync(0xffffffffu, upto - mine, l);
        SeqInfo x;
        x.tok0 = __shfl_sync(0xffffffffu, q.tok0, l);
        x.page0 = __shfl_sync(0xffffffffu, q.page0, l);
        x.first = __shfl_sync(0xffffffffu, q.first, l);
        x.n = __shfl_sync(0xffffffffu, q.n, l);
        x.len = __shfl_sync(0xffffffffu, q.len, l);
        if (a.unseen) {
          const SeenTiles st = seen_tiles(x, a.r);
          if (tile >= st.sinks) tile += st.window - st.sinks;
        }
        it.tok0 = x.tok0;
        it.first = x.first;
        it.j_lo = tile * WT_KEYS;
        it.j_hi = min(scored(a, x, false), it.j_lo + WT_KEYS) - 1;
        it.at = ((uint64_t)(s0 + l) * a.c.n_heads + it.kh) * a.score_cap + it.j_lo;
        seeing_tokens(x, a.r, it.j_lo, it.j_hi, &it.i0, &it.i1);
        it.n = (it.i1 - it.i0 + g.toks - 1) / g.toks;
        if (it.n == 0) {   // no token sees them
          for (uint32_t j = it.j_lo + lane; j <= it.j_hi; j += 32) {
            const uint64_t at = it.at + (j - it.j_lo);
            a.score[at] = a.past && (int64_t)j < it.first ? a.decay * a.past[at] : 0.f;
          }
        } else {
          const uint32_t j = it.j_lo + lane * g.box;
          if (lane < WT_KEYS / g.box && j <= it.j_hi) page = a.c.pages[x.page0 + page_index(a.c, j)];
        }
      }
      if (it.last || it.n > 0) {
        const uint32_t slot = k % WT_ITEMS;
        if (k >= WT_ITEMS) bar_wait_idle(b_item_free + 8 * slot, (k / WT_ITEMS - 1) & 1, &s_gave_up, a.err);
        WeighItem& to = s_item[slot];
        if (lane == 0) {
          to.tok0 = it.tok0, to.at = it.at, to.first = it.first;
          to.i0 = it.i0, to.i1 = it.i1, to.n = it.n;
          to.j_lo = it.j_lo, to.j_hi = it.j_hi, to.kh = it.kh, to.last = it.last;
        }
        to.page[lane] = page;
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
    uint32_t slot = 0, parity = 1, uses = 0;   // parity of the ring's round before
    for (uint32_t k = 0;; ++k) {
      const WeighItem& it = item(k);
      if (it.last || has_given_up(&s_gave_up)) break;
      const uint32_t n = it.n, kh = it.kh, j = it.j_lo + lane * g.box, page = it.page[lane], kb = k % S::KEYS;
      const uint64_t tok = it.tok0 + it.i0;
      bool load = lane < WT_KEYS / g.box && j <= it.j_hi;
      release(k);
      if (load && page >= a.c.n_pages) {
        record(a.err, ERR_INVAL);
        load = false;
      }
      const uint32_t loaded = __popc(__ballot_sync(0xffffffffu, load));
      if (k >= S::KEYS) bar_wait(b_ke + 8 * kb, (k / S::KEYS - 1) & 1, &s_gave_up, a.err);
      if (has_given_up(&s_gave_up)) break;
      if (lane == 0) bar_expect(b_k + 8 * kb, loaded * S::BLOCKS * g.box * 128);
      __syncwarp();
      if (load)
        for (uint32_t b = 0; b < S::BLOCKS; ++b)
          tma4(sm + kb * S::TILE_BYTES + b * S::BLOCK_BYTES + lane * g.box * 128, &g.k, b * 64,
               (int)(j - page_index(a.c, j) * a.c.page_size), (int)kh, (int)page, b_k + 8 * kb);
      const uint32_t want = n > WT_AHEAD ? n - WT_AHEAD : 0;
      for (uint32_t t = 0; t < n; ++t) {
        if (t == want && lane == 0) bar_arrive(b_want);
        if (uses >= S::STAGES) bar_wait(b_empty + 8 * slot, parity, &s_gave_up, a.err);
        if (has_given_up(&s_gave_up)) break;
        if (lane == 0) {
          const uint32_t rows = g.toks * G;   // fewer than a tile's where the group does not divide it
          bar_expect(b_full + 8 * slot, S::TILE_BYTES);
          for (uint32_t b = 0; b < S::BLOCKS; ++b) {
            const uint32_t dst = sm_q + slot * S::TILE_BYTES + b * S::BLOCK_BYTES;
            tma3(dst, &g.q, b * 64, (int)(kh * G), (int)(tok + t * g.toks), b_full + 8 * slot);
            if (rows < WT_ROWS)
              tma3(dst + rows * 128, &g.fill, b * 64, (int)(kh * G), (int)(tok + t * g.toks), b_full + 8 * slot);
          }
        }
        __syncwarp();
        uses = min(uses + 1, S::STAGES);
        if (++slot == S::STAGES) slot = 0, parity ^= 1;
      }
    }
  } else if (warp == 8) {
    // ---- products ----
    const uint32_t shape = mma_shape<T>(WT_ROWS, false), one = elect_lane();
    const uint32_t k_lo = operand_lo(sm, 16), q_lo = operand_lo(sm_q, 16);
    uint32_t slot = 0, parity = 0, tiles = 0;   // row tiles so far
    for (uint32_t k = 0;; ++k) {
      const WeighItem& it = item(k);
      if (it.last || has_given_up(&s_gave_up)) break;
      const uint32_t n = it.n, kb = k % S::KEYS, ka = k_lo + kb * (S::TILE_BYTES / 16);
      release(k);
      bar_wait(b_k + 8 * kb, (k / S::KEYS) & 1, &s_gave_up, a.err);
      for (uint32_t t = 0; t < n; ++t, ++tiles) {
        const uint32_t w = tiles & 1;
        bar_wait(b_full + 8 * slot, parity, &s_gave_up, a.err);
        if (tiles >= 2) bar_wait(b_free + 8 * w, (tiles / 2 - 1) & 1, &s_gave_up, a.err);
        tc_fence_after();
#pragma unroll
        for (uint32_t x = 0; x < DP / 16; ++x) {
          const uint32_t off = ((x / 4) * S::BLOCK_BYTES + (x % 4) * 32) / 16;
          mma_ss(one, tm + w * 128, ka + off, q_lo + slot * (S::TILE_BYTES / 16) + off, shape, x > 0);
        }
        tc_commit(one, b_s + 8 * w);
        tc_commit(one, b_empty + 8 * slot);
        if (t + 1 == n) tc_commit(one, b_ke + 8 * kb);
        if (has_given_up(&s_gave_up)) break;
        if (++slot == S::STAGES) slot = 0, parity ^= 1;
      }
    }
  } else {
    // ---- exponentials: a thread a slot ----
    const uint32_t w = warp >> 2, row = tid & 127, ts = tm + w * 128 + ((warp & 3) << 21);
    const uint64_t scale2 = pair(a.r.scale_log2, a.r.scale_log2);
    uint32_t tiles = 0;      // row tiles of the items before: the groups take them in turn
    for (uint32_t k = 0;; ++k) {
      const WeighItem& it = item(k);
      if (it.last || has_given_up(&s_gave_up)) break;
      const uint32_t n = it.n, i0 = it.i0, i1 = it.i1, kh = it.kh, j_lo = it.j_lo, j_hi = it.j_hi, j = j_lo + row;
      const uint64_t tok0 = it.tok0, at = it.at + row;
      const int64_t first = it.first;
      // the tokens [see_lo, see_hi) of the chunk see this slot
      const int64_t d = (int64_t)j - first;
      const int32_t see_lo = (int32_t)max((int64_t)0, min(d, (int64_t)INT32_MAX));
      const int32_t see_hi = a.r.window == 0u || j < a.r.sinks
                                 ? INT32_MAX
                                 : (int32_t)max((int64_t)0, min(d + (int64_t)a.r.window, (int64_t)INT32_MAX));
      // Row tiles [from, to) see all of the CTA's slots with every row: their
      // first token sees the last slot, their last one (they are full) the first.
      uint32_t from, to = (i1 - i0) / g.toks;
      {
        const int64_t x = (int64_t)j_hi - first - i0;       // the first token that sees the last slot, from i0 on
        from = x <= 0 ? 0u : (uint32_t)((x + g.toks - 1) / g.toks);
        if (a.r.window != 0u) {
          const int64_t y = (int64_t)j_lo + a.r.window - first - i0;   // tokens before it see the first slot
          to = min(to, y <= 0 ? 0u : (uint32_t)min(y / g.toks, (int64_t)INT32_MAX));
        }
      }
      uint64_t acc[4] = {0, 0, 0, 0};   // pairs of 32-bit sums
      // this thread's row of a tile, fetched a turn ahead: minus its lse, -inf for
      // rows past the end and rows that see nothing (they add 0); LSE_FILL for rows
      // that fill up a tile
      const float* lse = a.lse + (tok0 + i0 + row / G) * a.n_q_heads + kh * G + row % G;
      auto row_lse = [&](uint32_t t) -> float {
        if (row >= g.toks * G) return LSE_FILL * LN2;
        if (t >= n || i0 + t * g.toks + row / G >= i1) return INFINITY;
        return lse[(uint64_t)t * g.toks * a.n_q_heads];
      };
      uint32_t t = (w ^ tiles) & 1;
      float next = row_lse(t);
      for (; t < n; t += 2) {
        const uint32_t t0 = i0 + t * g.toks, turn = (tiles + t) >> 1, buf = turn & 1;
        s_lse[w][buf][row] = next == -INFINITY ? -INFINITY : next * -1.44269504088896340736f;
        s_tok[w][buf][row] = row < g.toks * G && t0 + row / G < i1 ? (int32_t)(t0 + row / G) : -1;
        next = row_lse(t + 2);
        __syncwarp();
        if (lane == 0) bar_arrive(b_z + 8 * w);
        bar_wait(b_z + 8 * w, turn & 1, &s_gave_up, a.err);
        bar_wait(b_s + 8 * w, turn & 1, &s_gave_up, a.err);
        tc_fence_after();
        const float4* z4 = (const float4*)s_lse[w][buf];
        if (t >= from && t < to) {
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            uint32_t x[32];
            tc_ld32(ts + i * 32, x);
            tc_wait_ld(x);
#pragma unroll
            for (int z = 0; z < 8; ++z) {
              const float4 l = z4[i * 8 + z];
              const uint64_t y0 = fma_pair(pair_bits(x[4 * z], x[4 * z + 1]), scale2, pair(l.x, l.y));
              const uint64_t y1 = fma_pair(pair_bits(x[4 * z + 2], x[4 * z + 3]), scale2, pair(l.z, l.w));
              acc[(2 * z) & 3] = add_pair(acc[(2 * z) & 3], pair(ex2(pair_lo(y0)), ex2(pair_hi(y0))));
              acc[(2 * z + 1) & 3] = add_pair(acc[(2 * z + 1) & 3], pair(ex2(pair_lo(y1)), ex2(pair_hi(y1))));
            }
          }
        } else {
          // rows whose tokens see this slot; what other rows hold (another sequence's) is not looked at
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            uint32_t x[32];
            tc_ld32(ts + i * 32, x);
            tc_wait_ld(x);
#pragma unroll
            for (int z = 0; z < 32; ++z) {
              const int32_t tok = s_tok[w][buf][i * 32 + z];
              const float p = ex2(fmaf(__uint_as_float(x[z]), a.r.scale_log2, s_lse[w][buf][i * 32 + z]));
              acc[z & 3] = add_pair(acc[z & 3], pair(tok >= see_lo && tok < see_hi ? p : 0.f, 0.f));
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(b_free + 8 * w);
      }   // (a wait that gave up ends the others at once)
      tiles += n;
      const uint64_t tot = add_pair(add_pair(acc[0], acc[1]), add_pair(acc[2], acc[3]));
      const float sum = pair_lo(tot) + pair_hi(tot);
      if (w == 1) {
        s_sum[k % WT_ITEMS][row] = sum;
        __syncwarp();
        if (lane == 0) bar_arrive(b_sum + 8 * (k % WT_ITEMS));
      } else {
        bar_wait(b_sum + 8 * (k % WT_ITEMS), (k / WT_ITEMS) & 1, &s_gave_up, a.err);
        if (j <= j_hi) {
          const float past = a.past && (int64_t)j < first ? a.decay * a.past[at] : 0.f;
          a.score[at] = past + (sum + s_sum[k % WT_ITEMS][row]);
        }
      }
      release(k);   // the other group's sums may be written again
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*(volatile uint32_t*)&s_gave_up) __nanosleep(1000000);   // copies and products in flight end by themselves
  if (warp == 8) {
    tc_fence_after();
    tmem_free(tm, WT_TMEM_COLS);
  }
}

bool weigh_tiles_fits(const WeighArgs& a) {
  return page_box(a.c.page_size, WT_KEYS) >= MIN_BOX && a.r.group <= WT_ROWS;
}

template <typename T, int DP>
static void launch_tiles(const LaunchCfg& L, const WeighTileArgs& g, int sms) {
  const uint64_t items = (uint64_t)g.a.tiles * g.a.c.n_seqs * g.a.c.n_heads;
  launch_k(L, K_WEIGH_TILES, weigh_tiles_kernel<T, DP>, (unsigned)std::min<uint64_t>(items, (uint64_t)sms * 2), WT_THREADS,
           WeighShape<DP>::SMEM, g);
}
bool launch_weigh_tiles(const LaunchCfg& L, const WeighArgs& a, int dtype, int sms) {
  WeighTileArgs g;
  g.a = a;
  g.toks = WT_ROWS / a.r.group;
  g.box = page_box(a.c.page_size, WT_KEYS);
  const uint32_t fill = WT_ROWS - g.toks * a.r.group;   // fewer than the group
  if (!rows_map(&g.q, a.r, a.c.head_dim, a.n_q_heads, dtype, a.r.group, g.toks) ||
      !pool_map(&g.k, a.c, a.c.k, dtype, g.box) ||
      (fill && !rows_map(&g.fill, a.r, a.c.head_dim, a.n_q_heads, dtype, fill, 1)))
    return false;
  if (a.unseen) {
    WeighArgs p = a;
    const uint64_t units = (uint64_t)a.c.n_seqs * a.c.n_heads;
    p.chunk = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(a.score_cap, WP_THREADS * 8),
                                                                  ceil_div((uint64_t)sms * 8, units)));
    launch_k(L, K_WEIGH, weigh_past_kernel, (unsigned)(units * p.chunk), WP_THREADS, 0, p);
  }
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == RO_BF16)
    narrow ? launch_tiles<__nv_bfloat16, 64>(L, g, sms) : launch_tiles<__nv_bfloat16, 128>(L, g, sms);
  else
    narrow ? launch_tiles<__half, 64>(L, g, sms) : launch_tiles<__half, 128>(L, g, sms);
  return true;
}

template <typename T, int DP>
static cudaError_t allow() {
  return cudaFuncSetAttribute(weigh_tiles_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)WeighShape<DP>::SMEM);
}
cudaError_t prepare_weigh_tiles_kernels() {
  for (cudaError_t e : {allow<__nv_bfloat16, 64>(), allow<__nv_bfloat16, 128>(), allow<__half, 64>(), allow<__half, 128>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
