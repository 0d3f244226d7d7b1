// k_weigh_tiles.cu — the attention weight cached tokens gathered
// (ro_cache_weigh) from chunks of rows, on the fifth-generation tensor cores.
//
//   S^T = K Q^T,  score_j = decay past_j + sum_r exp2(scale log2(e) S_jr - lse_r log2(e))
//
// Bound by the exponentials (one a pair of a row and a slot it sees; for heads
// of 64 dimensions the products take half their time).  A CTA holds 128 slots
// of one head of one sequence and runs over the row tiles that can see one of
// them: slots are the rows of the product, so a thread owns a slot and adds up
// its columns, in order, without talking to anyone.  A warp of TMA loads, a
// warp of products and two groups of four warps that take the row tiles in
// turn; two CTAs share an SM, so that some warps always have exponentials.
//
// Measured: 6 chunks of up to 1,024 tokens over up to 16,384 slots, 16 heads on
// 4 of 64: 103 us, the XU 49 % busy (mma.sync: 358 us).  Row tiles of 64, with a
// second S a group or two slots a thread, measured slower (105 to 131 us): each
// tile costs about 900 cycles beside its exponentials.
#include <algorithm>

#include "ro_tcgen05.cuh"

namespace ro {

constexpr int WT_THREADS = 320, WT_ROWS = 128;
constexpr uint32_t WT_STAGES = 2, WT_TMEM_COLS = 256;

template <int DP>
struct WeighShape {
  static constexpr uint32_t BLOCKS = DP / 64, BLOCK_BYTES = 128 * 128, TILE_BYTES = BLOCKS * BLOCK_BYTES;
  static constexpr uint32_t SMEM = 1024 + (1 + WT_STAGES) * TILE_BYTES;
};

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
  const uint32_t to = min(scored(a, q, false), st.window * WT_KEYS);
  const uint64_t row = (uint64_t)unit * a.score_cap;
  for (uint32_t j = st.sinks * WT_KEYS + part * WP_THREADS + threadIdx.x; j < to; j += a.chunk * WP_THREADS)
    a.score[row + j] = a.past ? a.decay * a.past[row + j] : 0.f;   // (before the window: no new slot)
}

template <typename T, int DP>
__global__ void __launch_bounds__(WT_THREADS, 2) weigh_tiles_kernel(const __grid_constant__ WeighTileArgs g) {
  using S = WeighShape<DP>;
  const WeighArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[1 + 2 * WT_STAGES + 4];
  __shared__ __align__(16) float s_lse[2][2][WT_ROWS];   // minus lse log2(e), by group and turn
  __shared__ int32_t s_tok[2][2][WT_ROWS];               // the row's token
  __shared__ float s_sum[WT_KEYS];
  __shared__ uint32_t s_tmem, s_gave_up;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t kh = blockIdx.x % a.c.n_heads, rest = blockIdx.x / a.c.n_heads;
  const uint32_t seq = rest / a.tiles;
  uint32_t tile = rest - seq * a.tiles;
  const SeqInfo q = seq_info(a.c, a.r, seq, a.err);
  const uint32_t len = scored(a, q, tile == 0 && tid == 0);
  if (a.unseen) {
    const SeenTiles st = seen_tiles(q, a.r);
    if (tile >= st.sinks) tile += st.window - st.sinks;
  }
  const uint64_t j0 = (uint64_t)tile * WT_KEYS;
  if (j0 >= len) return;
  const uint32_t j_lo = (uint32_t)j0, j_hi = min(len, j_lo + WT_KEYS) - 1;
  uint32_t i0, i1;
  seeing_tokens(q, a.r, j_lo, j_hi, &i0, &i1);
  const uint32_t G = a.r.group;
  const uint32_t n = (i1 - i0 + g.toks - 1) / g.toks;   // row tiles
  const uint64_t at = ((uint64_t)seq * a.c.n_heads + kh) * a.score_cap + j_lo + tid;   // this thread's slot's score
  if (n == 0) {
    if (tid < WT_KEYS && j_lo + tid <= j_hi)
      a.score[at] = a.past && (int64_t)(j_lo + tid) < q.first ? a.decay * a.past[at] : 0.f;
    return;
  }

  const uint32_t sm = (step_smem(smem_raw) + 1023u) & ~1023u, sm_q = sm + S::TILE_BYTES;
  const uint32_t b_k = step_smem(s_bar), b_full = b_k + 8, b_empty = b_full + 8 * WT_STAGES, b_s = b_empty + 8 * WT_STAGES,
                 b_free = b_s + 16;
  if (tid == 0) {
    s_gave_up = 0;
    bar_init(b_k, 1);
    for (uint32_t i = 0; i < WT_STAGES; ++i) {
      bar_init(b_full + 8 * i, 1);
      bar_init(b_empty + 8 * i, 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      bar_init(b_s + 8 * i, 1);
      bar_init(b_free + 8 * i, 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  // rows that no tile has (the group does not divide 128) are zero: their product is 0, their weight exp2(-inf)
  for (uint32_t x = g.toks * G * 8 + tid; x < WT_ROWS * 8; x += WT_THREADS)
    for (uint32_t b = 0; b < WT_STAGES * S::BLOCKS; ++b)
      asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(sm_q + b * S::BLOCK_BYTES + x * 16), "r"(0u) : "memory");
  fence_async_smem();
  if (warp == 8) tmem_alloc(step_smem(&s_tmem), WT_TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = __shfl_sync(0xffffffffu, s_tmem, 0);   // 128 columns for each group

  float sum = 0.f;
  if (warp == 9) {
    // ---- loads ----
    {
      const uint32_t j = j_lo + lane * g.box;
      bool load = lane < WT_KEYS / g.box && j <= j_hi;
      uint32_t page = 0;
      if (load) {
        page = a.c.pages[q.page0 + page_index(a.c, j)];
        if (page >= a.c.n_pages) {
          record(a.err, ERR_INVAL);
          load = false;
        }
      }
      const uint32_t loaded = __popc(__ballot_sync(0xffffffffu, load));
      if (lane == 0) bar_expect(b_k, loaded * S::BLOCKS * g.box * 128);
      __syncwarp();
      if (load)
        for (uint32_t b = 0; b < S::BLOCKS; ++b)
          tma4(sm + b * S::BLOCK_BYTES + lane * g.box * 128, &g.k, b * 64, (int)(j - page_index(a.c, j) * a.c.page_size), (int)kh,
               (int)page, b_k);
      uint32_t slot = 0, parity = 1;
      for (uint32_t t = 0; t < n; ++t) {
        if (t >= WT_STAGES) bar_wait(b_empty + 8 * slot, parity, &s_gave_up, a.err);
        if (has_given_up(&s_gave_up)) break;
        if (lane == 0) {
          bar_expect(b_full + 8 * slot, S::BLOCKS * g.toks * G * 128);
          for (uint32_t b = 0; b < S::BLOCKS; ++b)
            tma3(sm_q + slot * S::TILE_BYTES + b * S::BLOCK_BYTES, &g.q, b * 64, (int)(kh * G),
                 (int)(q.tok0 + i0 + t * g.toks), b_full + 8 * slot);
        }
        __syncwarp();
        if (++slot == WT_STAGES) slot = 0, parity ^= 1;
      }
    }
  } else if (warp == 8) {
    // ---- products ----
    const uint32_t shape = mma_shape<T>(WT_ROWS, false), one = elect_lane();
    const uint32_t k_lo = operand_lo(sm, 16), q_lo = operand_lo(sm_q, 16);
    bar_wait(b_k, 0, &s_gave_up, a.err);
    uint32_t slot = 0, parity = 0;
    for (uint32_t t = 0; t < n; ++t) {
      const uint32_t w = t & 1;
      bar_wait(b_full + 8 * slot, parity, &s_gave_up, a.err);
      if (t >= 2) bar_wait(b_free + 8 * w, (t / 2 - 1) & 1, &s_gave_up, a.err);
      tc_fence_after();
#pragma unroll
      for (uint32_t k = 0; k < DP / 16; ++k) {
        const uint32_t off = ((k / 4) * S::BLOCK_BYTES + (k % 4) * 32) / 16;
        mma_ss(one, tm + w * 128, k_lo + off, q_lo + slot * (S::TILE_BYTES / 16) + off, shape, k > 0);
      }
      tc_commit(one, b_s + 8 * w);
      tc_commit(one, b_empty + 8 * slot);
      if (has_given_up(&s_gave_up)) break;
      if (++slot == WT_STAGES) slot = 0, parity ^= 1;
    }
  } else {
    // ---- exponentials: a thread a slot ----
    const uint32_t w = warp >> 2, row = tid & 127, ts = tm + w * 128 + ((warp & 3) << 21);
    const uint32_t j = j_lo + row;
    const uint64_t scale2 = pair(a.r.scale_log2, a.r.scale_log2);
    // the tokens [see_lo, see_hi) of the chunk see this slot
    const int64_t d = (int64_t)j - q.first;
    const int32_t see_lo = (int32_t)max((int64_t)0, min(d, (int64_t)INT32_MAX));
    const int32_t see_hi = a.r.window == 0u || j < a.r.sinks
                               ? INT32_MAX
                               : (int32_t)max((int64_t)0, min(d + (int64_t)a.r.window, (int64_t)INT32_MAX));
    uint64_t acc[4] = {0, 0, 0, 0};   // pairs of 32-bit sums
    // this thread's row of a tile, fetched a turn ahead: minus its lse, -inf for
    // rows past the end and rows that see nothing (they add 0)
    auto row_lse = [&](uint32_t t) -> float {
      const uint32_t i = i0 + t * g.toks + row / G;
      if (t >= n || row >= g.toks * G || i >= i1) return INFINITY;
      return a.lse[(q.tok0 + i) * a.n_q_heads + kh * G + row % G];
    };
    float next = row_lse(w);
    for (uint32_t t = w; t < n; t += 2) {
      const uint32_t t0 = i0 + t * g.toks, buf = (t >> 1) & 1;
      s_lse[w][buf][row] = next == -INFINITY ? -INFINITY : next * -1.44269504088896340736f;
      s_tok[w][buf][row] = row < g.toks * G && t0 + row / G < i1 ? (int32_t)(t0 + row / G) : -1;
      next = row_lse(t + 2);
      if (w == 0)
        asm volatile("bar.sync 1, 128;" ::: "memory");
      else
        asm volatile("bar.sync 2, 128;" ::: "memory");
      const int64_t a_lo = q.first + t0, a_hi = q.first + min(i1, t0 + g.toks) - 1;
      const bool all = t0 + g.toks <= i1 && (int64_t)j_hi <= a_lo && (a.r.window == 0u || (int64_t)j_lo > a_hi - (int64_t)a.r.window);
      bar_wait(b_s + 8 * w, (t / 2) & 1, &s_gave_up, a.err);
      tc_fence_after();
      const float4* z4 = (const float4*)s_lse[w][buf];
      if (all) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x[32];
          tc_ld32(ts + i * 32, x);
          tc_wait_ld(x);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float4 z = z4[i * 8 + k];
            const uint64_t y0 = fma_pair(pair_bits(x[4 * k], x[4 * k + 1]), scale2, pair(z.x, z.y));
            const uint64_t y1 = fma_pair(pair_bits(x[4 * k + 2], x[4 * k + 3]), scale2, pair(z.z, z.w));
            acc[(2 * k) & 3] = add_pair(acc[(2 * k) & 3], pair(ex2(pair_lo(y0)), ex2(pair_hi(y0))));
            acc[(2 * k + 1) & 3] = add_pair(acc[(2 * k + 1) & 3], pair(ex2(pair_lo(y1)), ex2(pair_hi(y1))));
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
          for (int k = 0; k < 32; ++k) {
            const int32_t tok = s_tok[w][buf][i * 32 + k];
            const float p = ex2(fmaf(__uint_as_float(x[k]), a.r.scale_log2, s_lse[w][buf][i * 32 + k]));
            acc[k & 3] = add_pair(acc[k & 3], pair(tok >= see_lo && tok < see_hi ? p : 0.f, 0.f));
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(b_free + 8 * w);
      if (has_given_up(&s_gave_up)) break;
    }
    const uint64_t tot = add_pair(add_pair(acc[0], acc[1]), add_pair(acc[2], acc[3]));
    sum = pair_lo(tot) + pair_hi(tot);
    if (w == 1) s_sum[row] = sum;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*(volatile uint32_t*)&s_gave_up) __nanosleep(1000000);   // copies and products in flight end by themselves
  if (warp == 8) {
    tc_fence_after();
    tmem_free(tm, WT_TMEM_COLS);
  }
  if (tid < WT_KEYS && j_lo + tid <= j_hi) {
    const float past = a.past && (int64_t)(j_lo + tid) < q.first ? a.decay * a.past[at] : 0.f;
    a.score[at] = past + (sum + s_sum[tid]);
  }
}

bool weigh_tiles_fits(const WeighArgs& a) {
  return page_box(a.c.page_size, WT_KEYS) >= MIN_BOX && a.r.group <= WT_ROWS;
}

template <typename T, int DP>
static void launch_tiles(const LaunchCfg& L, const WeighTileArgs& g) {
  launch_k(L, K_WEIGH_TILES, weigh_tiles_kernel<T, DP>, g.a.tiles * g.a.c.n_seqs * g.a.c.n_heads, WT_THREADS,
           WeighShape<DP>::SMEM, g);
}
bool launch_weigh_tiles(const LaunchCfg& L, const WeighArgs& a, int dtype, int sms) {
  WeighTileArgs g;
  g.a = a;
  g.toks = WT_ROWS / a.r.group;
  g.box = page_box(a.c.page_size, WT_KEYS);
  if (!rows_map(&g.q, a.r, a.c.head_dim, a.n_q_heads, dtype, g.toks) || !pool_map(&g.k, a.c, a.c.k, dtype, g.box))
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
    narrow ? launch_tiles<__nv_bfloat16, 64>(L, g) : launch_tiles<__nv_bfloat16, 128>(L, g);
  else
    narrow ? launch_tiles<__half, 64>(L, g) : launch_tiles<__half, 128>(L, g);
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
