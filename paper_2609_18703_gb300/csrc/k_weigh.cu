// k_weigh.cu — the attention weight cached tokens gathered (ro_cache_weigh),
// where pages or groups fit no tensor tile.
//
//   score_j = decay past_j + sum_r exp2(x_rj - lse_r log2(e)) over the rows r
//   that see slot j; x_rj = scale log2(e) q_r.k_j.
//
// A CTA takes 64 slots of one cache head of one sequence and runs over the
// query rows that can see one of them: keys are the rows of the matrix
// product and stay in registers, query rows its columns, so a key's sum stays
// in the four lanes that hold its row and is added in a fixed order.  Bound by
// mma.sync and the exponentials between its products.
#include <algorithm>

#include "ro_step.cuh"

namespace ro {

template <typename T, int DP>
__global__ void __launch_bounds__(WG_THREADS) weigh_kernel(const __grid_constant__ WeighArgs a) {
  constexpr int CH = DP / 8, RPP = WG_THREADS / CH;
  __shared__ __align__(128) uint8_t s_tile[WG_ROWS * DP * 2];   // keys, then query rows
  __shared__ float s_lse[WG_ROWS];
  __shared__ uint32_t s_at[WG_ROWS];                            // token within the chunk
  wait_predecessor();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // a sequence's heads and then its key tiles are neighbours: its query rows stay in L2
  const uint32_t kh = blockIdx.x % a.c.n_heads, rest = blockIdx.x / a.c.n_heads;
  const uint32_t seq = rest / a.tiles, tile = rest - seq * a.tiles;
  const SeqInfo q = seq_info(a.c, a.r, seq, a.err);
  const uint64_t j0 = (uint64_t)tile * WG_KEYS;
  uint32_t len = q.len;
  if (len > a.score_cap) {
    if (tile == 0 && tid == 0) record(a.err, ERR_CAPACITY);
    len = (uint32_t)a.score_cap;
  }
  if (j0 >= len) return;
  const uint32_t jn = min((uint32_t)WG_KEYS, len - (uint32_t)j0), j_lo = (uint32_t)j0, j_hi = j_lo + jn - 1;
  uint32_t i0, i1;
  seeing_tokens(q, a.r, j_lo, j_hi, &i0, &i1);
  const uint32_t G = a.r.group, D = a.c.head_dim;
  const uint32_t rows = (i1 - i0) * G;
  const uint32_t sm = step_smem(s_tile);
  const uint32_t pc = tid % CH, pr = tid / CH;
  const bool piece_ok = pc * 8 < D;
  float sum[2] = {0.f, 0.f};
  const uint32_t my_key[2] = {j_lo + warp * 16 + lane / 4, j_lo + warp * 16 + lane / 4 + 8};
  if (rows > 0) {
    uint32_t kf[DP / 16][4];
#pragma unroll
    for (int i = 0; i < (int)WG_KEYS / RPP; ++i) {
      const uint32_t r = i * RPP + pr, j = j_lo + r;
      bool ok = r < jn && piece_ok;
      uint64_t e = 0;
      if (ok) {
        uint32_t pi, slot;
        split_slot(a.c, j, &pi, &slot);
        const uint32_t page = a.c.pages[q.page0 + pi];
        if (page < a.c.n_pages) {
          e = page * a.c.page_stride + kh * a.c.head_stride + slot * a.c.slot_stride + pc * 8;
        } else {
          record(a.err, ERR_INVAL);
          ok = false;
        }
      }
      cp_async16_or_zero(sm + r * DP * 2 + ((pc ^ (r & 7)) * 16), (const T*)a.c.k + e, ok);
    }
    cp_async_commit();
    cp_async_wait<0>();
    __syncthreads();
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      const uint32_t r = warp * 16 + (lane & 15), c = k * 2 + (lane >> 4);
      ldsm4(kf[k], sm + r * DP * 2 + ((c ^ (r & 7)) * 16));
    }
    for (uint32_t r0 = 0; r0 < rows; r0 += WG_ROWS) {
      const uint32_t rn = min(WG_ROWS, rows - r0);
      __syncthreads();   // the tile's last readers
#pragma unroll
      for (int i = 0; i < (int)WG_ROWS / RPP; ++i) {
        const uint32_t r = i * RPP + pr;
        const uint32_t x = r0 + min(r, rn - 1), t = i0 + x / G, g = x % G;
        const uint64_t e = piece_ok ? (q.tok0 + t) * a.r.q_tok + (uint64_t)(kh * G + g) * a.r.q_head + pc * 8 : 0;
        cp_async16_or_zero(sm + r * DP * 2 + ((pc ^ (r & 7)) * 16), (const T*)a.r.q + e, piece_ok);
      }
      cp_async_commit();
      if (tid < (int)WG_ROWS) {
        const uint32_t x = r0 + min((uint32_t)tid, rn - 1), t = i0 + x / G, g = x % G;
        float z = LSE_FILL;
        if (tid < (int)rn) {
          z = a.lse[(q.tok0 + t) * a.n_q_heads + kh * G + g] * 1.44269504088896340736f;
          if (z == -INFINITY) z = INFINITY;   // rows that see nothing add 0
        }
        s_lse[tid] = z;
        s_at[tid] = t;
      }
      cp_async_wait<0>();
      __syncthreads();
      // every row of this tile sees every slot of the CTA?
      const int64_t a_lo = q.first + i0 + r0 / G, a_hi = q.first + i0 + (r0 + rn - 1) / G;
      const bool all = (int64_t)j_hi <= a_lo && (a.r.window == 0u || (int64_t)j_lo > a_hi - (int64_t)a.r.window);
      for (uint32_t n0 = 0; n0 < rn; n0 += 16) {
        float s[2][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          const uint32_t r = n0 + (lane & 7) + ((lane >> 4) << 3), c = k * 2 + ((lane >> 3) & 1);
          uint32_t b[4];
          ldsm4(b, sm + r * DP * 2 + ((c ^ (r & 7)) * 16));
          mma16<T>(s[0], kf[k], b[0], b[1]);
          mma16<T>(s[1], kf[k], b[2], b[3]);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint32_t c = n0 + n * 8 + (lane & 3) * 2 + (z & 1);
            float p = exp2f(s[n][z] * a.r.scale_log2 - s_lse[c]);
            if (!all && !sees(a.r, q.first + s_at[c], my_key[z >> 1])) p = 0.f;
            sum[z >> 1] += p;
          }
      }
    }
  }
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 1);
    sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 2);
    if ((lane & 3) == 0 && my_key[z] <= j_hi) {
      const uint64_t e = ((uint64_t)seq * a.c.n_heads + kh) * a.score_cap + my_key[z];
      const float past = a.past && (int64_t)my_key[z] < q.first ? a.decay * a.past[e] : 0.f;
      a.score[e] = past + sum[z];
    }
  }
}

template <typename T>
static void launch_dim(const LaunchCfg& L, const WeighArgs& a) {
  const unsigned grid = a.tiles * a.c.n_seqs * a.c.n_heads;
  if (a.c.head_dim <= 64)
    launch_k(L, K_WEIGH, weigh_kernel<T, 64>, grid, WG_THREADS, 0, a);
  else
    launch_k(L, K_WEIGH, weigh_kernel<T, 128>, grid, WG_THREADS, 0, a);
}
void launch_weigh(const LaunchCfg& L, const WeighArgs& a, int dtype) {
  if (dtype == RO_BF16)
    launch_dim<__nv_bfloat16>(L, a);
  else
    launch_dim<__half>(L, a);
}

}  // namespace ro
