// k_weigh_few.cu — the attention weight cached tokens gathered
// (ro_cache_weigh) from at most 16 rows a sequence.
//
//   score_j = decay past_j + sum_r exp2(scale log2(e) q_r.k_j - lse_r log2(e))
//
// Bound by the bytes of K.  As for the attention of few rows a warp of loads
// keeps a ring of 16 KB stages of keys full and three warps take them in turn;
// keys are the rows of the matrix product, query rows its columns, so a key's
// sum stays in the four lanes that hold its row and is added in a fixed order.
// Stages that no row sees (behind the sinks, before a window) pass the ring by:
// their past scores are decayed in one sweep (37 single tokens of up to 23,302
// slots, 8 heads, window 3: 14 us; stage by stage 48).
//
// Measured: 32 single tokens, 336 MB of keys and scores: 56 us, 6.0 TB/s; a CTA
// for every 64 slots, without a ring: 143 us.
#include <algorithm>

#include "ro_tcgen05.cuh"

namespace ro {

constexpr int WF_WARPS = 3, WF_THREADS = 32 * (WF_WARPS + 1);
// A place for each warp and four CTAs on an SM: as many loads in flight as two
// CTAs with twice the ring, but more starts and ends beside them (1,000 single
// tokens over up to 200 slots: 59 us against 103; 128 over 1,000 slots 47 against
// 54; one of 100,000 slots 38 against 37).
constexpr uint32_t WF_STAGES = 3, WF_STAGE = 16384;
static_assert(WF_STAGES == WF_WARPS, "a place of the ring belongs to one warp, and each has one");
constexpr uint32_t WF_SMEM = 1024 + WF_STAGES * WF_STAGE;
template <int DP>
constexpr int wf_keys() {
  return (int)WF_STAGE / (DP * 2);
}

// The tiles of a run without those that no row sees.
template <int KEYS>
struct SeenSlots {
  SlotTiles<KEYS> all;
  uint32_t gap, skip;        // tiles before the gap, tiles in it
  __device__ __forceinline__ SlotTile at(uint32_t t) const { return all.at(t < gap ? t : t + skip); }
};

template <typename T, int DP>
__global__ void __launch_bounds__(WF_THREADS, 4) weigh_few_kernel(const __grid_constant__ WeighFewArgs g) {
  constexpr int KEYS = wf_keys<DP>();
  constexpr uint32_t BLOCK_BYTES = KEYS * 128;
  const WeighArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[2 * WF_STAGES];
  __shared__ float s_sum[WF_WARPS][KEYS];
  __shared__ uint32_t s_gave_up;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t G = a.r.group, D = a.c.head_dim;
  const uint32_t seq = blockIdx.x / a.c.n_heads, kh = blockIdx.x - seq * a.c.n_heads;
  const SeqInfo q = seq_info(a.c, a.r, seq, a.err);
  uint32_t len = q.len;
  if (len > a.score_cap) {
    if (blockIdx.y == 0 && tid == 0) record(a.err, ERR_CAPACITY);
    len = (uint32_t)a.score_cap;
  }
  const KeySpan every = {0u, 0u, len};
  const SlotTiles<KEYS> every_slot(every, g.box);
  const uint32_t per = max(a.chunk, (every_slot.n + a.tiles - 1) / a.tiles);
  const uint32_t c0 = blockIdx.y * per;
  if (c0 >= every_slot.n) return;
  const uint32_t c1 = min(c0 + per, every_slot.n);
  const uint32_t rows = q.n * G;
  const int64_t a_max = q.first + q.n - 1;
  const RowsArgs& r = a.r;
  uint32_t gap0 = c0, gap1 = c0;                      // the run's tiles that no row sees
  if (rows == 0) {
    gap1 = c1;
  } else if (r.window != 0u) {
    const int64_t from = q.first - (int64_t)r.window;   // slots above it lie in the first row's window
    gap0 = min(max(c0, r.sinks / KEYS + (r.sinks % KEYS != 0u ? 1u : 0u)), c1);
    gap1 = max(gap0, (uint32_t)min((int64_t)c1, from < 0 ? (int64_t)0 : (from + 1) / KEYS));
  }
  const uint32_t n = c1 - c0 - (gap1 - gap0);
  const SeenSlots<KEYS> slots = {every_slot, gap0, gap1 - gap0};

  const uint32_t sm = (step_smem(smem_raw) + 1023u) & ~1023u;
  const uint32_t b_full = step_smem(s_bar), b_empty = b_full + 8 * WF_STAGES;
  if (tid == 0) {
    s_gave_up = 0;
    for (uint32_t i = 0; i < WF_STAGES; ++i) {
      bar_init(b_full + 8 * i, g.tma ? 1 : 32);
      bar_init(b_empty + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  __syncthreads();
  if (warp == WF_WARPS) {
    load_stages<T, DP, KEYS, false>(a.c, &g.k, &g.k, g.tma != 0, g.box, WF_STAGES, slots, c0, n, kh, q.page0, sm, b_full,
                                               b_empty, &s_gave_up, a.err);
  } else {
    // query rows as the right operand, two groups of eight; each row's lse, +inf for rows that see nothing
    uint32_t qf[DP / 16][4];
    float lse[4];
    int64_t at[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const uint32_t x = (z >> 1) * 8 + (lane & 3) * 2 + (z & 1);
      lse[z] = LSE_FILL;
      at[z] = INT64_MIN / 2;
      if (x < rows) {
        const uint32_t i = x / G;
        at[z] = q.first + i;
        lse[z] = a.lse[(q.tok0 + i) * a.n_q_heads + kh * G + x % G] * 1.44269504088896340736f;
        if (lse[z] == -INFINITY) lse[z] = INFINITY;
      }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t x = min(z * 8 + lane / 4, rows - 1);
      const T* p = rows > 0 ? (const T*)r.q + (q.tok0 + x / G) * r.q_tok + (uint64_t)(kh * G + x % G) * r.q_head : nullptr;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t d = k * 16 + h * 8 + (lane & 3) * 2;
          qf[k][z * 2 + h] = p && d < D ? *(const uint32_t*)(p + d) : 0u;
        }
    }
    const uint64_t row = ((uint64_t)seq * a.c.n_heads + kh) * a.score_cap;
    if (gap1 > gap0)
      decay_past<32 * WF_WARPS>(a, row, gap0 * KEYS, min(gap1 * KEYS, len), tid);   // (no new slot among them)
    for (uint32_t t = warp; t < n; t += WF_WARPS) {
      const uint32_t round = t / WF_WARPS, slot = warp;
      const SlotTile st = slots.at(c0 + t);
      float past[KEYS / 32];   // under way while the keys arrive
#pragma unroll
      for (int i = 0; i < KEYS / 32; ++i) {
        const uint32_t j = st.t0 + i * 32 + lane;
        past[i] = a.past && j < st.hi && (int64_t)j < q.first ? a.past[row + j] : 0.f;
      }
      bar_wait(b_full + 8 * slot, round & 1, &s_gave_up, a.err);
      {
        const bool all = (int64_t)st.t0 + KEYS - 1 <= q.first && (r.window == 0u || (int64_t)st.t0 > a_max - (int64_t)r.window);
#pragma unroll
        for (int y = 0; y < KEYS / 16; ++y) {
          float s[2][4] = {};
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const uint32_t rr = y * 16 + (lane & 15), c = k * 2 + (lane >> 4);
            uint32_t kf[4];
            ldsm4(kf, sm + slot * WF_STAGE + (c / 8) * BLOCK_BYTES + rr * 128 + (((c & 7) ^ (rr & 7)) * 16));
            mma16<T>(s[0], kf, qf[k][0], qf[k][1]);
            if (rows > 8) mma16<T>(s[1], kf, qf[k][2], qf[k][3]);
          }
          float sum[2] = {0.f, 0.f};
#pragma unroll
          for (int z = 0; z < 2; ++z)        // key lane / 4 + 8 z
#pragma unroll
            for (int x = 0; x < 4; ++x) {    // row (x / 2) * 8 + ..
              float p = ex2(s[x >> 1][z * 2 + (x & 1)] * r.scale_log2 - lse[x]);
              if (!all && !sees(r, at[x], st.t0 + y * 16 + lane / 4 + 8 * z)) p = 0.f;
              sum[z] += p;
            }
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 1);
            sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 2);
            if ((lane & 3) == 0) s_sum[warp][y * 16 + lane / 4 + 8 * z] = sum[z];
          }
        }
      }
      __syncwarp();
      if (lane == 0) bar_arrive(b_empty + 8 * slot);
#pragma unroll
      for (int i = 0; i < KEYS / 32; ++i) {
        const uint32_t j = st.t0 + i * 32 + lane;
        if (j < st.hi) a.score[row + j] = a.decay * past[i] + s_sum[warp][i * 32 + lane];
      }
      __syncwarp();
    }
  }
  __syncwarp();
  if (s_gave_up) __nanosleep(1000000);   // copies in flight end by themselves
}

uint32_t weigh_few_keys(uint32_t head_dim) { return head_dim <= 64 ? wf_keys<64>() : wf_keys<128>(); }

template <typename T, int DP>
static void launch_few(const LaunchCfg& L, const WeighFewArgs& g) {
  launch_k(L, K_WEIGH, weigh_few_kernel<T, DP>, dim3(g.a.c.n_seqs * g.a.c.n_heads, g.a.tiles), WF_THREADS,
           WF_SMEM, g);
}
void launch_weigh_few(const LaunchCfg& L, const WeighArgs& a, int dtype) {
  WeighFewArgs g;
  g.a = a;
  g.box = page_box(a.c.page_size, weigh_few_keys(a.c.head_dim));
  g.tma = g.box >= MIN_BOX && pool_map(&g.k, a.c, a.c.k, dtype, g.box);
  if (!g.tma) g.box = 1;
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == RO_BF16)
    narrow ? launch_few<__nv_bfloat16, 64>(L, g) : launch_few<__nv_bfloat16, 128>(L, g);
  else
    narrow ? launch_few<__half, 64>(L, g) : launch_few<__half, 128>(L, g);
}

template <typename T, int DP>
static cudaError_t allow() {
  return cudaFuncSetAttribute(weigh_few_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)WF_SMEM);
}
cudaError_t prepare_weigh_few_kernels() {
  for (cudaError_t e : {allow<__nv_bfloat16, 64>(), allow<__nv_bfloat16, 128>(), allow<__half, 64>(), allow<__half, 128>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
