// k_attend_few.cu — attention of at most 16 rows a sequence over a paged cache
// (ro_cache_attend): single tokens, or a few, times the heads of a group.
//
//   o_r = sum_j p_rj v_j,  p_rj = exp2(x_rj - m_r) / l_r,
//   x_rj = scale log2(e) q_r.k_j over the slots j that row r sees,
// with the running maximum m and sum l of a softmax in one pass over the slots.
//
// Bound by the bytes of K and V, so everything serves keeping loads in flight:
// a warp of loads keeps a ring of 16 KB stages full (a stage is 32 slots of
// 128 dimensions or 64 of 64, keys and values; by TMA a part of a page at a
// time, or row by row where the page size is no multiple of 4), and three warps
// take the stages in turn, each with an (m, l, o) of its own, so that no
// barrier joins them before the end.  A long sequence is cut into runs; the
// last CTA of a tile to finish joins them in the order of the slots, so the
// result does not depend on which CTA that is.
//
// Measured: 64 single tokens, 32 heads on 8 of 128, 2.98 GB of cache: 427 us,
// 7.0 TB/s (the copy rate measured on this GPU: 6.7).  With four warps of cp.async
// and CTA barriers instead: 749 us.
#include <algorithm>

#include "ro_tcgen05.cuh"

namespace ro {

constexpr int AF_WARPS = 3, AF_THREADS = 32 * (AF_WARPS + 1), AF_ROWS = 16;
// two CTAs on an SM
constexpr uint32_t AF_STAGES = 6, AF_STAGE = 16384;
// A place of the ring always belongs to the same warp.  (Loads land in any
// order: a warp that waited for a place's next phase while another warp's load
// there was still in flight would find the parity of the phase before it.)
static_assert(AF_STAGES % AF_WARPS == 0, "a place of the ring belongs to one warp");

template <int DP, uint32_t STAGE = AF_STAGE>
struct FewShape {
  static constexpr int KEYS = (int)STAGE / (4 * DP);    // slots of a stage
  static constexpr uint32_t BLOCKS = DP / 64, BLOCK_BYTES = KEYS * 128, SIDE = STAGE / 2;
  static constexpr uint32_t SMEM = 1024 + AF_STAGES * STAGE;
  static_assert(BLOCKS * BLOCK_BYTES == SIDE, "a stage holds its keys and values");
};

// A warp's share of a tile of rows: the queries as matrix fragments, and the
// (m, l, o) of the slots it has seen.
template <typename T, int DP, uint32_t STAGE = AF_STAGE>
struct FewRows {
  using S = FewShape<DP, STAGE>;
  static constexpr int KEYS = S::KEYS;
  uint32_t qf[DP / 16][4];
  int64_t row_a[2];
  float o[DP / 8][4];
  float m[2], l[2];

  __device__ __forceinline__ void clear() {
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
#pragma unroll
      for (int z = 0; z < 4; ++z) o[i][z] = 0.f;
  }
  // rows past the tile's are zero
  __device__ __forceinline__ void load(const AttendArgs& a, const SeqInfo& q, uint32_t kh, uint32_t rows, uint32_t lane) {
    const uint32_t G = a.r.group, D = a.c.head_dim;
    const T* qp[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t r = lane / 4 + 8 * z;
      qp[z] = nullptr;
      row_a[z] = INT64_MIN / 2;
      if (r < rows) {
        const uint32_t i = r / G, h = kh * G + r % G;
        qp[z] = (const T*)a.r.q + (q.tok0 + i) * a.r.q_tok + (uint64_t)h * a.r.q_head;
        row_a[z] = q.first + i;
      }
    }
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const uint32_t d = k * 16 + (z >> 1) * 8 + (lane & 3) * 2;
        const T* p = qp[z & 1];
        qf[k][z] = p && d < D ? *(const uint32_t*)(p + d) : 0u;
      }
  }
  // one stage: its keys at kb in shared memory, its values behind them
  __device__ __forceinline__ void stage(const AttendArgs& a, const SeqInfo& q, const SlotTile& st, uint32_t kb, uint32_t lane) {
    const uint32_t vb = kb + S::SIDE;
    const bool whole = st.lo == st.t0 && st.hi == st.t0 + KEYS;
    if (!whole) {   // values no row sees must not reach the product: a weight of 0 does not silence a NaN
      for (uint32_t r = lane; r < (uint32_t)KEYS; r += 32)
        if (st.t0 + r < st.lo || st.t0 + r >= st.hi)
#pragma unroll
          for (uint32_t x = 0; x < S::BLOCKS * 8; ++x)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vb + (x / 8) * S::BLOCK_BYTES + r * 128 +
                                                                      (x % 8) * 16),
                         "r"(0u)
                         : "memory");
      __syncwarp();
    }
    float s[KEYS / 8][4];
#pragma unroll
    for (int i = 0; i < KEYS / 8; ++i)
#pragma unroll
      for (int z = 0; z < 4; ++z) s[i][z] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int x = 0; x < KEYS / 16; ++x) {
        const uint32_t r = x * 16 + (lane & 7) + ((lane >> 4) << 3), c = k * 2 + ((lane >> 3) & 1);
        uint32_t b[4];
        ldsm4(b, kb + (c / 8) * S::BLOCK_BYTES + r * 128 + (((c & 7) ^ (r & 7)) * 16));
        mma16<T>(s[2 * x], qf[k], b[0], b[1]);
        mma16<T>(s[2 * x + 1], qf[k], b[2], b[3]);
      }
    const bool all = whole && (st.sink || ((int64_t)st.t0 + KEYS - 1 <= q.first &&
                                           (a.r.window == 0u || (int64_t)st.t0 > (q.first + q.n - 1) - (int64_t)a.r.window)));
    float nm[2] = {m[0], m[1]};
#pragma unroll
    for (int x = 0; x < KEYS / 8; ++x)
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        float y = s[x][z] * a.r.scale_log2;
        if (!all) {
          const uint32_t j = st.t0 + x * 8 + (lane & 3) * 2 + (z & 1);
          if (j < st.lo || j >= st.hi || !sees(a.r, row_a[z >> 1], j)) y = -INFINITY;
        }
        s[x][z] = y;
        nm[z >> 1] = fmaxf(nm[z >> 1], y);
      }
    float f[2], sub[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      nm[z] = fmaxf(nm[z], __shfl_xor_sync(0xffffffffu, nm[z], 1));
      nm[z] = fmaxf(nm[z], __shfl_xor_sync(0xffffffffu, nm[z], 2));
      const float top = nm[z] == -INFINITY ? 0.f : nm[z];   // a row that has seen nothing yet
      f[z] = ex2(m[z] - top);
      sub[z] = top - WEIGHT_UP<T>;
    }
    if (__any_sync(0xffffffffu, nm[0] > m[0] || nm[1] > m[1])) {
#pragma unroll
      for (int i = 0; i < DP / 8; ++i)
#pragma unroll
        for (int z = 0; z < 4; ++z) o[i][z] *= f[z >> 1];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        l[z] *= f[z];
        m[z] = nm[z];
      }
    }
    uint32_t p[KEYS / 16][4];
#pragma unroll
    for (int x = 0; x < KEYS / 8; ++x) {
      float e[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        e[z] = ex2(s[x][z] - sub[z >> 1]);
        l[z >> 1] += e[z];
      }
      // rounded to the cache's type for the product with V; l sums what is not rounded
      p[x / 2][(x & 1) * 2] = pack2<T>(e[0], e[1]);
      p[x / 2][(x & 1) * 2 + 1] = pack2<T>(e[2], e[3]);
    }
#pragma unroll
    for (int x = 0; x < KEYS / 16; ++x)
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        const uint32_t r = x * 16 + (lane & 15), c = d * 2 + (lane >> 4);
        uint32_t b[4];
        ldsm4_t(b, vb + (c / 8) * S::BLOCK_BYTES + r * 128 + (((c & 7) ^ (r & 7)) * 16));
        mma16<T>(o[2 * d], p[x], b[0], b[1]);
        mma16<T>(o[2 * d + 1], p[x], b[2], b[3]);
      }
    if (!whole) fence_async_smem();   // (this warp's zeros lie in a stage that TMA writes next)
  }
  __device__ __forceinline__ void sum_rows() {
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      l[z] += __shfl_xor_sync(0xffffffffu, l[z], 1);
      l[z] += __shfl_xor_sync(0xffffffffu, l[z], 2);
    }
  }
};

template <typename T, int DP>
__global__ void __launch_bounds__(AF_THREADS, 2) attend_few_kernel(const __grid_constant__ AttendFewArgs g) {
  using S = FewShape<DP>;
  constexpr int KEYS = S::KEYS;
  const AttendArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[2 * AF_STAGES];
  __shared__ float s_m[AF_WARPS][AF_ROWS], s_l[AF_WARPS][AF_ROWS];
  __shared__ uint32_t s_last, s_gave_up;
  wait_predecessor();
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t G = a.r.group, D = a.c.head_dim;
  const uint32_t seq = blockIdx.x / a.c.n_heads, kh = blockIdx.x - seq * a.c.n_heads;
  const SeqInfo q = seq_info(a.c, a.r, seq, a.err);
  if (q.n == 0) return;
  const uint32_t rows = q.n * G;
  const KeySpan ks = key_span(q, a.r, 0, q.n);
  const SlotTiles<KEYS> slots(ks, g.box);
  const uint32_t per = max(a.chunk, slots.n / a.max_chunks + 1);   // stages of a run
  const uint32_t n_chunks = max(1u, (slots.n + per - 1) / per);
  if (blockIdx.y >= n_chunks) return;
  const uint32_t c0 = blockIdx.y * per, n = min(per, slots.n - min(slots.n, c0));

  const uint32_t sm = (step_smem(smem_raw) + 1023u) & ~1023u;
  const uint32_t b_full = step_smem(s_bar), b_empty = b_full + 8 * AF_STAGES;
  if (tid == 0) {
    s_gave_up = 0;
    for (uint32_t i = 0; i < AF_STAGES; ++i) {
      bar_init(b_full + 8 * i, g.tma ? 1 : 32);
      bar_init(b_empty + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  __syncthreads();

  if (warp == AF_WARPS) {
    load_stages<T, DP, KEYS, true>(a.c, &g.k, &g.v, g.tma != 0, g.box, AF_STAGES, slots, c0, n, kh, q.page0, sm, b_full,
                                              b_empty, &s_gave_up, a.err);
  }

  FewRows<T, DP> f;
  f.clear();
  if (warp < AF_WARPS) {
    f.load(a, q, kh, rows, lane);
    for (uint32_t t = warp; t < n; t += AF_WARPS) {
      const uint32_t slot = t % AF_STAGES;
      const SlotTile st = slots.at(c0 + t);
      bar_wait(b_full + 8 * slot, (t / AF_STAGES) & 1, &s_gave_up, a.err);
      f.stage(a, q, st, sm + slot * AF_STAGE, lane);
      __syncwarp();
      if (lane == 0) bar_arrive(b_empty + 8 * slot);
    }
    f.sum_rows();
  }
  __syncthreads();
  if (*(volatile uint32_t*)&s_gave_up) __nanosleep(1000000);   // copies in flight end by themselves
  // the warps join their results: o in shared memory, [warp][16][DP]
  float* so = (float*)(smem_raw + (sm - step_smem(smem_raw)));
  if (warp < AF_WARPS) {
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int r = lane / 4 + 8 * z;
      if ((lane & 3) == 0) {
        s_m[warp][r] = f.m[z];
        s_l[warp][r] = f.l[z];
      }
#pragma unroll
      for (int i = 0; i < DP / 8; ++i)
        *(float2*)(so + (warp * AF_ROWS + r) * DP + i * 8 + (lane & 3) * 2) = make_float2(f.o[i][z * 2], f.o[i][z * 2 + 1]);
    }
  }
  __syncthreads();
  const uint64_t run = (uint64_t)blockIdx.x * a.max_chunks + blockIdx.y;
  float* part = a.partial + run * AF_ROWS * DP;
  float2* ml = (float2*)(a.partial + (uint64_t)gridDim.x * a.max_chunks * AF_ROWS * DP) + run * AF_ROWS;
  T* out = (T*)a.out;
  float* joined = so + AF_WARPS * AF_ROWS * DP;   // cluster: this run's result, [16][DP], then (m, l) by row
  for (uint32_t x = tid; x < rows * (DP / 4); x += AF_THREADS) {
    const uint32_t r = x / (DP / 4), d = (x % (DP / 4)) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < AF_WARPS; ++k) M = fmaxf(M, s_m[k][r]);
    const float sub = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < AF_WARPS; ++k) {
      const float f = ex2(s_m[k][r] - sub);
      L += f * s_l[k][r];
      const float4 v = *(const float4*)(so + (k * AF_ROWS + r) * DP + d);
      acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
    }
    if (n_chunks > 1 && g.cluster) {
      *(float4*)(joined + r * DP + d) = acc;
      if (d == 0) *(float2*)(joined + AF_ROWS * DP + 2 * r) = make_float2(M, L);
    } else if (n_chunks > 1) {
      __stcg((float4*)(part + r * DP + d), acc);
      if (d == 0) __stcg(ml + r, make_float2(M, L));
    } else {
      const uint64_t t = q.tok0 + r / G;
      const uint32_t h = kh * G + r % G;
      const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
      if (d < D)
        *(uint2*)(out + t * a.out_tok + h * a.out_head + d) =
            make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
      if (d == 0 && a.lse) a.lse[t * a.n_q_heads + h] = row_lse<T>(M, L);
    }
  }
  if (n_chunks == 1) return;
  uint32_t first = tid, step = AF_THREADS;        // the pieces of the join that are this thread's
  if (g.cluster) {
    cluster_sync();
    first += blockIdx.y * AF_THREADS;
    step *= n_chunks;
  } else {
    __threadfence();
    __syncthreads();
    if (tid == 0) s_last = ticket(a.counter + blockIdx.x) == n_chunks - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    part = a.partial + (uint64_t)blockIdx.x * a.max_chunks * AF_ROWS * DP;
    ml = (float2*)(a.partial + (uint64_t)gridDim.x * a.max_chunks * AF_ROWS * DP) +
         (uint64_t)blockIdx.x * a.max_chunks * AF_ROWS;
  }
  // the runs in order; their maxima and sums are few enough to read again for every piece
  const uint32_t js = step_smem(joined);
  for (uint32_t x = first; x < rows * (DP / 4); x += step) {
    const uint32_t r = x / (DP / 4), d = (x % (DP / 4)) * 4;
    float M = -INFINITY, L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (uint32_t k = 0; k < n_chunks; ++k) {
      float2 z;
      float4 v;
      if (g.cluster) {
        z = cluster_load2(js + (AF_ROWS * DP + 2 * r) * 4, k);
        v = cluster_load4(js + (r * DP + d) * 4, k);
      } else {
        z = __ldcg(ml + k * AF_ROWS + r);
        v = __ldcg((const float4*)(part + ((uint64_t)k * AF_ROWS + r) * DP + d));
      }
      const float nm = fmaxf(M, z.x), sub = nm == -INFINITY ? 0.f : nm;
      const float f = ex2(M - sub), e = ex2(z.x - sub);
      M = nm;
      L = L * f + z.y * e;
      acc.x = acc.x * f + v.x * e;
      acc.y = acc.y * f + v.y * e;
      acc.z = acc.z * f + v.z * e;
      acc.w = acc.w * f + v.w * e;
    }
    const uint64_t t = q.tok0 + r / G;
    const uint32_t h = kh * G + r % G;
    const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
    if (d < D)
      *(uint2*)(out + t * a.out_tok + h * a.out_head + d) =
          make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
    if (d == 0 && a.lse) a.lse[t * a.n_q_heads + h] = row_lse<T>(M, L);
  }
  if (g.cluster)
    cluster_sync();                               // no CTA leaves while another reads its shared memory
  else if (tid == 0)
    a.counter[blockIdx.x] = 0u;                   // for the next call
}

// The same for many short sequences: a warp, alone in its CTA, for each sequence
// and head, with a ring of its own of 8 KB stages (16 slots of 128 dimensions or
// 32 of 64) that it loads itself: a place again as soon as it is done with it.
// Nothing is joined.  A CTA of four warps takes about 6 us for a sequence of any
// few stages, most of it waiting for one thing after another; of these nine
// share an SM, and while some start or end the others' loads are in flight.
//
// Measured (32 heads on 8 of 128): 256 single tokens over 40 slots 13 us (41 with
// CTAs of four warps), over 300 slots 55 us (79; its bytes at the copy rate: 48);
// 1,000 over up to 200 slots 63 us (159).  Two stages: 14, 65, 57; four: 17, 69, 73.
constexpr uint32_t AS_STAGES = 3, AS_STAGE = 8192;
template <typename T, int DP>
__global__ void __launch_bounds__(32) attend_short_kernel(const __grid_constant__ AttendFewArgs g) {
  using S = FewShape<DP, AS_STAGE>;
  constexpr int KEYS = S::KEYS;
  const AttendArgs& a = g.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[AS_STAGES];
  __shared__ uint32_t s_gave_up;
  const uint32_t lane = threadIdx.x, sm = (step_smem(smem_raw) + 1023u) & ~1023u, b_full = step_smem(s_bar);
  if (lane == 0) {
    s_gave_up = 0;
    for (uint32_t i = 0; i < AS_STAGES; ++i) bar_init(b_full + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  __syncwarp();
  wait_predecessor();
  const uint32_t G = a.r.group, D = a.c.head_dim;
  const uint32_t seq = blockIdx.x / a.c.n_heads, kh = blockIdx.x - seq * a.c.n_heads;
  const SeqInfo q = seq_info(a.c, a.r, seq, a.err);
  if (q.n == 0) return;
  const uint32_t rows = q.n * G;
  const SlotTiles<KEYS> slots(key_span(q, a.r, 0, q.n), g.box);
  const uint32_t n = slots.n;
  const uint32_t boxes = KEYS / g.box, ahead = 32 / boxes;   // boxes of a stage, a lane each; stages whose pages the lanes hold
  auto has_box = [&](const SlotTile& st, uint32_t j) { return j < st.hi && j + g.box > st.lo; };
  auto page_of = [&](uint32_t t) -> uint32_t {
    const uint32_t u = t + lane / boxes;
    if (u >= n) return 0u;
    const SlotTile st = slots.at(u);
    const uint32_t j = st.t0 + (lane % boxes) * g.box;
    return has_box(st, j) ? a.c.pages[q.page0 + page_index(a.c, j)] : 0u;
  };
  uint32_t page = 0, next = page_of(0);
  auto issue = [&](uint32_t t) {
    if (t % ahead == 0) {
      page = next;
      next = page_of(t + ahead);
    }
    const SlotTile st = slots.at(t);
    const uint32_t b = lane % boxes, j = st.t0 + b * g.box;
    bool load = lane / boxes == t % ahead && has_box(st, j);
    if (load && page >= a.c.n_pages) {
      record(a.err, ERR_INVAL);
      load = false;
    }
    const uint32_t loaded = __popc(__ballot_sync(0xffffffffu, load));
    const uint32_t full = b_full + 8 * (t % AS_STAGES), dst = sm + (t % AS_STAGES) * AS_STAGE + b * g.box * 128;
    if (lane == 0) bar_expect(full, 2 * loaded * S::BLOCKS * g.box * 128);
    __syncwarp();
    if (load) {
      const int y = (int)(j - page_index(a.c, j) * a.c.page_size);
#pragma unroll
      for (uint32_t x = 0; x < S::BLOCKS; ++x) {
        tma4(dst + x * S::BLOCK_BYTES, &g.k, x * 64, y, (int)kh, (int)page, full);
        tma4(dst + S::SIDE + x * S::BLOCK_BYTES, &g.v, x * 64, y, (int)kh, (int)page, full);
      }
    }
  };
  for (uint32_t t = 0; t < min(n, AS_STAGES); ++t) issue(t);
  FewRows<T, DP, AS_STAGE> f;
  f.clear();
  f.load(a, q, kh, rows, lane);
  for (uint32_t t = 0; t < n; ++t) {
    bar_wait(b_full + 8 * (t % AS_STAGES), (t / AS_STAGES) & 1, &s_gave_up, a.err);
    if (has_given_up(&s_gave_up)) break;
    f.stage(a, q, slots.at(t), sm + (t % AS_STAGES) * AS_STAGE, lane);
    __syncwarp();
    if (t + AS_STAGES < n) issue(t + AS_STAGES);
  }
  if (*(volatile uint32_t*)&s_gave_up) __nanosleep(1000000);   // copies in flight end by themselves
  f.sum_rows();
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const uint32_t r = lane / 4 + 8 * z;
    if (r >= rows) continue;
    const uint64_t t = q.tok0 + r / G;
    const uint32_t h = kh * G + r % G;
    const float inv = f.l[z] > 0.f || f.l[z] != f.l[z] ? 1.f / f.l[z] : 0.f;
    T* out = (T*)a.out + t * a.out_tok + (uint64_t)h * a.out_head + (lane & 3) * 2;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
      if ((uint32_t)i * 8 + (lane & 3) * 2 < D) *(uint32_t*)(out + i * 8) = pack2<T>(f.o[i][z * 2] * inv, f.o[i][z * 2 + 1] * inv);
    if ((lane & 3) == 0 && a.lse) a.lse[t * a.n_q_heads + h] = row_lse<T>(f.m[z], f.l[z]);
  }
}

uint32_t attend_few_keys(uint32_t head_dim) { return head_dim <= 64 ? FewShape<64>::KEYS : FewShape<128>::KEYS; }
uint32_t attend_short_keys(uint32_t head_dim) {
  return head_dim <= 64 ? FewShape<64, AS_STAGE>::KEYS : FewShape<128, AS_STAGE>::KEYS;
}
size_t attend_few_partial(const AttendArgs& a) {
  const size_t dp = a.c.head_dim <= 64 ? 64 : 128;
  return (size_t)a.tiles * a.c.n_heads * a.max_chunks * AF_ROWS * (dp + 2) * sizeof(float);
}

template <typename T, int DP>
static void launch_few(const LaunchCfg& L, const AttendFewArgs& g, bool alone) {
  if (alone) {
    launch_k(L, K_ATTEND_ROWS, attend_short_kernel<T, DP>, g.a.tiles * g.a.c.n_heads, 32, 1024 + AS_STAGES * AS_STAGE, g);
    return;
  }
  launch_k(L, K_ATTEND_ROWS, attend_few_kernel<T, DP>, dim3(g.a.tiles * g.a.c.n_heads, g.a.max_chunks), AF_THREADS,
           FewShape<DP>::SMEM, g, dim3(1, g.cluster ? g.a.max_chunks : 1));
}
void launch_attend_few(const LaunchCfg& L, const AttendArgs& a, int dtype, bool cluster, bool alone) {
  AttendFewArgs g;
  g.a = a;
  g.cluster = cluster;
  g.box = page_box(a.c.page_size, alone ? attend_short_keys(a.c.head_dim) : attend_few_keys(a.c.head_dim));
  g.tma = g.box >= MIN_BOX && pool_map(&g.k, a.c, a.c.k, dtype, g.box) && pool_map(&g.v, a.c, a.c.v, dtype, g.box);
  if (!g.tma) g.box = 1;
  alone = alone && g.tma;
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == RO_BF16)
    narrow ? launch_few<__nv_bfloat16, 64>(L, g, alone) : launch_few<__nv_bfloat16, 128>(L, g, alone);
  else
    narrow ? launch_few<__half, 64>(L, g, alone) : launch_few<__half, 128>(L, g, alone);
}

template <typename T, int DP>
static cudaError_t allow() {
  const cudaError_t e = cudaFuncSetAttribute(attend_short_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(1024 + AS_STAGES * AS_STAGE));
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(attend_few_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)FewShape<DP>::SMEM);
}
cudaError_t prepare_attend_few_kernels() {
  for (cudaError_t e : {allow<__nv_bfloat16, 64>(), allow<__nv_bfloat16, 128>(), allow<__half, 64>(), allow<__half, 128>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
