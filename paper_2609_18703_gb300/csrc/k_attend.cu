// k_attend.cu — attention over a paged cache whose pages or groups fit no tensor
// tile (ro_cache_attend): any page size, any number of heads in a group.
//
//   o_r = sum_j p_rj v_j,  p_rj = exp2(x_rj - m_r) / l_r,
//   x_rj = scale log2(e) q_r.k_j over the slots j that row r sees,
// with the running maximum m and sum l of a softmax in one pass over the keys.
// The rows of a tile are the tokens of one sequence times the query heads that
// share a cache head, so a key is read once for all of them.
//
// A CTA of four warps takes 64 rows (a token's heads, tokens of one sequence)
// and a run of keys, staged by cp.async three deep with pages looked up a
// stage ahead; each warp has 16 rows.  A long sequence is cut into runs of
// `chunk` keys; the last CTA of a tile to finish joins the runs' (m, l, o) in
// the order of the keys, so the result does not depend on which CTA that is.
// mma.sync bounds it, at about an eighth of what the tensor-core tiles reach
// (chunks of 2,048 tokens over up to 16,384 slots: 205 TFLOP/s against 1,550);
// it also takes scales of 0 or less, whose softmax has its maximum elsewhere.
// Biased (ro_cache_attend_biased): scores are capped, fall with distance and are
// masked row by row before the maximum; slots nobody sees are loaded as zeros.
#include <algorithm>

#include "ro_step.cuh"

namespace ro {

constexpr int AR_THREADS = 128, AR_STAGES = 3, AR_KEYS = 64, AR_ROWS = 64;

template <int DP>
constexpr size_t attend_rows_smem() {
  return (size_t)AR_STAGES * 2 * AR_KEYS * DP * 2;
}

template <typename T, int DP, bool BIASED>
__global__ void __launch_bounds__(AR_THREADS) attend_rows_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int KW = AR_KEYS, ROWS = AR_ROWS;
  constexpr int CH = DP / 8;                         // 16-byte pieces of a row
  constexpr int RPP = AR_THREADS / CH, PASSES = AR_KEYS / RPP;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t s_seq, s_part, s_found, s_last;
  wait_predecessor();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t G = a.r.group, D = a.c.head_dim;
  const uint32_t tile = blockIdx.x / a.c.n_heads, kh = blockIdx.x - tile * a.c.n_heads;
  const uint32_t toks = max(1u, ROWS / G), row_tiles = (G + ROWS - 1) / ROWS;   // more heads than rows: several tiles a token
  if (warp == 0) {
    uint32_t s = 0, p = 0;
    const bool f = find_tile(a.r, a.c.n_seqs, tile / row_tiles, toks, &s, &p, a.err);
    if (lane == 0) {
      s_seq = s;
      s_part = p;
      s_found = f;
    }
  }
  __syncthreads();
  if (!s_found) return;
  const SeqInfo q = seq_info(a.c, a.r, s_seq, a.err);
  const uint32_t g0 = (tile % row_tiles) * ROWS;          // first head of the group in this tile
  const uint32_t gn = min(G - g0, (uint32_t)ROWS);         // heads of the group in this tile
  const uint32_t i0 = s_part * toks, i1 = min(q.n, i0 + toks);
  if (i0 >= i1) return;
  const uint32_t rows = (i1 - i0) * gn;
  const auto ks = [&] {
    if constexpr (BIASED)
      return bias_span(q, a.r, a.b, i0, i1);
    else
      return key_span(q, a.r, i0, i1);
  }();
  // runs of `chunk` keys, longer ones where max_chunks of them would not reach
  const uint32_t chunk = max(a.chunk, (ks.total / a.max_chunks / AR_KEYS + 1) * AR_KEYS);
  const uint32_t n_chunks = max(1u, (ks.total + chunk - 1) / chunk);
  if (blockIdx.y >= n_chunks) return;
  const uint32_t u0 = blockIdx.y * chunk, u1 = min(ks.total, u0 + chunk);
  const uint32_t n_steps = u1 > u0 ? (u1 - u0 + AR_KEYS - 1) / AR_KEYS : 0;

  const uint32_t sm = step_smem(smem);
  const uint32_t stage_bytes = 2 * AR_KEYS * DP * 2;
  // this thread's piece of the rows it stages
  const uint32_t pc = tid % CH, pr = tid / CH;
  const bool piece_ok = pc * 8 < D;
  // element offset of a key's row in the pools (~0: reads zeros)
  auto row_at = [&](uint32_t u) -> uint64_t {
    if (u >= u1) return ~0ull;
    uint32_t pi, slot;
    const uint32_t j = ks.slot(u);
    if constexpr (BIASED)
      if (!somebody_sees(q, a.r, a.b, ks.holes, ks.s_lo + ks.s_n, i0, i1, j)) return ~0ull;
    split_slot(a.c, j, &pi, &slot);
    const uint32_t page = a.c.pages[q.page0 + pi];
    if (page >= a.c.n_pages) {
      record(a.err, ERR_INVAL);
      return ~0ull;
    }
    return page * a.c.page_stride + kh * a.c.head_stride + slot * a.c.slot_stride;
  };
  uint64_t at[PASSES];
  auto look_up = [&](uint32_t step) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) at[i] = row_at(u0 + step * AR_KEYS + i * RPP + pr);
  };
  auto fetch = [&](uint32_t step) {
    const uint32_t base = sm + (step % AR_STAGES) * stage_bytes;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const uint32_t r = i * RPP + pr;
      const uint32_t off = r * DP * 2 + ((pc ^ (r & 7)) * 16);
      const bool ok = at[i] != ~0ull && piece_ok;
      const uint64_t e = ok ? at[i] + pc * 8 : 0;
      cp_async16_or_zero(base + off, (const T*)a.c.k + e, ok);
      cp_async16_or_zero(base + AR_KEYS * DP * 2 + off, (const T*)a.c.v + e, ok);
    }
  };
  look_up(0);
#pragma unroll
  for (int s = 0; s < AR_STAGES - 1; ++s) {
    if (s < (int)n_steps) {
      fetch(s);
      look_up(s + 1);
    }
    cp_async_commit();
  }

  // queries as matrix fragments; rows past the tile's are zero
  uint32_t qf[DP / 16][4];
  int64_t row_a[2];
  RowSee see[2] = {};          // biased: what the rows see, their slopes
  float slope[2] = {0.f, 0.f};
  {
    const T* qp[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t r = warp * 16 + lane / 4 + 8 * z;
      qp[z] = nullptr;
      row_a[z] = INT64_MIN / 2;
      if (r < rows) {
        const uint32_t i = i0 + r / gn, g = g0 + r % gn;
        qp[z] = (const T*)a.r.q + (q.tok0 + i) * a.r.q_tok + (uint64_t)(kh * G + g) * a.r.q_head;
        row_a[z] = q.first + i;
        if constexpr (BIASED) {
          see[z] = row_see(q, a.r, a.b, i);
          slope[z] = slope_log2(a.b, kh * G + g);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const uint32_t d = k * 16 + (z >> 1) * 8 + (lane & 3) * 2;
        const T* p = qp[z & 1];
        qf[k][z] = p && d < D ? *(const uint32_t*)(p + d) : 0u;
      }
    }
  }
  float o[DP / 8][4];
#pragma unroll
  for (int i = 0; i < DP / 8; ++i)
#pragma unroll
    for (int z = 0; z < 4; ++z) o[i][z] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const int64_t a_min = q.first + i0, a_max = q.first + i1 - 1;

  for (uint32_t step = 0; step < n_steps; ++step) {
    cp_async_wait<AR_STAGES - 2>();
    __syncthreads();
    if (step + AR_STAGES - 1 < n_steps) {
      fetch(step + AR_STAGES - 1);
      look_up(step + AR_STAGES);
    }
    cp_async_commit();
    const uint32_t kb = sm + (step % AR_STAGES) * stage_bytes, vb = kb + AR_KEYS * DP * 2;
    float s[KW / 8][4];
#pragma unroll
    for (int i = 0; i < KW / 8; ++i)
#pragma unroll
      for (int z = 0; z < 4; ++z) s[i][z] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
#pragma unroll
      for (int n = 0; n < KW / 16; ++n) {
        const uint32_t r = n * 16 + (lane & 7) + ((lane >> 4) << 3), c = k * 2 + ((lane >> 3) & 1);
        uint32_t b[4];
        ldsm4(b, kb + r * DP * 2 + ((c ^ (r & 7)) * 16));
        mma16<T>(s[2 * n], qf[k], b[0], b[1]);
        mma16<T>(s[2 * n + 1], qf[k], b[2], b[3]);
      }
    }
    // what each row sees of these keys
    const uint32_t ub = u0 + step * AR_KEYS;
    const uint32_t j_lo = ks.slot(ub), j_hi = ks.slot(min(ub + AR_KEYS, u1) - 1);
    bool all = ub + AR_KEYS <= u1;
    if constexpr (BIASED)
      all = all && ks.holes == 0u && j_lo >= ks.all_lo && j_hi < ks.all_hi;
    else
      all = all && (int64_t)j_hi <= a_min && (a.r.window == 0u || (int64_t)j_lo > a_max - (int64_t)a.r.window);
#pragma unroll
    for (int n = 0; n < KW / 8; ++n)
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const uint32_t u = ub + n * 8 + (lane & 3) * 2 + (z & 1);
        float x;
        if constexpr (BIASED) {
          const uint32_t j = ks.slot(u);
          x = a.b.cap_log2 != 0.f ? capped(a.b, s[n][z]) : s[n][z] * a.r.scale_log2;
          x = fmaf(-slope[z >> 1], fabsf((float)(row_a[z >> 1] - (int64_t)j)), x);
          if (!all && (u >= u1 || !see[z >> 1].sees(j))) x = -INFINITY;
        } else {
          x = s[n][z] * a.r.scale_log2;
          if (!all && (u >= u1 || !sees(a.r, row_a[z >> 1], ks.slot(u)))) x = -INFINITY;
        }
        s[n][z] = x;
      }
    float nm[2] = {m[0], m[1]};
#pragma unroll
    for (int n = 0; n < KW / 8; ++n)
#pragma unroll
      for (int z = 0; z < 4; ++z) nm[z >> 1] = fmaxf(nm[z >> 1], s[n][z]);
    float f[2], sub[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      nm[z] = fmaxf(nm[z], __shfl_xor_sync(0xffffffffu, nm[z], 1));
      nm[z] = fmaxf(nm[z], __shfl_xor_sync(0xffffffffu, nm[z], 2));
      const float top = nm[z] == -INFINITY ? 0.f : nm[z];   // a row that has seen nothing yet
      f[z] = exp2f(m[z] - top);
      sub[z] = weight_base<T>(top);
      m[z] = nm[z];
      l[z] *= f[z];
    }
    uint32_t p[KW / 16][4];
#pragma unroll
    for (int n = 0; n < KW / 8; ++n) {
      float e[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        e[z] = exp2f(s[n][z] - sub[z >> 1]);
        l[z >> 1] += e[z];
      }
      // rounded to the cache's type for the product with V; l sums what is not rounded
      p[n / 2][(n & 1) * 2] = pack2<T>(e[0], e[1]);
      p[n / 2][(n & 1) * 2 + 1] = pack2<T>(e[2], e[3]);
    }
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
#pragma unroll
      for (int z = 0; z < 4; ++z) o[i][z] *= f[z >> 1];
#pragma unroll
    for (int n = 0; n < KW / 16; ++n) {
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        const uint32_t r = n * 16 + (lane & 15), c = d * 2 + (lane >> 4);
        uint32_t b[4];
        ldsm4_t(b, vb + r * DP * 2 + ((c ^ (r & 7)) * 16));
        mma16<T>(o[2 * d], p[n], b[0], b[1]);
        mma16<T>(o[2 * d + 1], p[n], b[2], b[3]);
      }
    }
  }
  cp_async_wait<0>();
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    l[z] += __shfl_xor_sync(0xffffffffu, l[z], 1);
    l[z] += __shfl_xor_sync(0xffffffffu, l[z], 2);
  }
  __syncthreads();
  // each warp's rows are its own: to the output, or to this run's partial result
  float* part = a.partial + (((uint64_t)blockIdx.x * a.max_chunks + blockIdx.y) * ROWS) * (uint64_t)(DP + 2);
  T* out = (T*)a.out;
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const uint32_t r = warp * 16 + lane / 4 + 8 * z;
    if (r >= rows) continue;
    const uint64_t t = q.tok0 + i0 + r / gn;
    const uint32_t h = kh * G + g0 + r % gn;
    const float inv = l[z] > 0.f || l[z] != l[z] ? 1.f / l[z] : 0.f;
    float* pp = part + r * (DP + 2);
    if (n_chunks > 1) {
      if ((lane & 3) == 0) __stcg((float2*)(pp + DP), make_float2(m[z], l[z]));
    } else if ((lane & 3) == 0 && a.lse) {
      a.lse[t * a.n_q_heads + h] = row_lse<T>(m[z], l[z]);
    }
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
      const uint32_t d = i * 8 + (lane & 3) * 2;
      if (n_chunks > 1)
        __stcg((float2*)(pp + d), make_float2(o[i][z * 2], o[i][z * 2 + 1]));
      else if (d < D)
        *(uint32_t*)(out + t * a.out_tok + h * a.out_head + d) = pack2<T>(o[i][z * 2] * inv, o[i][z * 2 + 1] * inv);
    }
  }
  if (n_chunks == 1) return;
  __threadfence();
  __syncthreads();
  if (tid == 0) s_last = ticket(a.counter + blockIdx.x) == n_chunks - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const float* p0 = a.partial + ((uint64_t)blockIdx.x * a.max_chunks * ROWS) * (uint64_t)(DP + 2);
  const uint64_t step = (uint64_t)ROWS * (DP + 2);
  for (uint32_t x = tid; x < rows * (DP / 2); x += AR_THREADS) {
    const uint32_t r = x / (DP / 2), d = (x - r * (DP / 2)) * 2;
    const float* pp = p0 + r * (DP + 2);
    float M = -INFINITY;
    for (uint32_t k = 0; k < n_chunks; ++k) M = fmaxf(M, __ldcg(pp + k * step + DP));
    const float sub = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    float2 acc = make_float2(0.f, 0.f);
    for (uint32_t k = 0; k < n_chunks; ++k) {
      const float2 ml = __ldcg((const float2*)(pp + k * step + DP));
      const float2 v = __ldcg((const float2*)(pp + k * step + d));
      const float f = exp2f(ml.x - sub);
      L += f * ml.y;
      acc.x += f * v.x;
      acc.y += f * v.y;
    }
    const uint64_t t = q.tok0 + i0 + r / gn;
    const uint32_t h = kh * G + g0 + r % gn;
    const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
    if (d < D)
      *(uint32_t*)(out + t * a.out_tok + h * a.out_head + d) = pack2<T>(acc.x * inv, acc.y * inv);
    if (d == 0 && a.lse) a.lse[t * a.n_q_heads + h] = row_lse<T>(M, L);
  }
  if (tid == 0) a.counter[blockIdx.x] = 0u;   // for the next call
}

template <typename T, int DP>
static void launch_rows(const LaunchCfg& L, const AttendArgs& a) {
  launch_k(L, K_ATTEND_ROWS, a.biased ? attend_rows_kernel<T, DP, true> : attend_rows_kernel<T, DP, false>,
           dim3(a.tiles * a.c.n_heads, a.max_chunks), AR_THREADS, attend_rows_smem<DP>(), a);
}
void launch_attend_rows(const LaunchCfg& L, const AttendArgs& a, int dtype) {
  const bool narrow = a.c.head_dim <= 64;
  if (dtype == RO_BF16)
    narrow ? launch_rows<__nv_bfloat16, 64>(L, a) : launch_rows<__nv_bfloat16, 128>(L, a);
  else
    narrow ? launch_rows<__half, 64>(L, a) : launch_rows<__half, 128>(L, a);
}

template <typename T, int DP>
static cudaError_t allow() {
  const int bytes = (int)attend_rows_smem<DP>();
  const cudaError_t e =
      cudaFuncSetAttribute(attend_rows_kernel<T, DP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e != cudaSuccess
             ? e
             : cudaFuncSetAttribute(attend_rows_kernel<T, DP, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
cudaError_t prepare_attend_kernels() {
  for (cudaError_t e : {allow<__nv_bfloat16, 64>(), allow<__nv_bfloat16, 128>(), allow<__half, 64>(), allow<__half, 128>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace ro
