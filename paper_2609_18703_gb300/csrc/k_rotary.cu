// k_rotary.cu — rotary positions with several axes (ro_rotary, ro_cache_append).
//
// Pair p of a head turns by theta = pos[axis(p)] * base^(-p/R):
//   (x0, x1) -> (x0 cos - x1 sin, x1 cos + x0 sin),  theta negated turns back.
// The frequency is held in 1/2^64 of a turn, so the 64-bit product with the
// integer position is the angle modulo a turn, exactly: nothing is lost for
// large positions.  Its upper 32 bits become a float for the sine and cosine,
// which errs by 9.4e-8 radians at most (near half a turn).
//
// Bound by memory: every element is read and written once.  A CTA takes a few
// tokens, computes their R sines and cosines once in shared memory and turns
// all heads with them; a thread moves two vectors of up to 16 bytes.
// Measured: 65,536 tokens of 32 heads of 128 (1.07 GB) 171 us, 6.3 TB/s; the
// append of 24 ragged chunks (687 MB) 113 us, 6.1 TB/s.
#include <algorithm>

#include "ro_step.cuh"

namespace ro {

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T v[V];
};

template <typename T, int V>
__global__ void __launch_bounds__(TURN_THREADS) turn_kernel(const __grid_constant__ TurnArgs a) {
  extern __shared__ float2 s_turn[];   // [tokens_per_cta][pairs]: cos, sin
  __shared__ uint64_t s_at[8];   // paged parts: the token's place in the pool, ~0: left out
  wait_predecessor();
  const uint32_t tid = threadIdx.x;
  const uint64_t t0 = (uint64_t)blockIdx.x * a.tokens_per_cta;
  const uint32_t nt = (uint32_t)(a.n_tokens - t0 < a.tokens_per_cta ? a.n_tokens - t0 : a.tokens_per_cta);
  const uint32_t R = a.rope.pairs;
  for (uint32_t i = tid; i < nt * R; i += TURN_THREADS) {
    const uint32_t t = i / R, p = i - t * R;
    const int64_t pos = a.pos[(t0 + t) * a.rope.n_axes + a.rope.axis[p]];
    const int32_t turn = (int32_t)(((uint64_t)pos * a.rope.freq[p]) >> 32);   // of 2^32
    float sn, cs;
    sincospif((float)turn * 0x1p-31f, &sn, &cs);
    s_turn[i] = make_float2(cs, a.inverse ? -sn : sn);
  }
  if (a.tok_base != nullptr && tid < nt) {
    // the token's page and slot
    const uint64_t t = t0 + tid;
    const uint32_t s = a.tok_seq[t];
    uint64_t at = ~0ull;
    bool bad = s >= a.n_seqs, full = false;
    if (!bad) {
      const uint64_t b0 = a.tok_base[s], b1 = a.tok_base[s + 1], p0 = a.page_base[s], p1 = a.page_base[s + 1],
                     end = a.page_base[a.n_seqs];
      const uint32_t len = a.len[s];
      bad = t < b0 || t >= b1 || p1 < p0 || p1 > end || len >= 0x80000000u;
      const int64_t slot = (int64_t)len - (int64_t)(b1 - b0) + (int64_t)(t - b0);
      if (!bad && slot >= 0) {
        const uint32_t pi = (uint32_t)slot / a.page_size;
        if (pi >= p1 - p0) {
          full = true;
        } else {
          const uint32_t page = a.pages[p0 + pi];
          if (page >= a.n_pages)
            bad = true;
          else
            at = page * a.page_stride + ((uint32_t)slot - pi * a.page_size) * a.slot_stride;
        }
      }
    }
    if (bad) record(a.err, ERR_INVAL);
    if (full) record(a.err, ERR_CAPACITY);
    s_at[tid] = at;
  }
  __syncthreads();
  // items: for each token, each part's heads in turn, D / 2V pairs of vectors
  const uint32_t half = a.head_dim / 2, per = half / V;
  uint32_t heads = 0;
  for (uint32_t k = 0; k < a.n_parts; ++k) heads += a.part[k].heads;
  const uint32_t items = nt * heads * per;
  for (uint32_t i = tid; i < items; i += TURN_THREADS) {
    const uint32_t row = i / per, m = (i - row * per) * V;
    const uint32_t t = row / heads;
    uint32_t h = row - t * heads, k = 0;
    while (h >= a.part[k].heads) h -= a.part[k++].heads;
    const TurnPart& pt = a.part[k];
    const T* src = (const T*)pt.src + (t0 + t) * pt.src_tok + h * pt.src_head;
    T* dst = (T*)pt.dst;
    if (pt.paged) {
      if (s_at[t] == ~0ull) continue;
      dst += s_at[t] + h * pt.dst_head;
    } else {
      dst += (t0 + t) * pt.dst_tok + h * pt.dst_head;
    }
    typedef Vec<T, V> W;
    if (a.rope.interleaved || !pt.turn) {   // 2V neighbouring elements
      const uint32_t e = 2 * m;
      alignas(16) T x[2 * V];
      *(W*)x = *(const W*)(src + e);
      *(W*)(x + V) = *(const W*)(src + e + V);
      if (pt.turn && m < R) {
        const float2* cs = s_turn + t * R + m;
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const float u = to_f32(x[2 * q]), w = to_f32(x[2 * q + 1]);
          x[2 * q] = from_f32<T>(u * cs[q].x - w * cs[q].y);
          x[2 * q + 1] = from_f32<T>(w * cs[q].x + u * cs[q].y);
        }
      }
      *(W*)(dst + e) = *(const W*)x;
      *(W*)(dst + e + V) = *(const W*)(x + V);
    } else {                                 // V pairs, halves R apart; then the rest in two halves
      const bool turn = m < R;
      const uint32_t e0 = turn ? m : R + m, e1 = turn ? m + R : half + m;
      W x0 = *(const W*)(src + e0), x1 = *(const W*)(src + e1);
      if (turn) {
        const float2* cs = s_turn + t * R + m;
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const float u = to_f32(x0.v[q]), w = to_f32(x1.v[q]);
          x0.v[q] = from_f32<T>(u * cs[q].x - w * cs[q].y);
          x1.v[q] = from_f32<T>(w * cs[q].x + u * cs[q].y);
        }
      }
      *(W*)(dst + e0) = x0;
      *(W*)(dst + e1) = x1;
    }
  }
}

template <typename T>
static void launch_vec(const LaunchCfg& L, const TurnArgs& a, int vec, int grid, size_t smem) {
  if (vec == 8 && sizeof(T) == 2)
    launch_k(L, K_ROTARY, turn_kernel<T, sizeof(T) == 2 ? 8 : 4>, grid, TURN_THREADS, smem, a);
  else if (vec >= 4)
    launch_k(L, K_ROTARY, turn_kernel<T, 4>, grid, TURN_THREADS, smem, a);
  else if (vec == 2)
    launch_k(L, K_ROTARY, turn_kernel<T, 2>, grid, TURN_THREADS, smem, a);
  else
    launch_k(L, K_ROTARY, turn_kernel<T, 1>, grid, TURN_THREADS, smem, a);
}

void launch_turn(const LaunchCfg& L, const TurnArgs& in, int dtype, int vec, int sms) {
  TurnArgs a = in;
  // Tokens of a CTA: enough that its sines fill the threads (256 of them; at
  // most 8 tokens), fewer when there would not be four CTAs for every SM.
  const uint64_t fill = std::min<uint64_t>(8, std::max<uint64_t>(1, TURN_THREADS / std::max<uint32_t>(a.rope.pairs, 1)));
  a.tokens_per_cta = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(fill, a.n_tokens / ((uint64_t)sms * 4)));
  const int grid = (int)ceil_div(a.n_tokens, a.tokens_per_cta);
  const size_t smem = (size_t)a.tokens_per_cta * a.rope.pairs * sizeof(float2);
  if (dtype == RO_BF16)
    launch_vec<__nv_bfloat16>(L, a, vec, grid, smem);
  else if (dtype == RO_F16)
    launch_vec<__half>(L, a, vec, grid, smem);
  else
    launch_vec<float>(L, a, vec, grid, smem);
}

}  // namespace ro
