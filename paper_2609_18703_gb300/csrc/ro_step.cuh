// ro_step.cuh — device helpers shared by the model-step kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ro_step.h"

namespace ro {

constexpr float LN2 = 0.69314718055994530942f;

__device__ __forceinline__ uint32_t step_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void record(uint32_t* err, uint32_t bit) { atomicOr(err, bit); }

// 16 bytes to shared memory, zeros instead when !ok (src is then not read)
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}

// c += a (16 x 16) * b (16 x 8), 32-bit accumulation
template <typename T>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                     uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ float to_f32(T x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Softmax weights are rounded to the cache's type for the product with the
// values.  f16 has nothing below 2^-25, so its weights are held 2^UP times
// higher, up to 2^15: behind a heavy first token the light ones, many of them,
// would else add to the row's sum and not to its output.  The sums l and o are
// 2^UP times higher too; only the logarithm of l has to know.  bf16 has the
// exponents of 32 bits.  SLACK: log2 of what weights may pass 1.
template <typename T, int SLACK = 0>
constexpr int WEIGHT_UP = 0;
template <int SLACK>
constexpr int WEIGHT_UP<__half, SLACK> = 15 - SLACK;
// ln sum_j exp(..) of a row from its maximum (in log2) and its sum
template <typename T, int SLACK = 0>
__device__ __forceinline__ float row_lse(float m, float l) {
  constexpr float down = 1.f / (1u << WEIGHT_UP<T, SLACK>);
  return l == 0.f ? -INFINITY : (m + log2f(l * down)) * LN2;
}

// Rows that fill up a tile of weights repeat a row of the tile, with this for
// the lse (in log2): their weights are 0 where that row's are finite, and
// infinite or NaN only where its are.  (Rows of zeros would make NaN of a key
// with an infinity, whose own weight is 0.)
constexpr float LSE_FILL = 1e38f;

// ---- clusters ------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// every thread of the cluster; shared memory written before it is seen after it
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// an address of this CTA's shared memory in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t cluster_at(uint32_t addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t addr, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(cluster_at(addr, rank))
               : "memory");
  return v;
}
__device__ __forceinline__ float2 cluster_load2(uint32_t addr, uint32_t rank) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_at(addr, rank)) : "memory");
  return v;
}

// One sequence's rows and pages, read once per CTA.
struct SeqInfo {
  uint64_t tok0;             // first of its new tokens
  uint32_t n;                // new tokens
  uint32_t len;              // cached tokens, at most what its pages hold
  uint64_t page0;            // first entry of its page list
  int64_t first;             // slot of its first new token (negative: before the cache)
  bool ok;
};
// Checks what the GPU alone can see; a sequence that fails is left out (ok false).
__device__ __forceinline__ SeqInfo seq_info(const PagedArgs& c, const RowsArgs& r, uint32_t s, uint32_t* err) {
  SeqInfo q;
  // (all loads at once: a short-circuited one would wait for the others)
  const uint64_t t0 = r.tok_base[s], t1 = r.tok_base[s + 1], p0 = c.page_base[s], p1 = c.page_base[s + 1],
                 end = c.page_base[c.n_seqs];
  const uint32_t len = r.len[s];
  q.tok0 = t0;
  q.n = (uint32_t)(t1 - t0);
  q.len = len;
  q.page0 = p0;
  q.ok = t0 <= t1 && t1 <= r.n_tokens && t1 - t0 <= r.max_new && p0 <= p1 && p1 <= end &&
         len < 0x80000000u;
  if (!q.ok) {
    if ((threadIdx.x & 31u) == 0) record(err, ERR_INVAL);
    q.n = 0;
    q.len = 0;
  } else if ((uint64_t)len > (p1 - p0) * c.page_size) {
    if ((threadIdx.x & 31u) == 0) record(err, ERR_CAPACITY);
    q.len = (uint32_t)((p1 - p0) * c.page_size);
  }
  q.first = (int64_t)len - (int64_t)q.n;
  return q;
}
__device__ __forceinline__ uint32_t page_index(const PagedArgs& c, uint32_t j) {
  return c.page_shift >= 0 ? j >> c.page_shift : j / c.page_size;
}
__device__ __forceinline__ void split_slot(const PagedArgs& c, uint32_t j, uint32_t* page, uint32_t* slot) {
  *page = page_index(c, j);
  *slot = j - *page * c.page_size;
}

// The keys that the tokens [i0, i1) of a sequence see, numbered without the
// gap between the sinks and the window: u < s_hi is slot u, then slot
// lo + (u - s_hi).
struct KeySpan {
  uint32_t s_hi, lo, total;
  __device__ __forceinline__ uint32_t slot(uint32_t u) const { return u < s_hi ? u : lo + (u - s_hi); }
};
__device__ __forceinline__ KeySpan key_span(const SeqInfo& q, const RowsArgs& r, uint32_t i0, uint32_t i1) {
  KeySpan k;
  const int64_t a0 = q.first + i0, a1 = q.first + i1 - 1;
  int64_t hi = a1 + 1 < (int64_t)q.len ? a1 + 1 : (int64_t)q.len;
  if (hi < 0 || i1 <= i0) hi = 0;
  int64_t lo = r.window ? a0 - (int64_t)r.window + 1 : 0;
  if (lo < 0) lo = 0;
  if (lo > hi) lo = hi;
  k.lo = (uint32_t)lo;
  k.s_hi = (uint32_t)((int64_t)r.sinks < lo ? (int64_t)r.sinks : lo);
  k.total = k.s_hi + (uint32_t)(hi - lo);
  return k;
}
__device__ __forceinline__ bool sees(const RowsArgs& r, int64_t a, uint32_t j) {
  return (int64_t)j <= a && (r.window == 0u || (int64_t)j > a - (int64_t)r.window || j < r.sinks);
}

// The slots that a CTA's rows see, cut into tiles of KEYS: tiles over the
// sinks, then tiles from the window's first slot (rounded down to `box`, the
// slots that are loaded together) on.  [lo, hi) of a tile are the slots that
// count.
struct SlotTile {
  uint32_t t0, lo, hi;
  bool sink;
};
template <int KEYS>
struct SlotTiles {
  uint32_t s_hi, lo, hi, first, sink_tiles, n;
  __device__ __forceinline__ SlotTiles(const KeySpan& ks, uint32_t box) {
    s_hi = ks.s_hi;
    lo = ks.lo;
    hi = ks.lo + (ks.total - ks.s_hi);
    first = lo & ~(box - 1u);
    sink_tiles = (s_hi + KEYS - 1) / KEYS;
    n = sink_tiles + (hi > lo ? (hi - first + KEYS - 1) / KEYS : 0);
  }
  __device__ __forceinline__ SlotTile at(uint32_t t) const {
    SlotTile s;
    s.sink = t < sink_tiles;
    s.t0 = s.sink ? t * KEYS : first + (t - sink_tiles) * KEYS;
    s.lo = s.sink ? s.t0 : max(s.t0, lo);
    s.hi = min(s.t0 + KEYS, s.sink ? s_hi : hi);
    return s;
  }
};

// The new tokens [i0, i1) of a sequence that can see one of the slots
// [j_lo, j_hi].
__device__ __forceinline__ void seeing_tokens(const SeqInfo& q, const RowsArgs& r, uint32_t j_lo, uint32_t j_hi,
                                              uint32_t* i0, uint32_t* i1) {
  *i0 = 0;
  *i1 = q.n;
  const int64_t f = (int64_t)j_lo - q.first;
  if (f > 0) *i0 = (uint32_t)min((int64_t)q.n, f);
  if (r.window && j_lo >= r.sinks) {
    const int64_t e = (int64_t)j_hi + r.window - q.first;   // a < j + window
    *i1 = (uint32_t)max((int64_t)*i0, min((int64_t)q.n, e));
  }
}

// score = decay past for the slots [from, to) of a row of scores that no token
// sees (from a multiple of 4), four at a time where the rows are aligned to it.
template <int THREADS>
__device__ __forceinline__ void decay_past(const WeighArgs& a, uint64_t row, uint32_t from, uint32_t to, uint32_t thread) {
  float* score = a.score + row;
  const float* past = a.past ? a.past + row : nullptr;
  uint32_t done = from;
  if (((reinterpret_cast<uintptr_t>(score) | reinterpret_cast<uintptr_t>(past)) & 15u) == 0u) {
    const uint32_t end = to & ~3u;
    for (uint32_t j = from + thread * 4; j < end; j += THREADS * 16) {
      float4 v[4];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (j + i * THREADS * 4 < end)
          v[i] = past ? *(const float4*)(past + j + i * THREADS * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (j + i * THREADS * 4 < end)
          *(float4*)(score + j + i * THREADS * 4) =
              past ? make_float4(a.decay * v[i].x, a.decay * v[i].y, a.decay * v[i].z, a.decay * v[i].w) : v[i];
    }
    done = max(from, end);
  }
  for (uint32_t j = done + thread; j < to; j += THREADS * 4) {
    float v[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[i] = past && j + i * THREADS < to ? past[j + i * THREADS] : 0.f;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (j + i * THREADS < to) score[j + i * THREADS] = past ? a.decay * v[i] : 0.f;
  }
}

// Row tile `tile` (of toks_per_tile tokens): its sequence and its place among
// that sequence's tiles.  A whole warp calls it; with one tile per sequence
// (max_new tokens fit a tile) it is the sequence itself.  The host launches
// one tile more than there can be, so that some CTA walks the whole list and
// records a range that has no tiles because it is out of bounds.
__device__ __forceinline__ bool find_tile(const RowsArgs& r, uint32_t n_seqs, uint32_t tile, uint32_t toks_per_tile,
                                          uint32_t* seq, uint32_t* part, uint32_t* err) {
  if (r.max_new <= toks_per_tile) {
    *seq = tile;
    *part = 0;
    return tile < n_seqs;
  }
  const uint32_t lane = threadIdx.x & 31u;
  uint64_t before = 0;
  for (uint32_t s0 = 0; s0 < n_seqs; s0 += 32) {
    const uint32_t s = s0 + lane;
    uint32_t t = 0;
    if (s < n_seqs) {
      const uint64_t b0 = r.tok_base[s], b1 = r.tok_base[s + 1];
      if (b1 >= b0 && b1 - b0 <= r.max_new && b1 <= r.n_tokens)
        t = (uint32_t)((b1 - b0 + toks_per_tile - 1) / toks_per_tile);
      else
        record(err, ERR_INVAL);
    }
    const uint32_t inc = warp_incl_scan(t);
    const uint32_t total = __shfl_sync(0xffffffffu, inc, 31);
    if (tile < before + total) {
      const uint32_t want = (uint32_t)(tile - before);
      const uint32_t hit = __ballot_sync(0xffffffffu, inc > want);
      const int l = __ffs(hit) - 1;
      *seq = s0 + l;
      *part = want - (__shfl_sync(0xffffffffu, inc, l) - __shfl_sync(0xffffffffu, t, l));
      return true;
    }
    before += total;
  }
  return false;
}

// The same with the tiles that see the most slots first (without a window a
// tile's work is the slot after its last token, `hi`), so that the last CTAs
// to start are short ones.  The tile of rank r has the largest hi = w with at
// least r + 1 tiles at or above w, found by bisection: a sequence's tiles at
// or above w are counted in closed form.  At most 32 * FT_SEQS sequences.
constexpr uint32_t FT_SEQS = 4;
__device__ __forceinline__ bool find_tile_heavy(const RowsArgs& r, uint32_t n_seqs, uint32_t rank,
                                                uint32_t toks_per_tile, uint32_t* seq, uint32_t* part, uint32_t* err) {
  const uint32_t lane = threadIdx.x & 31u, nk = (n_seqs + 31) / 32;
  const uint32_t recip = 0xFFFFFFFFu / toks_per_tile + 1u;   // a division by product: the order may err by a slot
  int32_t first[FT_SEQS], len[FT_SEQS], top = 0;
  uint32_t tiles[FT_SEQS];
#pragma unroll
  for (uint32_t k = 0; k < FT_SEQS; ++k) {
    const uint32_t s = lane * nk + k;   // a lane's sequences are neighbours: ranks follow their order
    first[k] = len[k] = 0;
    tiles[k] = 0;
    if (k < nk && s < n_seqs) {
      const uint64_t b0 = r.tok_base[s], b1 = r.tok_base[s + 1];
      if (b1 >= b0 && b1 - b0 <= r.max_new && b1 <= r.n_tokens) {
        len[k] = (int32_t)(r.len[s] & 0x7FFFFFFFu);
        first[k] = len[k] - (int32_t)(b1 - b0);
        top = max(top, len[k]);
        tiles[k] = (uint32_t)((b1 - b0 + toks_per_tile - 1) / toks_per_tile);
      } else {
        record(err, ERR_INVAL);
      }
    }
  }
  auto at_least = [&](uint32_t k, uint32_t w) -> uint32_t {   // sequence k's tiles with hi >= w
    if (w == 0) return tiles[k];
    if (w > (uint32_t)len[k]) return 0;
    const int32_t d = (int32_t)w - first[k];   // at most its new tokens
    return tiles[k] - (d <= 0 ? 0u : min(tiles[k], __umulhi((uint32_t)d - 1u, recip)));
  };
  auto count = [&](uint32_t w) -> uint32_t {
    uint32_t c = 0;
#pragma unroll
    for (uint32_t k = 0; k < FT_SEQS; ++k)
      if (k < nk) c += at_least(k, w);
    return __reduce_add_sync(0xffffffffu, c);
  };
  if (count(0) <= rank) return false;
  uint32_t lo = 0, hi = (uint32_t)__reduce_max_sync(0xffffffffu, top) + 1u;   // count(lo) > rank >= count(hi)
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (count(mid) > rank)
      lo = mid;
    else
      hi = mid;
  }
  // of the tiles with hi == lo (0: or below), the one of what rank is left
  uint32_t left = rank - count(lo + 1), mine = 0;
  uint32_t eq[FT_SEQS];
#pragma unroll
  for (uint32_t k = 0; k < FT_SEQS; ++k) {
    eq[k] = at_least(k, lo) - at_least(k, lo + 1);
    mine += eq[k];
  }
  const uint32_t inc = warp_incl_scan(mine);
  const int l = __ffs(__ballot_sync(0xffffffffu, inc > left)) - 1;
  uint32_t s = 0, p = 0;
  left -= inc - mine;   // (of use in lane l)
#pragma unroll
  for (uint32_t k = 0; k < FT_SEQS; ++k) {
    if (left < eq[k]) {
      s = lane * nk + k;
      p = tiles[k] - at_least(k, lo) + left;
      left = 0xFFFFFFFFu;
    } else if (left != 0xFFFFFFFFu) {
      left -= eq[k];
    }
  }
  *seq = __shfl_sync(0xffffffffu, s, l);
  *part = __shfl_sync(0xffffffffu, p, l);
  return true;
}

}  // namespace ro
