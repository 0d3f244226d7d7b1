// ro_tcgen05.cuh — tensor-core, TMA and barrier primitives of the tiled model-step kernels.
//
// Operand tiles lie in shared memory in blocks of 64 columns (128 bytes) with
// the 128-byte swizzle, as TMA writes them: 8-row groups of 1,024 bytes.
#pragma once

#include <cuda.h>

#include "ro_step.cuh"

namespace ro {

// ---- barriers ---------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok)
               : "r"(bar), "r"(parity)
               : "memory");
  return ok != 0u;
}
__device__ __forceinline__ unsigned long long timer_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Every wait is bounded: past two seconds it records ERR_TIMEOUT and sets the
// CTA's flag, which ends all its other waits; the kernel then runs to its end
// without waiting, frees its TMEM and the call's results are void.
__device__ __forceinline__ void bar_wait_slow(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up,
                                                  uint32_t* err) {
  const unsigned long long t0 = timer_ns();
  for (uint32_t spins = 1;; ++spins) {
    if (bar_try(bar, parity) || *gave_up) return;
    if ((spins & 63u) == 0u && timer_ns() - t0 > 2000000000ull) {
      record(err, ERR_TIMEOUT);
      *gave_up = 1u;
      return;
    }
  }
}
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t* err) {
  if (!bar_try(bar, parity)) bar_wait_slow(bar, parity, gave_up, err);
}
// A wait that need not end at once: it leaves the issue slots to others.
__device__ __forceinline__ void bar_wait_idle(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t* err) {
  const unsigned long long t0 = timer_ns();
  while (!bar_try(bar, parity) && !*gave_up) {
    if (timer_ns() - t0 > 2000000000ull) {
      record(err, ERR_TIMEOUT);
      *gave_up = 1u;
    }
    __nanosleep(200);
  }
}
// a whole warp, so that it leaves a loop together
__device__ __forceinline__ bool has_given_up(volatile uint32_t* gave_up) {
  return __any_sync(0xffffffffu, *gave_up != 0u);
}

// ---- TMA ----------------------------------------------------------------------------------
__device__ __forceinline__ void tma4(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::
          "r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void tma3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- TMEM ----------------------------------------------------------------------------------
// a whole warp; the address lands in shared memory
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Waits for this thread's loads from TMEM into r (and all earlier ones): what
// uses r comes after it.
template <int N>
__device__ __forceinline__ void tc_wait_ld(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the barrier is arrived at when every product issued by the elected lane so far is done
__device__ __forceinline__ void tc_commit(uint32_t one, uint32_t bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.u32 q, %1, 0;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar),
      "r"(one)
      : "memory");
}
// 32 columns of this warp's 32 lanes: thread = lane, register = column
__device__ __forceinline__ void tc_ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tc_ld16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
      : "memory");
}

// ---- matrix products -------------------------------------------------------------------------
// Shared-memory operand with the 128-byte swizzle, in two 32-bit halves: the
// low one holds the address (advance it by bytes / 16) and the distance of
// blocks of 64 m or n; the high one the distance of 8-row groups, 1,024 bytes.
// K-major (rows of 64 consecutive k): `lead` unused.  MN-major (rows of 64
// consecutive m or n, one row per k): lead = bytes between blocks.
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr, uint32_t lead) {
  return ((addr & 0x3FFFFu) >> 4) | ((lead >> 4) << 16);
}
constexpr uint32_t OPERAND_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
// 16-bit operands, 32-bit accumulators, M = 128
template <typename T>
__host__ __device__ constexpr uint32_t mma_shape(uint32_t n, bool b_mn_major);
template <>
__host__ __device__ constexpr uint32_t mma_shape<__nv_bfloat16>(uint32_t n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
template <>
__host__ __device__ constexpr uint32_t mma_shape<__half>(uint32_t n, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
// One lane of the warp, the same every time.  The products are issued under
// this predicate by a warp that has not diverged, so that their operands stay
// in uniform registers; moved there from a divergent branch each product cost
// 80 cycles of issue, more than it takes.
__device__ __forceinline__ uint32_t elect_lane() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p;
}
// d (+)= a b, a and b in shared memory
__device__ __forceinline__ void mma_ss(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.u32 p, %5, 0;\n setp.ne.u32 q, %6, 0;\n"
      " mov.b64 a, {%1, %4};\n mov.b64 b, {%2, %4};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(shape), "r"(OPERAND_HI), "r"((uint32_t)add), "r"(one)
      : "memory");
}
// the same with a in TMEM
__device__ __forceinline__ void mma_ts(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 b;\n setp.ne.u32 p, %5, 0;\n setp.ne.u32 q, %6, 0;\n"
      " mov.b64 b, {%2, %4};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(shape), "r"(OPERAND_HI), "r"((uint32_t)add), "r"(one)
      : "memory");
}

// two 32-bit floats in one operation
__device__ __forceinline__ uint64_t pair_bits(uint32_t lo, uint32_t hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
  return v;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  return pair_bits(__float_as_uint(lo), __float_as_uint(hi));
}
__device__ __forceinline__ float pair_lo(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float pair_hi(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// ---- a ring of stages of slots -----------------------------------------------------------------
// One warp's work: keep a ring of `stages` stages full with the tiles
// [c0, c0 + n) of one sequence and head, KEYS slots of DP dimensions each, keys
// (and values behind them).  By TMA a box (part of a page) a lane; without, row
// by row with cp.async, 32 arrivals on a full stage instead of one.
template <typename T, int DP, int KEYS, bool VALUES, class Slots>
__device__ __forceinline__ void load_stages(const PagedArgs& c, const CUtensorMap* km, const CUtensorMap* vm, bool tma,
                                            uint32_t box, uint32_t stages, const Slots& slots, uint32_t c0,
                                            uint32_t n, uint32_t kh, uint64_t page0, uint32_t sm, uint32_t b_full, uint32_t b_empty,
                                            uint32_t* gave_up, uint32_t* err) {
  constexpr uint32_t BLOCKS = DP / 64, BLOCK_BYTES = KEYS * 128, SIDE = BLOCKS * BLOCK_BYTES;
  constexpr uint32_t STAGE = VALUES ? 2 * SIDE : SIDE;
  const uint32_t lane = threadIdx.x & 31u;
  uint32_t slot = 0, parity = 1;
  if (tma) {
    const uint32_t boxes = KEYS / box;            // of a stage, a lane each
    const uint32_t ahead = 32 / boxes;            // stages whose pages the lanes hold
    auto has_box = [&](const SlotTile& st, uint32_t j) { return j < st.hi && j + box > st.lo; };
    // the page of this lane's box among the boxes of stages t .. t + ahead - 1
    auto page_of = [&](uint32_t t) -> uint32_t {
      const uint32_t u = t + lane / boxes;
      if (u >= n) return 0u;
      const SlotTile st = slots.at(c0 + u);
      const uint32_t j = st.t0 + (lane % boxes) * box;
      return has_box(st, j) ? c.pages[page0 + page_index(c, j)] : 0u;
    };
    uint32_t next = page_of(0), page = 0;
    for (uint32_t t = 0; t < n; ++t) {
      if (t % ahead == 0) {
        page = next;
        next = page_of(t + ahead);
      }
      const SlotTile st = slots.at(c0 + t);
      const uint32_t b = lane % boxes, j = st.t0 + b * box;
      bool load = lane / boxes == t % ahead && has_box(st, j);
      if (load && page >= c.n_pages) {
        record(err, ERR_INVAL);
        load = false;
      }
      const uint32_t loaded = __popc(__ballot_sync(0xffffffffu, load));
      if (t >= stages) bar_wait(b_empty + 8 * slot, parity, gave_up, err);
      if (has_given_up(gave_up)) break;
      const uint32_t full = b_full + 8 * slot, dst = sm + slot * STAGE + b * box * 128;
      if (lane == 0) bar_expect(full, (VALUES ? 2 : 1) * loaded * BLOCKS * box * 128);
      __syncwarp();
      if (load) {
        const int y = (int)(j - page_index(c, j) * c.page_size);
#pragma unroll
        for (uint32_t x = 0; x < BLOCKS; ++x) {
          tma4(dst + x * BLOCK_BYTES, km, x * 64, y, (int)kh, (int)page, full);
          if (VALUES) tma4(dst + SIDE + x * BLOCK_BYTES, vm, x * 64, y, (int)kh, (int)page, full);
        }
      }
      if (++slot == stages) slot = 0, parity ^= 1;
    }
  } else {
    // The pages of a stage's rows are looked up together, a row or more a lane,
    // while the stage before it is being loaded (40 single tokens over 2,000
    // slots in pages of 5: attention 102 us, weights 41 us; looked up row by row
    // 445 and 422 us).
    constexpr uint32_t CH = DP / 8, PER = 32 / CH;   // 16-byte pieces of a row; rows at a time
    constexpr uint32_t R = KEYS / 32;
    const uint32_t pc = lane % CH;
    auto slot_of = [&](const SlotTile& st, uint32_t i) { return st.t0 + i * 32 + lane; };
    auto pages_of = [&](uint32_t t, uint32_t* page) {
#pragma unroll
      for (uint32_t i = 0; i < R; ++i) {
        page[i] = 0;
        if (t >= n) continue;
        const SlotTile st = slots.at(c0 + t);
        const uint32_t j = slot_of(st, i);
        if (j >= st.lo && j < st.hi) page[i] = c.pages[page0 + page_index(c, j)];
      }
    };
    uint32_t next[R];
    pages_of(0, next);
    for (uint32_t t = 0; t < n; ++t) {
      const SlotTile st = slots.at(c0 + t);
      uint64_t row[R];                              // where this lane's rows start; none: all ones
#pragma unroll
      for (uint32_t i = 0; i < R; ++i) {
        const uint32_t j = slot_of(st, i);
        row[i] = ~0ull;
        if (j >= st.lo && j < st.hi) {
          if (next[i] < c.n_pages)
            row[i] = next[i] * c.page_stride + kh * c.head_stride + (j - page_index(c, j) * c.page_size) * c.slot_stride;
          else
            record(err, ERR_INVAL);
        }
      }
      pages_of(t + 1, next);
      if (t >= stages) bar_wait(b_empty + 8 * slot, parity, gave_up, err);
      if (has_given_up(gave_up)) break;
#pragma unroll
      for (uint32_t y = 0; y < (uint32_t)KEYS; y += PER) {
        const uint32_t r = y + lane / CH;
        const uint64_t e = __shfl_sync(0xffffffffu, row[y / 32], r % 32);
        const bool ok = e != ~0ull && pc * 8 < c.head_dim;
        const uint32_t dst = sm + slot * STAGE + (pc / 8) * BLOCK_BYTES + r * 128 + (((pc & 7) ^ (r & 7)) * 16);
        cp_async16_or_zero(dst, (const T*)c.k + (ok ? e + pc * 8 : 0), ok);
        if (VALUES) cp_async16_or_zero(dst + SIDE, (const T*)c.v + (ok ? e + pc * 8 : 0), ok);
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(b_full + 8 * slot) : "memory");
      if (++slot == stages) slot = 0, parity ^= 1;
    }
    cp_async_commit();
    cp_async_wait<0>();
  }
}

// ---- host: tensor maps -----------------------------------------------------------------------
// Slots that one TMA box loads: the largest power of two that divides the
// pages, at most `most`.  A box starts at any multiple of 128 bytes of a
// swizzled tile: the swizzle goes by the address.  Below 4 slots a box the
// loads go row by row.
constexpr uint32_t MIN_BOX = 4;
inline uint32_t page_box(uint32_t page_size, uint32_t most) {
  const uint32_t b = page_size & (0u - page_size);
  return b < most ? b : most;
}
// 64-column blocks with the 128-byte swizzle; false: the tensor cannot be mapped
bool tile_map(CUtensorMap* m, int dtype, const void* p, int dims, const uint64_t* size, const uint64_t* stride,
              const uint32_t* box);
// a cache's pool, boxes of `box` slots of one page and head
bool pool_map(CUtensorMap* m, const PagedArgs& c, const void* pool, int dtype, uint32_t box);
// the query rows, boxes of `toks` tokens times `heads` heads
bool rows_map(CUtensorMap* m, const RowsArgs& r, uint32_t head_dim, uint32_t n_q_heads, int dtype, uint32_t heads,
              uint32_t toks);

struct AttendTileArgs {
  AttendArgs a;
  CUtensorMap q, k, v;
  uint32_t toks;             // tokens of a row tile
  uint32_t box;              // slots of a TMA box
  uint32_t wide;             // output rows are aligned to 32 bytes
};
struct WeighFewArgs {
  WeighArgs a;
  CUtensorMap k;
  uint32_t box, tma;
};
struct WeighTileArgs {
  WeighArgs a;
  CUtensorMap q, k;
  CUtensorMap fill;          // the heads of one token that fill up a row tile
  uint32_t toks, box;
};
struct AttendFewArgs {
  AttendArgs a;
  CUtensorMap k, v;
  uint32_t box;              // slots loaded together
  uint32_t tma;              // 0: row by row
  uint32_t cluster;          // a tile's runs are one cluster, which joins them in its shared memory
};

}  // namespace ro
