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
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
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
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- host: tensor maps -----------------------------------------------------------------------
// 64-column blocks with the 128-byte swizzle; false: the tensor cannot be mapped
bool tile_map(CUtensorMap* m, int dtype, const void* p, int dims, const uint64_t* size, const uint64_t* stride,
              const uint32_t* box);
// a cache's pool, boxes of `box` slots of one page and head
bool pool_map(CUtensorMap* m, const PagedArgs& c, const void* pool, int dtype, uint32_t box);

struct AttendTileArgs {
  AttendArgs a;
  CUtensorMap q, k, v;
  uint32_t toks;             // tokens of a row tile
  uint32_t box;              // slots of a TMA box
};
struct AttendFewArgs {
  AttendArgs a;
  CUtensorMap k, v;
  uint32_t box;              // slots loaded together
  uint32_t tma;              // 0: row by row
};

}  // namespace ro
