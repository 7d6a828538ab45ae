// 5th-generation tensor core instructions (sm_100a `tcgen05.*`), tiled copies (`cp.async.bulk.tensor`) and what joins
// them: thin wrappers around the PTX instructions, written from the PTX ISA.
//
// CTAS is the `cta_group`: 1, or 2 for a pair of CTAs (a cluster of two) that work on one tile with twice the rows and
// twice the columns, each CTA holding half of both operands and half of the accumulator's rows.
//
// Operand tiles in shared memory are 128 rows x 64 bf16 as two boxes of 64 x 64 elements, 128-byte swizzled, whichever
// of the two axes is contiguous in global memory:
//   K-major   (the summed axis contiguous): rows of 128 bytes, groups of 8 rows 1024 bytes apart.
//   MN-major  (the other axis contiguous): every box holds 64 values of k, each a row of 64 consecutive outer indices;
//             groups of 8 k's 1024 bytes apart, boxes (64 outer indices) 8192 bytes apart.
#pragma once
#include <cuda.h>

#include "hdet_bulk.cuh"

namespace hdet {
namespace umma {

constexpr int kTileRows = 128;                               // rows of one CTA's operand tile
constexpr int kBlockK = 64;                                  // summed indices per stage
constexpr int kBoxBytes = 64 * 64 * 2;                       // one 64 x 64 box of bf16
constexpr int kOperandBytes = 2 * kBoxBytes;                 // 128 x 64

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared address of the same variable in the cluster's CTA 0.
__device__ __forceinline__ uint32_t in_leader(uint32_t smem) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem));
  return r;
}

// Shared address of the same variable in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t in_cta(uint32_t smem, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem), "r"(rank));
  return r;
}

// A store to, and an arrival at, shared memory of any CTA of the cluster (addresses from in_cta); the arrival releases what
// this thread wrote before it to threads that wait with wait_cluster.
__device__ __forceinline__ void store_cluster(uint32_t at, int value) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(value) : "memory");
}

__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// bulk::barrier_wait for arrivals from anywhere in the cluster; as bounded as that.
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, long long limit_cycles = bulk::kWaitLimitCycles) {
  if (try_wait_cluster(bar, parity)) return true;
  const long long start = clock64();
  for (;;) {
    for (int i = 0; i < 32; ++i)
      if (try_wait_cluster(bar, parity)) return true;
    if (clock64() - start > limit_cycles) return false;
  }
}

// The instructions below are issued by one lane, which `elect.sync` picks, while the whole warp runs the loop around them with
// the same values in every lane: their operands live in registers that the warp shares.  In a loop that one lane runs alone,
// every operand is moved there first, and the loop of the products took longer than the tensor cores need (282 us instead
// of 263 for 2048 x 50176 logits of width 2048).

// One 64 x 64 box into this CTA's shared memory; completion counted in bytes on `bar` (in the leader's CTA for a pair).
// Coordinates: x in elements along the contiguous axis (a multiple of 64 here, so 16-byte aligned), y, z.  Whole warp.
template <int CTAS>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (CTAS == 1) {
    asm volatile(
        "{\n .reg .pred q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n"
        " @q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  } else {
    asm volatile(
        "{\n .reg .pred q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n"
        " @q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];\n}" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  }
}

// bulk::barrier_expect by one lane.
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n .reg .pred q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}" ::"r"(bar),
      "r"(bytes)
      : "memory");
}

// bulk::barrier_wait by a whole warp, with one answer for all of its lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, long long limit_cycles = bulk::kWaitLimitCycles) {
  if (__all_sync(0xffffffffu, bulk::barrier_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, bulk::barrier_wait(bar, parity, limit_cycles));
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Tensor memory: `columns` columns x 128 lanes of 32 bits.  Whole warp; for a pair, one warp of each CTA.
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, int columns) {
  if constexpr (CTAS == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}

template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t tmem, int columns) {
  if constexpr (CTAS == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}

__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory descriptor of an operand tile: start address, leading and stride byte offsets (all in units of 16
// bytes), descriptor version 1, 128-byte swizzle.
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem, bool mn_major) {
  const uint64_t leading = mn_major ? kBoxBytes >> 4 : 1;    // not used by swizzled K-major tiles
  return (uint64_t)((smem >> 4) & 0x3FFF) | (leading << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// Bytes from one group of 16 summed indices to the next inside a stage.
__device__ __forceinline__ uint32_t k_step_bytes(bool mn_major) { return mn_major ? 2048 : 32; }

// Instruction descriptor: bf16 x bf16 -> fp32, (128 * CTAS) x columns x 16.
template <int CTAS>
__device__ __forceinline__ uint32_t instruction_desc(int columns, bool a_mn_major, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn_major << 15) | ((uint32_t)b_mn_major << 16) |
         ((uint32_t)(columns / 8) << 17) | ((uint32_t)(128 * CTAS / 16) << 24);
}

// D (+)= A B^T for 16 summed indices.  Whole warp (of the leader's CTA).
template <int CTAS>
__device__ __forceinline__ void mma(uint32_t tmem, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if constexpr (CTAS == 1) {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  } else {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
        " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  }
}

// Arrives on `bar` once everything that this warp's lane has issued to the tensor core is done; for a pair, on the barrier at
// the same place in both CTAs.  Whole warp.
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (CTAS == 1) {
    asm volatile(
        "{\n .reg .pred q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n"
        " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar)
        : "memory");
  } else {
    asm volatile(
        "{\n .reg .pred q;\n .reg .b32 r;\n elect.sync r|q, 0xffffffff;\n"
        " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
  }
}

// 32 consecutive columns of this warp's 32 lanes (lane i of the warp holds row 32 * (warp % 4) + i).
__device__ __forceinline__ void tmem_load32(uint32_t tmem, float (&x)[32]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]),
        "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]),
        "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(tmem));
}

// Waits for this thread's loads from tensor memory; x goes through it so that no use of x moves ahead of the wait.
__device__ __forceinline__ void tmem_load_wait(float (&x)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
        "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]),
        "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]),
        "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31])
      :
      : "memory");
}

// The same for 16 columns, and the wait for them.
__device__ __forceinline__ void tmem_load16(uint32_t tmem, float (&x)[16]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(tmem));
}

__device__ __forceinline__ void tmem_load_wait(float (&x)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
        "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15])
      :
      : "memory");
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace umma
}  // namespace hdet
