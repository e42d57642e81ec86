// Inline-PTX wrappers of the block-scaled 8-bit products (tcgen05 kind::mxf8f6f4) and of thread-block
// pairs (cta_group::2): shared by the kernels of ham_fp8.cu and ham_experts.cu.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "ham_ptx.cuh"

namespace ham {
namespace {

// Instruction descriptor of kind::mxf8f6f4: e4m3 A and B (format code 0), E8M0 scales, fp32 D, both
// operands K-major.  Byte `sf` of a row's 32-bit scale word in tensor memory scales the product's 32
// elements of K (both operands use the same byte).
__host__ __device__ constexpr uint32_t idesc_mx(int M, int N, int sf) {
  return ((uint32_t)sf << 4) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 4) << 24) |
         ((uint32_t)sf << 29);
}
// D (TMEM) = (A 2^sa) (B 2^sb) (+ D if accumulate), K = 32, one thread (of the pair's first CTA for
// kCtas = 2).  sfa / sfb: TMEM columns of the scale words: row r of the operand in lane r % 32 of
// every lane quarter, column r / 32.
template <int kCtas>
__device__ __forceinline__ void tc_mma_mx(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                          uint32_t idesc, uint32_t sfa, uint32_t sfb, bool accumulate) {
  if constexpr (kCtas == 1)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
        : "memory");
}
// 512 bytes of shared memory (32 rows of 16 bytes, 8-row groups 128 bytes apart) -> four TMEM columns,
// the 32 rows copied to every lane quarter (of both CTAs for kCtas = 2, each from its own shared
// memory).  In order with the products the same thread issues.
template <int kCtas>
__device__ __forceinline__ void tc_copy_scales_of(uint32_t tmem, uint64_t desc) {
  if constexpr (kCtas == 1)
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint32_t smem_addr) {
  tc_copy_scales_of<kCtas>(tmem, smem_desc_plain(smem_addr, 0, 128));
}

// ---- pairs of CTAs (cta_group::2) ----------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
template <uint32_t kCols>
__device__ __forceinline__ void tmem_alloc_pair(uint32_t *slot) {  // one warp of each CTA
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_u32(slot)),
               "n"(kCols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
template <uint32_t kCols>
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "n"(kCols)
               : "memory");
}
__device__ __forceinline__ void tmem_alloc_n(uint32_t *slot, uint32_t cols) {  // whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_u32(slot)),
               "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_n(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols)
               : "memory");
}
// The barrier at the same place in every CTA of `mask` (a bit a cluster rank) receives one arrival once
// every tcgen05 operation that this thread issued so far is complete.
__device__ __forceinline__ void tc_commit_pair(uint64_t *bar, uint32_t mask) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"((uint16_t)mask)
      : "memory");
}
// Arrive on a barrier of a CTA of the cluster (a shared::cluster address).  With `release` at cluster
// scope the thread's earlier writes are ordered before it, which costs a round trip to L2 (about a
// microsecond under load).  Without, it orders execution alone: enough for tensor-memory operations
// behind tcgen05.fence::before_thread_sync.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ bool mbar_test_cluster(uint64_t *bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// The whole warp waits on a phase whose arrivals come from both CTAs, bounded (2 s); warp-uniform.
__device__ __forceinline__ bool warp_wait_cluster(uint64_t *bar, uint32_t parity,
                                                  volatile int *abort_flag) {
  uint64_t t0 = 0;
#pragma unroll 1
  for (uint32_t n = 0;; ++n) {
    if (__all_sync(kFull, mbar_test_cluster(bar, parity))) return true;
    if (n == 0) t0 = global_timer_ns();
    else if ((n & 15u) == 0 &&
             __any_sync(kFull, *abort_flag != 0 || global_timer_ns() - t0 > kWaitLimitNs))
      return false;
  }
}
// The same by one thread.
__device__ __forceinline__ bool thread_wait_cluster(uint64_t *bar, uint32_t parity, volatile int *abort_flag) {
  if (mbar_test_cluster(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
#pragma unroll 1
  for (uint32_t n = 1; !mbar_test_cluster(bar, parity); ++n)
    if ((n & 15u) == 0 && (*abort_flag != 0 || global_timer_ns() - t0 > kWaitLimitNs)) return false;
  return true;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t a, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
// Rank-2 tiled TMA copy into this CTA's shared memory whose bytes count at a barrier of the pair's
// first CTA (`bar`: its shared::cluster address).
__device__ __forceinline__ void tma_load_2d_pair(void *dst, const CUtensorMap *map, int x, int y,
                                                 uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar), "l"(policy)
      : "memory");
}

// Four rows (r) of the map's matrix, 128 bytes of each from column x on, one after another into this CTA's shared memory
// (the map's box is one row high); their bytes count at a barrier of the pair's first CTA.
__device__ __forceinline__ void tma_gather4_pair(void *dst, const CUtensorMap *map, int x, const int4 &r, uint32_t bar,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(bar), "l"(policy)
      : "memory");
}

// Registers of this warpgroup's threads from here on (all four warps).
template <int kRegs>
__device__ __forceinline__ void setmaxnreg_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void setmaxnreg_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
// 32 bytes to global memory (32-byte aligned): a whole sector a thread.
__device__ __forceinline__ void st_global_32(void *p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// A barrier of `threads` threads that also tells whether `ok` held in all of them.
__device__ __forceinline__ bool named_barrier_and(int id, int threads, bool ok) {
  uint32_t all;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %3, 0;\n bar.red.and.pred q, %1, %2, p;\n"
      " selp.u32 %0, 1, 0, q;\n}"
      : "=r"(all)
      : "r"(id), "r"(threads), "r"((uint32_t)ok)
      : "memory");
  return all != 0;
}
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

}  // namespace
}  // namespace ham
