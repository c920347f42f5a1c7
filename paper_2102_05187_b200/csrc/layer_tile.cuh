// What the tensor-core forms of the layer operators share: barriers with bounded waits, tensor-map copies, tcgen05 products and their
// descriptors. 16-bit operands, fp32 accumulators in tensor memory. Internal: not part of the C ABI.
#pragma once

#include <cuda.h>

#include "layer.cuh"

namespace comet {

// Every wait gives up after some seconds (`patience`, in cycles; 0: `failed` from the start): the kernel then skips the rest, waits for its products and
// copies in flight, frees its tensor memory, sets a word of the handle's pinned memory and returns. The next call of a layer operator reports it.
// (The cycle counter, not the global timer: reading that one took longer than most waits.)
constexpr int64_t kEndCycles = 4000000000ll;   // for what is in flight at the end, which nothing can hold up

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// False once a wait of this CTA has run out (then and from then on, unless the barrier is there already).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *failed, int64_t patience) {
  if (bar_try(bar, parity)) return true;
  const int64_t since = clock64();
  while (!*failed) {
    for (int i = 0; i < 64; ++i)
      if (bar_try(bar, parity)) return true;
    if (clock64() - since > patience) *failed = 1;
  }
  return false;
}
// The same for a warp whose lanes go on together.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int *failed, int64_t patience) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity, failed, patience));
}
// For what a CTA that gives up has in flight.
__device__ __forceinline__ void bar_wait_end(uint32_t bar, uint32_t parity) {
  const int64_t since = clock64();
  while (!bar_try(bar, parity) && clock64() - since < kEndCycles) {}
}

__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map),
               "r"(x), "r"(y), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_bar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D (tensor memory) = A B (+ D): 128 x N x 16 of 16-bit operands in shared memory; one thread issues it.
__device__ __forceinline__ void tc_product(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
      : "memory");
}
// The barrier is arrived at when all products issued so far by this thread are done.
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// At the end of a CTA whose waits have run out, by the thread that issued the copies, `issued` of them, one stage after the other: the last one of every
// stage lands before the shared memory is given up (the ones before it have: its stage was free), and the host is told. Nothing but the
// copies completes the barriers at `landed`.
__device__ __forceinline__ void give_up(uint32_t landed, int stages, int32_t issued, int32_t *status) {
  for (int s = 0; s < stages && s < issued; ++s) bar_wait_end(landed + 8 * s, (uint32_t)((issued - 1 - s) / stages) & 1);
  *(volatile int32_t *)status = 1;
  __threadfence_system();
}

// 16 consecutive columns of this warp's 32 rows: lane = row.
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&x)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}

// Shared-memory operand descriptors, 128-byte swizzle: start address, the distance between blocks of 64 values along the row dimension where
// that one is contiguous (`across`), the distance between groups of 8 rows (`groups`), version 1 (sm_100).
__device__ __forceinline__ uint64_t operand_at(uint32_t address, uint32_t across, uint32_t groups) {
  return (uint64_t)((address & 0x3ffff) >> 4) | (uint64_t)(across >> 4) << 16 | (uint64_t)(groups >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: fp32 accumulator, both operands bf16 or both fp16, A with k contiguous, B with k or with n contiguous.
__device__ __forceinline__ uint32_t product_kind(bool bf16, bool b_by_n, int m, int n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_by_n ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

// Map of a row-major rows x cols matrix of 16-bit values for copies of `box_rows` rows x 64 values, 128-byte swizzle, zeros
// outside. False where the driver refuses it.
bool tile_map(CUtensorMap *map, bool bf16, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows);

}  // namespace comet
