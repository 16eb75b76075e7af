// Issuing tcgen05.mma from a whole warp.  The tensor core takes its descriptors from uniform registers, and every instruction
// that moves a value there sits between two products: one product of 128 x 128 x 16 takes 64 cycles, and an issuing loop whose
// descriptors live in ordinary registers needs about 130 for each.  So the warp's control flow and addresses are kept
// uniform by construction -- values from memory pass through a warp reduction, whose result IS a uniform register, and waits
// end on a vote -- and the products of one operand pair are one block of instructions under one election.
#pragma once

#include "stief_tc.cuh"

namespace stief {
namespace tc {

// A value that all lanes hold alike, as a uniform register
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }

// mbar_wait for a converged warp whose control flow stays uniform
__device__ __forceinline__ void mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  for (uint32_t i = 0; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++i) {
    if ((i & 1023u) == 1023u && (__any_sync(0xffffffffu, *abort_flag != 0) || i >= kWaitSpins)) {
      if (i >= kWaitSpins) {
        *abort_flag = 1;
        report(status, STIEF_ERR_TIMEOUT);
      }
      return;
    }
  }
}

// After a wait that ran out: about two milliseconds, in which every copy still in flight reaches shared memory, before the
// CTA leaves it
__device__ __forceinline__ void let_copies_land() {
  const long long t0 = clock64();
  while (clock64() - t0 < (4ll << 20)) {
  }
}

// Low word of a shared-memory matrix descriptor (address and leading byte offset); the high word (stride byte offset, version,
// layout) is the same for every operand of one swizzle mode
__device__ __forceinline__ uint32_t desc_lo(uint32_t lbo_bytes, uint32_t smem_addr) { return ((lbo_bytes >> 4) << 16) | ((smem_addr & 0x3FFFFu) >> 4); }
__device__ __forceinline__ uint32_t desc_hi(uint64_t tmpl) { return (uint32_t)(tmpl >> 32); }

// One product of K = 16: D[tmem] (+)= A[smem] B[smem], issued by the warp's elected lane
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p;\n\t.reg .b64 da, db;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
      ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// the same with A in TMEM
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p;\n\t.reg .b64 db;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// One arrival at the mbarrier when every product issued so far by the elected lane has completed
__device__ __forceinline__ void umma_commit_warp(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
      : "memory");
}

}  // namespace tc
}  // namespace stief
