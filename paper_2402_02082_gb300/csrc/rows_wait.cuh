// The bounded waits of the attention of packed rows.
#pragma once

#include "common.cuh"

namespace glide {
namespace {

// What a CTA's waits look at, in shared memory: the abort flag, and the time (globaltimer's low word) at which they give up.
struct __align__(8) Watch {
  int abort;
  uint32_t deadline;
};

// The waits have limit_ns from now on.  One thread, at every step of the work that the others may wait for: an item, and 32 keys of a
// row that is computed again by the definition, which takes as long as it takes (seconds for 32 rows of a million keys) and ends by itself.
__device__ __forceinline__ void put_off(Watch* watch, uint32_t limit_ns = (uint32_t)kWaitLimitNs) {
  uint32_t now;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(now));
  *reinterpret_cast<volatile uint32_t*>(&watch->deadline) = now + limit_ns;
}

// As mbar_wait_small, but with the CTA's deadline for the wait's own limit (and no more code than that has: the kernel has some twenty
// waits, and five instructions more in each cost 2 to 4% of a call).  The difference of times is signed, so deadlines may be 2 s off.
__device__ __forceinline__ bool wait_watched(uint64_t* bar, uint32_t parity, Watch* watch) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .u32 t0, t1;\n\t"
      "mov.u32 %0, 1;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n"
      "AGAIN:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n\t"
      "ld.volatile.shared.v2.u32 {t1, t0}, [%3];\n\t"
      "setp.ne.u32 p, t1, 0;\n\t"
      "@p bra GIVEUP;\n\t"
      "mov.u32 t1, %%globaltimer_lo;\n\t"
      "sub.u32 t1, t1, t0;\n\t"
      "setp.lt.s32 p, t1, 0;\n\t"
      "@p bra AGAIN;\n"
      "GIVEUP:\n\t"
      "st.volatile.shared.u32 [%3], 1;\n\t"
      "mov.u32 %0, 0;\n"
      "DONE:\n\t}"
      : "=&r"(ok)
      : "r"(smem_u32(bar)), "r"(parity), "r"(smem_u32(watch))
      : "memory");
  return ok != 0;
}
// For every lane of a converged warp, with one outcome.
__device__ __forceinline__ bool warp_wait_watched(uint64_t* bar, uint32_t parity, Watch* watch) {
  return __all_sync(0xffffffffu, wait_watched(bar, parity, watch));
}

}  // namespace
}  // namespace glide
