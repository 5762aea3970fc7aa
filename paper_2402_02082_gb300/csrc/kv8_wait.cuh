// The bounded waits of the 8-bit cache's tcgen05 kernel.
#pragma once

#include "common.cuh"

namespace glide {
namespace {

// Waits of at most a second, as mbar_wait_small, in few instructions: those that a wait spins through are taken from
// the warps that work.  On giving up it sets *abort.
__device__ __noinline__ bool wait_long(uint64_t* bar, uint32_t parity, volatile int* abort) {
  const uint64_t t0 = global_timer_ns();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .u32 n;\n\t"
        "mov.u32 %0, 1;\n\tmov.u32 n, 64;\n"
        "AGAIN:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\t"
        "setp.ne.u32 p, n, 0;\n\t"
        "@p bra AGAIN;\n\t"
        "mov.u32 %0, 0;\n"
        "DONE:\n\t}"
        : "=&r"(ok)
        : "r"(smem_u32(bar)), "r"(parity), "r"(1000u)
        : "memory");
    if (ok) return true;
    if (*abort) return false;
    if (global_timer_ns() - t0 > kWaitLimitNs) {
      *abort = 1;
      return false;
    }
  }
}
// For every lane of a converged warp, with one outcome.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait_long(bar, parity, abort));
}

}  // namespace
}  // namespace glide
