// Shared-memory barriers of the asynchronous copy and matrix units, with bounded waits.
#pragma once
#include <stdint.h>

namespace stand {

constexpr unsigned SPIN_LIMIT = 1u << 22;  // bounded waits: about a second, then the kernel gives up

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait; false if the limit ran out or another thread of the CTA already gave up.
__device__ __forceinline__ bool mbar_wait_bounded(uint32_t bar, uint32_t parity, const volatile int* abort_flag,
                                                  unsigned limit = SPIN_LIMIT) {
  for (unsigned spin = 0; spin < limit; ++spin) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
  }
  return false;
}
// A wait bounded by time: a poll may itself be suspended for long, so polls alone bound little.  `limit` counts units of
// 512 clock cycles (SPIN_LIMIT: about a second); 0 gives up at once.
__device__ __forceinline__ bool mbar_wait_timed(uint32_t bar, uint32_t parity, const volatile int* abort_flag, unsigned limit) {
  const long long end = clock64() + (long long)limit * 512;
  while (limit && clock64() < end) {
    if (mbar_try_wait(bar, parity)) return true;
    if (abort_flag && *abort_flag) return false;
  }
  return false;
}

}  // namespace stand
