// LDS reads that stay in flight across other instructions, and loops whose counters are constants.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mfma_types.h"

namespace hinm {

// LDS reads as raw instructions, not waited for here: the compiler would hold every one until all copies in flight had
// landed.  To it an output is written at once, so it has to stay in its register until `pin`: lds_reads.py looks at the built
// code and the build fails where anything touches such a register before the wait.
template <int OFFSET>
__device__ __forceinline__ void lds_read_b128(uint32_t addr, u32x4& r) {
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(r) : "v"(addr), "n"(OFFSET));
}
template <int OFFSET>
__device__ __forceinline__ void lds_read_tr16(uint32_t addr, uint64_t& r) {
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=&v"(r) : "v"(addr), "n"(OFFSET));
}
// No use of the register is moved before this point.
template <class T>
__device__ __forceinline__ void pin(T& r) {
  asm volatile("" : "+v"(r));
}

template <int I, int N, class F>
__device__ __forceinline__ void unroll(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unroll<I + 1, N>(f);
  }
}

}  // namespace hinm
