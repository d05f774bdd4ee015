// Workgroups and the lists of work that they share out.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hinm {

// Workgroups go to the eight XCDs in turn: each XCD takes a contiguous run of a list of `items`, so that neighbours in the
// list share operands in its L2.  -1: nothing left for this workgroup.
__device__ __forceinline__ int item_of(int workgroup, int workgroups, int items) {
  const int per = workgroups >> 3;
  const int item = (workgroup & 7) * per + (workgroup >> 3);
  return item < items ? item : -1;
}
__device__ __forceinline__ int item_of_workgroup(int items) { return item_of(blockIdx.x, gridDim.x, items); }
inline uint32_t grid_of_items(int64_t items) { return (uint32_t)((items + 7) / 8 * 8); }

}  // namespace hinm
