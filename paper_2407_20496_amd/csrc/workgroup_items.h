// Workgroups and the lists of work that they share out.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hinm {

// Workgroups go to the eight XCDs in turn: each XCD takes a contiguous run of a list of `items`, so that neighbours in the
// list share operands in its L2.  -1: nothing left for this workgroup.
__device__ __forceinline__ int item_of_workgroup(int items) {
  const int per = gridDim.x >> 3;
  const int item = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  return item < items ? item : -1;
}
inline uint32_t grid_of_items(int64_t items) { return (uint32_t)((items + 7) / 8 * 8); }

}  // namespace hinm
