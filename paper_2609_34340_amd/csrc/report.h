// Device errors of the layer operators.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace vp {
namespace {

// The first error of calls that were given no status since it was last taken; a word for each source file that
// includes this, on each device, there from the start (no allocation, also while a graph is captured).
__device__ int32_t unclaimed = 0;

__device__ inline void report(int32_t* status, int32_t code) { atomicCAS(status ? status : &unclaimed, 0, code); }

__global__ void take_unclaimed_kernel(int32_t* out) {
  const int32_t code = atomicExch(&unclaimed, 0);
  if (code != 0) atomicCAS(out, 0, code);
}

}  // namespace
}  // namespace vp
