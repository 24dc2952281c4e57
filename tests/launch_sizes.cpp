// fake_hip.cpp with the bound of a launch: grid times block below 2^32 in every
// dimension, or the launch is refused.  The log's entries are "<kernel> <workgroups in x>".
#define hipLaunchKernel fake_launch
#define hipGetLastError fake_last_error
#include "fake_hip.cpp"
#undef hipLaunchKernel
#undef hipGetLastError

static hipError_t last = hipSuccess;

extern "C" {

hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  const bool fits = (uint64_t)grid.x * block.x >> 32 == 0 && (uint64_t)grid.y * block.y >> 32 == 0 &&
                    (uint64_t)grid.z * block.z >> 32 == 0 && grid.x && grid.y && grid.z;
  last = fits ? hipSuccess : hipErrorInvalidConfiguration;
  if (fits) text += names[f] + " " + std::to_string(grid.x) + "\n";
  return last;
}
hipError_t hipGetLastError() {
  const hipError_t e = last;
  last = hipSuccess;
  return e;
}
}
