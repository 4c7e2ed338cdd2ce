// Launches where kernels are host code, in place of the library's header of
// the same name: at once, on a grid that the GPU's dispatch would take.
#pragma once

#include <hip/hip_runtime.h>

namespace host_hip {
inline bool only_grids = false;  // check launches' grids, and run nothing
}

namespace adst {
namespace {

template <class P>
struct AsIs {
  typedef P type;
};

template <class... P>
hipError_t start(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t,
                 const typename AsIs<P>::type&... args) {
  if (grid.x == 0 || grid.y == 0 || grid.z == 0 || (uint64_t)grid.x * threads >> 32 ||
      grid.y >> 16 || grid.z >> 16)
    return hipErrorInvalidValue;
  if (!host_hip::only_grids) host_hip::launch(grid, dim3(threads), [=] { kernel(args...); });
  return hipSuccess;
}

}  // namespace
}  // namespace adst
