// Launches of the sequence operators' kernels.
#pragma once

#include <hip/hip_runtime.h>

namespace adst {
namespace {

template <class P>
struct AsIs {
  typedef P type;
};

// kernel(args...) on a grid of workgroups of `threads`. Returns the launch's own
// status: hipGetLastError after a launch would also report, and clear, an error
// that an earlier HIP call of the caller's thread left.
template <class... P>
hipError_t start(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t st,
                 const typename AsIs<P>::type&... args) {
  void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  const hipError_t e =
      hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, st);
  if (e != hipSuccess) (void)hipGetLastError();  // it is reported once, from here
  return e;
}

}  // namespace
}  // namespace adst
