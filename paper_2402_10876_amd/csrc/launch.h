// Internal: kernel launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace twg {

template <class T> struct same_type { typedef T type; };

// One launch call of the runtime and its own status, where the <<< >>> form pushes and pops a configuration and asks
// for the thread's last error in front and behind (2.70 -> 2.46 us of the host per launch, which is what bounds small
// products).  A failed launch leaves no error behind for the next caller.  A dimension of 2^32 threads and more, which the runtime
// refuses as it does a failure of its own, is told apart: hipErrorInvalidValue, the launchers' word for a size they do not have.
template <class... P>
inline hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, typename same_type<P>::type... args) {
  if ((uint64_t)grid.x * block.x > 0xffffffffull) return hipErrorInvalidValue;
  void* list[] = {(void*)&args...};
  const hipError_t e = hipLaunchKernel((const void*)kernel, grid, block, list, 0, stream);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

}  // namespace twg
