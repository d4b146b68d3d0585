// flr_launch.h -- a kernel launch that returns its own status.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

namespace flr {

// Enqueues a kernel.  The status is this launch's own: an error that an earlier call
// of the runtime left behind is not this one's, and stays for who asks for it.
template <typename T>
struct Same {
  using type = T;
};
template <typename... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t lds, hipStream_t st,
                  typename Same<P>::type... args) {
  void* at[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, lds, st);
}

}  // namespace flr
