// Kernel launches whose result is their own: hipGetLastError() would also report what an earlier
// call of the program left behind.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace sfc {

template <class... P>
inline hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t stream,
                                std::type_identity_t<P>... args) {
  void* list[] = {&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, list, lds, stream);
}

}  // namespace sfc
