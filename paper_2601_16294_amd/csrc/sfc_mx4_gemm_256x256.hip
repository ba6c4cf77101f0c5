// 4-bit products on 256x256 blocks.
#include "sfc_mx4_kernel.h"

namespace sfc {

hipError_t launch_mx4_256x256(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream) {
  return mx4_launch<256, 256>(p, mode, out_bf16, grid, stream);
}

}  // namespace sfc
