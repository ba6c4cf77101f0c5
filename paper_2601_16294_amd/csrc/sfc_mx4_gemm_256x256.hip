// 4-bit products on 256x256 blocks.
#include "sfc_mx4_kernel.h"

namespace sfc {

hipError_t launch_mx4_256x256(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream) {
  return out_bf16 ? mx4_launch<256, 256, true>(p, mode, grid, stream) : mx4_launch<256, 256, false>(p, mode, grid, stream);
}

}  // namespace sfc
