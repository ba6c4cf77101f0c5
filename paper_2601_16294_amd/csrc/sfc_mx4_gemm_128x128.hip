// 4-bit products on 128x128 blocks, two workgroups to a CU.
#include "sfc_mx4_kernel.h"

namespace sfc {

hipError_t launch_mx4_128x128(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream) {
  return out_bf16 ? mx4_launch<128, 128, true>(p, mode, grid, stream) : mx4_launch<128, 128, false>(p, mode, grid, stream);
}

}  // namespace sfc
