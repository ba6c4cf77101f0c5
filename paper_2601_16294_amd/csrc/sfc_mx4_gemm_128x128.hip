// 4-bit products on 128x128 blocks, two workgroups to a CU.
#include "sfc_mx4_kernel.h"

namespace sfc {

hipError_t launch_mx4_128x128(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream) {
  return mx4_launch<128, 128>(p, mode, out_bf16, grid, stream);
}

}  // namespace sfc
