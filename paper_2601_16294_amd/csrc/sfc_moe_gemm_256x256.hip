// Experts' bf16 products on 256x256 blocks.
#include "sfc_moe_gemm_kernel.h"

namespace sfc {

hipError_t launch_moe_256x256(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream) {
  return moe_launch<256, 256>(p, layout, out_bf16, grid, stream);
}

}  // namespace sfc
