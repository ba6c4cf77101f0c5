// Experts' bf16 products on 64x64 blocks, four workgroups to a CU.
#include "sfc_moe_gemm_kernel.h"

namespace sfc {

hipError_t launch_moe_64x64(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream) {
  return moe_launch<64, 64>(p, layout, out_bf16, grid, stream);
}

}  // namespace sfc
