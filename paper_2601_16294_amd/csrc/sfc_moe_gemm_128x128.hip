// Experts' bf16 products on 128x128 blocks, two workgroups to a CU.
#include "sfc_moe_gemm_kernel.h"

namespace sfc {

hipError_t launch_moe_128x128(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream) {
  return moe_launch<128, 128>(p, layout, out_bf16, grid, stream);
}

}  // namespace sfc
