// Internal interface between the C-ABI layer of the bf16 expert and adapter operators
// (sfc_rows_api.cpp) and their HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sfc {

// How the operands of a product lie in memory.
enum MoeLayout {
  kMoeNK = 0,                // C[p] = A[p] B[e]^T: both along K
  kMoeKN = 1,                // C[p] = A[p] B[e]: A along K, B's rows along N
  kMoeTN = 2,                // C[e] = A[segment]^T B[segment]: K runs over the rows of both
};
struct MoeGemmParams {
  int64_t M, N, K;           // kMoeTN: M x N for every expert, K rows of all of them
  const uint16_t* A;
  int64_t lda;               // elements
  const int32_t* order;      // A's row p is A[order[p] / topk] (null: row p)
  int64_t a_rows;            // rows that A has (with order)
  int topk;
  const uint16_t* B;
  int64_t ldb, stride_b;     // stride_b: from one expert's B to the next
  void* C;
  int64_t ldc, stride_c;     // stride_c between experts (kMoeTN)
  const int32_t* offsets;    // experts + 1
  int experts;
  const int32_t* table;      // curve of gm x gn blocks (kMoeTN)
  int gm, gn;
  bool past;                 // C goes past the caches
};
// Blocks of 256 x 256, one workgroup to a CU, of 128 x 128, two, or of 64 x 64, four.
hipError_t launch_moe_256x256(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream);
hipError_t launch_moe_64x64(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream);
hipError_t launch_moe_128x128(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream);
// Few rows of each expert, kMoeNK: 16 * fn rows of an expert's weights past 16 * fm of its rows (fm = fn = 1, or fm = 2 or 4
// and fn = 2).
hipError_t launch_moe_rows(const MoeGemmParams& p, int fm, int fn, bool out_bf16, hipStream_t stream);

}  // namespace sfc
