// Internal interface between the C-ABI layer of the 4-bit and expert operators
// (sfc_ops_api.cpp) and their HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sfc {

constexpr int kMxBlock = 32;         // values that share one scale
constexpr int kMaxExperts = 1024;

// A launch has less than 2^32 threads.  The row kernels take at most 256 of them for a row, the
// gradient of combine also 256 for 16 rows to clear, quantisation along the columns 512 for
// 256 rows x 128 columns (256 for 128 rows): longer matrices are dealt to several launches.
constexpr int64_t kLaunchRows = (int64_t)1 << 23;
constexpr int64_t kLaunchBlocks = (int64_t)1 << 22;

// Quantisation of X, or of its rows X[order[p] / topk] (order != nullptr).
struct Mx4QuantParams {
  int64_t rows;              // rows to quantise (entries of `order`, or rows of X)
  int64_t cols;
  const void* X;
  int64_t ldx;               // elements
  const int32_t* order;
  int64_t x_rows;            // rows that X has
  int topk;
  uint8_t *Q, *S;            // blocks along columns: [rows][ceil(cols/32)*16], [rows][ceil(cols/32)]
  int64_t ldq, lds;
  uint8_t *Qt, *St;          // blocks along rows, transposed: [cols][ceil(rows/32)*16], [cols][ceil(rows/32)]
  int64_t ldqt, ldst;
};
// Q and S, and / or Qt and St (those that are not null).
hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool in_bf16, int num_cus, hipStream_t stream);

struct Mx4DequantParams {
  int64_t rows, cols;
  const uint8_t *Q, *S;
  int64_t ldq, lds;
  void* Y;
  int64_t ldy;
};
hipError_t launch_mx4_dequant(const Mx4DequantParams& p, bool out_bf16, int num_cus, hipStream_t stream);

// Product of 4-bit operands, C = A B^T.
enum Mx4Mode {
  kMxDense = 0,              // C[M][N] = A[M][K] B[N][K]^T
  kMxRows = 1,               // rows offsets[e] .. offsets[e+1]-1 of A times B[e]^T; rows past the last segment: 0
  kMxDepth = 2,              // C[e] = A[:, offsets[e] .. offsets[e+1]-1] B[:, the same]^T
};
struct Mx4GemmParams {
  int64_t M, N, K;           // kMxDepth: K values in a row of A and B, of all experts together
  const uint8_t *A, *As, *B, *Bs;
  int64_t lda, ldas, ldb, ldbs;        // bytes
  int64_t stride_b, stride_bs;         // bytes from one expert's B to the next (kMxRows)
  void* C;
  int64_t ldc, stride_c;     // elements; stride_c between experts (kMxDepth) or layer copies
  const int32_t* table;      // curve of gm x gn blocks (kMxDense, kMxDepth)
  int gm, gn;
  int experts;
  const int32_t* offsets;    // experts + 1
  int layers;                // kMxDense: ranges of K, each with a copy of C
  bool past;                 // C goes past the caches
  // launch_mx4_few: A as fp32 or bf16 rows (X, ldx elements, x_cols of them in a row), brought
  // to 4 bits on the way in
  const void* X;
  int64_t ldx, x_cols;
};
enum Mx4Rows { kRowsCodes = 0, kRowsBf16 = 1, kRowsF32 = 2 };    // what A is
// Blocks of 256 x 256, one workgroup to a CU, or of 128 x 128, two.
hipError_t launch_mx4_256x256(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream);
hipError_t launch_mx4_128x128(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream);

// Few rows of A, or of each expert: a workgroup streams 32 rows of B (`narrow`, fm = 1: 16) past
// 16 * fm rows of A at a time (fm = 1, 2, 4).
hipError_t launch_mx4_rows(const Mx4GemmParams& p, Mx4Mode mode, int fm, bool narrow, bool out_bf16, hipStream_t stream);
// Up to 16 rows of A, given as `rows` says, and K up to kFewDepth (kConvertDepth for rows that
// are not codes); dense products.
constexpr int64_t kFewDepth = 32 * 512, kConvertDepth = 8 * 512;
hipError_t launch_mx4_few(const Mx4GemmParams& p, Mx4Rows rows, int num_cus, bool out_bf16, hipStream_t stream);

// Slots sorted by expert.
struct MoeSortParams {
  int64_t slots;
  int experts, align;
  const int32_t* ids;
  int64_t rows;              // entries of `order`
  int32_t *offsets, *order, *pos;
  int32_t* counts;           // [chunks (+ 1: sums, past kSortScan)][experts] (more than one chunk)
};
constexpr int kSortChunk = 4096;     // slots that one workgroup ranks
constexpr int kSortScan = 128;       // chunks up to which every workgroup of the sort adds up the counts itself
hipError_t launch_moe_sort(const MoeSortParams& p, hipStream_t stream);

struct MoeRowsParams {
  int64_t tokens, rows, cols;          // tokens, sorted rows, columns
  int topk;
  const void* X;             // dispatch: tokens x cols; combine: rows x cols; gradient: dy, tokens x cols
  int64_t ldx;
  const void* Ys;            // gradient: the experts' rows, rows x cols
  int64_t ldys;
  const int32_t *order, *pos;
  const float* weights;      // per slot, or null: 1
  void* Y;                   // dispatch: rows x cols; combine: tokens x cols; gradient: rows x cols
  int64_t ldy;
  float* dW;                 // gradient: per slot
  // gradient: the tokens and the rows to clear of this launch, first .. end - 1
  int64_t first_token, end_token, first_row, end_row;
};
hipError_t launch_moe_dispatch(const MoeRowsParams& p, bool bf16, int num_cus, hipStream_t stream);
hipError_t launch_moe_combine(const MoeRowsParams& p, bool bf16, int num_cus, hipStream_t stream);
hipError_t launch_moe_combine_grad(const MoeRowsParams& p, bool bf16, int num_cus, hipStream_t stream);

}  // namespace sfc
