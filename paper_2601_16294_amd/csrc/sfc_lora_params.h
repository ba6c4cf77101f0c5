// Internal interface between the C-ABI layer of the low-rank adapters (sfc_rows_api.cpp) and
// their HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sfc {

constexpr int kMaxRank = 256;

struct LoraParams {
  int64_t rows;
  int64_t cols;              // down: K; up: N; gradient: columns of Z
  int rank, adapters;
  int first_adapter;         // gradient: of this launch
  const int32_t* ids;        // adapter of every row; one outside 0 .. adapters-1: none
  // down: rows x cols; gradient: Z, rows x cols
  const uint16_t* X;
  int64_t ldx;
  // down: A, rank x cols (nk) or cols x rank; up: B, cols x rank (nk) or rank x cols
  const uint16_t* W;
  int64_t ldw, stride_w;
  const float* scales;       // down: per adapter, or null
  float* V;                  // rows x rank: written by down, else read
  int64_t ldv;
  // up: base and Y, rows x cols (base may be null, or Y); gradient: cols x rank (nk) or rank x cols
  const void* base;
  int64_t ld_base;
  void* Y;
  int64_t ldy, stride_y;     // stride_y: gradient, between adapters
  // down: ranges of K, their sums (splits > 1) [splits][rows][rank].  gradient: parts of the rows that are
  // dealt out over the adapters (splits > 1), the sums of those that are not alone, each as G, and for every
  // adapter the first of its parts among them and their number; this launch's first column
  int splits;
  float* sums;
  int32_t* parts;
  int64_t all_cols, first_col;
};
constexpr int kDownTile = 64;                            // rows and ranks of a tile of down
constexpr int kGradWaves = 4, kGradColumns = 64 * kGradWaves;
constexpr int kGradAdapters = 1024;                      // most adapters whose rows are dealt out in parts

// Whether rows are taken one by one, each reading its adapter's weights (from the L2 for the most part).  That takes
// about the same time in any order of the rows; the tiles are faster where rows come in runs and slower where they do not,
// which the host does not know (us of up, bf16, one by one / tiles of 8 runs / tiles of 32 adapters at random: 64 rows x
// 14336, rank 64 15 / 23 / 85; 256 x 14336, rank 16 14 / 7 / 41; 512 x 4096, rank 16 9 / 5 / 39; 2048 x 4096, rank 64 107 /
// 11 / 102).  Up to 256 rows may be a decode step, a request each; more are taken for prompts.
inline bool lora_by_rows(int64_t rows, int64_t cols, int rank) {
  return rows <= 4096 && rows * rank * cols <= (int64_t)(rows <= 64 ? 256 : rows <= 256 ? 128 : 32) << 20;
}

// Row by row, weights N x K: ranks of a wave in down.  One while that takes few waves, else 4, which read X once (us, K = 4096, 1 / 4:
// 16 rows, rank 16 3.7 / 4.9, 128 rows 4.3 / 5.0, 256 rows 5.2 / 5.3, 128 rows, rank 64 7.2 / 6.5).
inline int lora_row_ranks(int64_t rows, int rank) { return rows * rank <= 2048 ? 1 : 4; }
// Lanes of 8 ranks each that share a row of the weights, up to `most`.
inline int lora_row_lanes(int rank, int most) {
  int lanes = 1;
  while (lanes < most && 8 * lanes < rank) lanes *= 2;
  return lanes;
}

// Up in tiles: chunks of 32 ranks that a kernel holds.
constexpr int lora_up_chunks(int rank) { return rank <= 32 ? 1 : rank <= 64 ? 2 : rank <= 128 ? 4 : 8; }
// Columns of a workgroup.  Wide blocks read V least often, narrow ones take fewer
// registers (us at 64 / 128 / 256 columns: bf16 4096x14336 rank 64 70 / 55 / 53, 8192x4096 rank 16 27 / 25 / 26, fp32
// 1003x5003 rank 12 14 / 14 / 22, bf16 4096x4096 rank 128 35 / 25 / 27).  Ranks over 128: 64 hold all of their ranks in
// registers; 128 spill up to 46 with fp32 results and leave small batches few workgroups, but large ones would gain (rank 256, 64 /
// 128: 600x520 15 / 19, fp32 1000x14336 69 / 81, bf16 4096x4096 54 / 38).
constexpr int lora_up_columns(int chunks, bool bf16) { return chunks == 2 && bf16 ? 256 : chunks <= 4 ? 128 : 64; }
// Tiles of 16 rows of each of a workgroup's 4 waves.  256 rows to a workgroup read the weights least often; 64 where there would
// be few workgroups (us, bf16, 8 runs, 64 / 256: 1024 rows x 4096, rank 64 7.4 / 16.4, 2048 11.5 / 17.2, 4096 21.1 / 20.7; 4096 x
// 14336 57 / 50; 8192 x 4096, rank 16 27 / 25; 4096 x 4096, rank 256 70 / 55).
inline int lora_up_tiles(int64_t rows, int64_t cols, int rank, bool bf16, int num_cus) {
  const int columns = lora_up_columns(lora_up_chunks(rank), bf16);
  return (cols + columns - 1) / columns * ((rows + 255) / 256) >= 2 * num_cus ? 4 : 1;
}

// Weight gradient: rows of Z or V of fewer than 8 elements, which are loaded one by one; ranks of a workgroup, in 16.
inline bool lora_grad_narrow(int64_t cols, int rank) { return cols < 8 || rank < 8; }
inline int lora_grad_ranks(int64_t cols, int rank) { return lora_grad_narrow(cols, rank) ? 1 : rank <= 64 ? (rank + 15) / 16 : 4; }

// Ranges of K in the tiles of down.
inline int lora_down_splits(int64_t rows, int64_t cols, int rank, int num_cus) {
  if (lora_by_rows(rows, cols, rank)) return 1;
  // a workgroup to a CU, or 4 ranges while that is two to a CU at most, each of 4 stages at least (us with 1 / 2 / 4 / 8
  // ranges of K = 4096: 4096 rows, rank 64 35 / 25 / 20 / 28; 8192, rank 16, K x rank 31 / 24 / 22 / 31; 16384, rank 64 38 /
  // 44 / 52 / 69)
  const int64_t tiles = (rows + kDownTile - 1) / kDownTile * ((rank + kDownTile - 1) / kDownTile), stages = (cols + 63) / 64;
  int64_t splits = num_cus / tiles > 4 ? num_cus / tiles : 4;
  if (splits > 2 * num_cus / tiles) splits = 2 * num_cus / tiles;
  if (splits > stages / 4) splits = stages / 4;
  return splits < 1 ? 1 : splits > 16 ? 16 : (int)splits;
}

// Parts of the rows that the weight gradient deals out over the adapters.
inline int lora_wgrad_splits(int64_t rows, int64_t cols, int rank, int adapters, int num_cus) {
  if (adapters > kGradAdapters) return 1;
  // parts of the rows, so that all workgroups, two to a CU, are in flight at once; each of 4 chunks at least (8
  // where there are few: a sum takes longer than 8 chunks).  Their sums are written and read back: 16 MB at
  // most.  (2^22: one launch.)
  const int fr = lora_grad_ranks(cols, rank);
  const int64_t groups = (cols + kGradColumns - 1) / kGradColumns * ((rank + 16 * fr - 1) / (16 * fr));
  const int64_t chunks = (rows + 31) / 32, each = cols * rank;
  if (each < 1 || groups * (adapters + 32) > (int64_t)1 << 22) return 1;
  int64_t splits = 2 * (int64_t)num_cus / groups - adapters;
  if (splits < num_cus / groups) splits = num_cus / groups;
  const int64_t most = chunks >= 32 ? chunks / 4 : chunks / 8;
  if (splits > most) splits = most;
  if (splits > 32) splits = 32;
  if (splits > ((int64_t)4 << 20) / each) splits = ((int64_t)4 << 20) / each;
  return splits < 2 ? 1 : (int)splits;
}

hipError_t launch_lora_down(const LoraParams& p, bool nk, hipStream_t stream);
hipError_t launch_lora_down_tiles(const LoraParams& p, bool nk, hipStream_t stream);
hipError_t launch_lora_up(const LoraParams& p, bool nk, bool bf16, int num_cus, hipStream_t stream);
hipError_t launch_lora_wgrad(const LoraParams& p, bool nk, bool bf16, hipStream_t stream);

}  // namespace sfc
