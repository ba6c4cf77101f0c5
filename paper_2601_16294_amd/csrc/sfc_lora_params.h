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
int lora_wgrad_splits(int64_t rows, int64_t cols, int rank, int adapters, int num_cus);
bool lora_by_rows(int64_t rows, int64_t cols, int rank);
int lora_down_splits(int64_t rows, int64_t cols, int rank, int num_cus);
hipError_t launch_lora_down(const LoraParams& p, bool nk, hipStream_t stream);
hipError_t launch_lora_down_tiles(const LoraParams& p, bool nk, hipStream_t stream);
hipError_t launch_lora_up(const LoraParams& p, bool nk, bool bf16, int num_cus, hipStream_t stream);
hipError_t launch_lora_wgrad(const LoraParams& p, bool nk, bool bf16, hipStream_t stream);

}  // namespace sfc
