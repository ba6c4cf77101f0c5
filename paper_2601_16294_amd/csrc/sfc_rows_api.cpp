// C ABI of the bf16 operators whose weights depend on the row (declarations and contracts in
// include/sfcgemm.h): argument checks, the choice of kernel and launches.  No entry point
// synchronises the device or a stream.
#include <hip/hip_runtime.h>

#include <mutex>

#include "sfc_host.h"
#include "sfc_lora_params.h"
#include "sfc_moe_params.h"
#include "sfc_ops_params.h"
#include "sfc_params.h"
#include "sfc_rows_validate.h"
#include "sfcgemm.h"

namespace {

using sfc::Checked;

int reject(const Checked& c) { return sfc::host_error(c.code, c.msg); }
hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
const uint16_t* bf16(const void* p) { return static_cast<const uint16_t*>(p); }

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Whether a C of so many elements goes past the caches: from 32 MB on, as for the 4-bit products.  Not the largest whose
// rows are stored in parts of lines where the depth of `stages` is soon computed, so that stores bound the call (us past
// the caches / through them, weight gradients with inputs and results in rotation over four sets: fp32, 60 experts 1407x2047, 17
// rows each, 691 MB 286 / 200; 64 of 2001x1503, 128 rows, 770 MB 278 / 254; 64 of 1001x1503, 250 rows, 385 MB 172 / 153; 32 of
// 2001x1503, 128 rows, 385 MB 130 / 130; bf16, 60 of 1407x2047, 17 rows, 346 MB 210 / 132; 64 of 2047x2047, 250 rows, 536 MB 429 /
// 412.  Whole lines, fp32, 60 of 1408x2048, 17 rows, 692 MB 124 / 128; deep, 8 of 4095x4095, 2048 rows, 537 MB 624 / 631).
// Below 256 MB it goes either way: 16 of 1001x1503, 96 MB, 250 rows 46 / 47, but 64 rows 38 / 30.
bool past_caches(int64_t elements, int out_type, const void* C, int64_t ldc, int64_t stages) {
  const int64_t size = sfc::type_size(out_type), bytes = elements * size;
  const bool whole = ((uintptr_t)C | (uintptr_t)(ldc * size)) % 16 == 0;
  return bytes >= (int64_t)32 << 20 && (whole || stages > 16 || bytes < (int64_t)256 << 20);
}

// Microseconds of `tasks` blocks of b x b over `stages` 64-deep stages on the tile kernels, fitted to timings of
// random operands (rows from 2 to 16384 over 1 to 64 experts, sides 512 to 14336, weight gradients too;
// mostly within 20 %): what a full round of blocks takes, and a last, partial one, with its stores.
double moe_tile_us(int b, double tasks, double stages, bool out_f32, int num_cus) {
  const double slots = (b == 256 ? 1.0 : b == 128 ? 2.0 : 4.0) * num_cus;
  const double full = (double)(int64_t)(tasks / slots), part = tasks / slots - full;
  if (b == 256) return full * (1.5 * stages + (out_f32 ? 14 : 9)) + (part > 0 ? (1.3 + 0.2 * part) * stages + 3 + (out_f32 ? 11 : 6) * part : 0);
  if (b == 128) {
    const double last = part <= 0.5 ? (0.58 + 0.3 * part) * stages + 3.5 : (0.3 + 0.75 * part) * stages + (out_f32 ? 5 : 3);
    return full * (1.02 * stages + (out_f32 ? 7 : 4)) + (part > 0 ? last : 0);
  }
  return full * (1.1 * stages + 4) + (part > 0 ? (0.45 + 0.65 * part) * stages + 2 : 0);
}

// The block shape of the least estimated time; tasks(b) is the number of b x b blocks.
template <class F>
int moe_block_of(F tasks, double stages, bool out_f32, int num_cus) {
  int best = 256;
  double us = moe_tile_us(256, tasks(256), stages, out_f32, num_cus);
  for (int b = 128; b >= 64; b /= 2) {
    const double t = moe_tile_us(b, tasks(b), stages, out_f32, num_cus);
    if (t < us) {
      us = t;
      best = b;
    }
  }
  return best;
}

hipError_t moe_tiles(int b, const sfc::MoeGemmParams& p, sfc::MoeLayout layout, bool ob, int64_t tasks, int num_cus, hipStream_t stream) {
  const int64_t slots = (b == 256 ? 1 : b == 128 ? 2 : 4) * (int64_t)num_cus;
  const int grid = (int)(tasks < slots ? tasks : slots);
  return b == 256   ? sfc::launch_moe_256x256(p, layout, ob, grid, stream)
         : b == 128 ? sfc::launch_moe_128x128(p, layout, ob, grid, stream)
                    : sfc::launch_moe_64x64(p, layout, ob, grid, stream);
}

// Whether an experts' product runs on the kernel that streams the weights past 16 fm rows at a time (fm > 0), us
// there / on the best blocks.  Rows of 16-byte pieces: 8 an expert on average (8 experts 4096x4096, 2 rows
// 17 / 34, 32 rows 42 / 50, 64 rows 47 / 52, 128 rows 71 / 53; 64 experts 2048x4096, 128 rows 140 / 182, 512 rows 195 /
// 229), or few in all and too few blocks to fill the chip (1 expert, 64 rows 25 / 34).  Others, whose loads
// straddle lines: less than a row to an expert (8 experts 4096x4095, 2 rows 33 / 42, 32 rows 160 / 60).
int moe_few_rows(int64_t rows, int64_t N, int experts, bool aligned, int num_cus) {
  if (sfc::ceil_div(N, 16) * 512 * experts >= (int64_t)1 << 31) return 0;
  if (!aligned) return 2 * rows <= experts ? 1 : 0;
  if (rows <= 8 * (int64_t)experts) return 1;
  if (rows <= 64 && sfc::ceil_div(N, 32) * experts <= num_cus) return rows <= 32 ? 2 : 4;
  return 0;
}

// Launches a part at a time: rows first .. first + count - 1 and columns col .. col + width - 1, so
// that a launch has less than 2^32 threads (at most 512 for a row, and 4 for a row and column).
template <class F>
hipError_t lora_parts(int64_t rows, int64_t cols, F launch) {
  const int64_t width = least(cols, (int64_t)1 << 20);
  const int64_t height = width > (1 << 12) ? (int64_t)1 << 17 : (int64_t)1 << 21;
  for (int64_t first = 0; first < rows; first += height)
    for (int64_t col = 0; col < cols; col += width) {
      const hipError_t e = launch(first, least(height, rows - first), col, least(width, cols - col));
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

// Bytes of the sums that the adapters' down calls keep of ranges of K, the most that one of its launches needs.
size_t down_sums(int64_t rows, int64_t K, int64_t rank, int cus) {
  size_t most = 0;
  (void)lora_parts(rows, 1, [&](int64_t, int64_t count, int64_t, int64_t) {
    const int splits = sfc::lora_down_splits(count, K, (int)rank, cus);
    const size_t need = splits > 1 ? (size_t)splits * (size_t)count * (size_t)rank * 4u : 0;
    most = need > most ? need : most;
    return hipSuccess;
  });
  return most;
}

// Bytes that an adapters' weight gradient over parts of the rows keeps: two numbers for every adapter, then the sums.
size_t lora_table(int adapters) { return (size_t)((adapters * (int64_t)8 + 15) / 16 * 16); }
size_t lora_sums(int splits, int64_t columns, int64_t rank, int adapters) {
  return splits > 1 ? lora_table(adapters) + (size_t)splits * (size_t)columns * (size_t)rank * 4u : 0;
}

}  // namespace

extern "C" {

int sfc_moe_gemm_ex(int64_t rows, int64_t N, int64_t K, int experts, const void* A, int64_t lda, const int32_t* order,
                    int64_t a_rows, int topk, const void* B, int64_t ldb, int64_t stride_b, int b_layout,
                    const int32_t* offsets, void* C, int64_t ldc, int out_type, void* stream) {
  const Checked c = sfc::check_moe_gemm(rows, N, K, experts, sfc::kMaxExperts, A, lda, order, a_rows, topk, B, ldb, stride_b,
                                        b_layout, offsets, C, ldc, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || N == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::MoeGemmParams p = {rows, N, K, bf16(A), lda, order, a_rows, order ? topk : 1, bf16(B), ldb, stride_b, C, ldc, 0,
                          offsets, experts, nullptr, 0, 0, past_caches(rows * N, out_type, C, ldc, sfc::ceil_div(K, 64))};
  const bool ob = out_type == SFC_OUT_BF16;
  const bool aligned = ((uintptr_t)A | (uintptr_t)B) % 16 == 0 && (lda | ldb | stride_b) % 8 == 0;
  const int fm = b_layout == SFC_B_NK ? moe_few_rows(rows, N, experts, aligned, cus) : 0;
  hipError_t e;
  if (fm) {
    e = sfc::launch_moe_rows(p, fm, fm == 1 ? 1 : 2, ob, as_stream(stream));
  } else {
    // rows of an expert that has some fill a block at least, and part of a last one
    const double used = (double)least(rows, experts), each = (double)rows / used;
    auto tasks = [&](int b) { return used * (each > 0.5 * b ? each / b + 0.5 : 1.0) * (double)sfc::ceil_div(N, b); };
    const int b = moe_block_of(tasks, (double)sfc::ceil_div(K > 0 ? K : 1, 64), !ob, cus);
    p.gn = (int)sfc::ceil_div(N, b);
    e = moe_tiles(b, p, b_layout == SFC_B_NK ? sfc::kMoeNK : sfc::kMoeKN, ob, (sfc::ceil_div(rows, b) + experts) * p.gn, cus, as_stream(stream));
  }
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "experts' product");
}

int sfc_moe_wgrad_ex(int64_t M, int64_t N, int64_t rows, int experts, const void* A, int64_t lda, const void* B,
                     int64_t ldb, const int32_t* offsets, void* C, int64_t ldc, int64_t stride_c, int out_type,
                     void* stream) {
  const Checked c = sfc::check_moe_wgrad(M, N, rows, experts, sfc::kMaxExperts, A, lda, B, ldb, offsets, C, ldc, stride_c,
                                         out_type);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::MoeGemmParams p = {M, N, rows, bf16(A), lda, nullptr, 0, 1, bf16(B), ldb, 0, C, ldc, stride_c,
                          offsets, experts, nullptr, 0, 0, past_caches(M * N * experts, out_type, C, ldc, sfc::ceil_div(rows, 64 * (int64_t)experts))};
  const bool ob = out_type == SFC_OUT_BF16;
  auto tasks = [&](int b) { return (double)(sfc::ceil_div(M, b) * sfc::ceil_div(N, b)) * experts; };
  const int b = moe_block_of(tasks, (double)sfc::ceil_div(rows > 0 ? rows : 1, 64 * (int64_t)experts), !ob, cus);
  p.gm = (int)sfc::ceil_div(M, b);
  p.gn = (int)sfc::ceil_div(N, b);
  rc = sfc::host_table(p.gm, p.gn, st, &p.table);
  if (rc != SFC_OK) return rc;
  const hipError_t e = moe_tiles(b, p, sfc::kMoeTN, ob, (int64_t)p.gm * p.gn * experts, cus, st);
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "experts' weight gradient");
}

size_t sfc_lora_down_ws_size(int64_t rows, int64_t K, int64_t rank, int adapters) {
  if (sfc::check_lora_sizes(rows, K, rank, adapters, sfc::kMaxRank, SFC_B_NK).code != SFC_OK || rows == 0 || rank == 0) return 0;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  if (sfc::host_num_cus(&cus) != SFC_OK) return 0;
  return down_sums(rows, K, rank, cus);
}

int sfc_lora_down(int64_t rows, int64_t K, int64_t rank, int adapters, const void* X, int64_t ldx, const void* A, int64_t lda,
                  int64_t stride_a, int layout, const int32_t* ids, const float* scales, float* V, int64_t ldv, void* ws,
                  size_t ws_bytes, void* stream) {
  Checked c = sfc::check_lora_down(rows, K, rank, adapters, sfc::kMaxRank, X, ldx, A, lda, stride_a, layout, ids, scales,
                                   V, ldv);
  if (c.code == SFC_OK) c = sfc::check_workspace(ws);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || rank == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const size_t need = down_sums(rows, K, rank, cus);
  if (ws && ws_bytes < need) return sfc::host_error(SFC_ERR_WORKSPACE, "workspace smaller than sfc_lora_down_ws_size()");
  if (need && !ws) {
    rc = sfc::host_workspace(as_stream(stream), need, &ws);
    if (rc != SFC_OK) return rc;
  }
  const hipError_t e = lora_parts(rows, 1, [&](int64_t first, int64_t count, int64_t, int64_t) {
    sfc::LoraParams p = {};
    p.rows = count;
    p.cols = K;
    p.rank = (int)rank;
    p.adapters = adapters;
    p.ids = ids + first;
    p.X = bf16(X) + first * ldx;
    p.ldx = ldx;
    p.W = bf16(A);
    p.ldw = lda;
    p.stride_w = stride_a;
    p.scales = scales;
    p.V = V + first * ldv;
    p.ldv = ldv;
    p.splits = sfc::lora_down_splits(count, K, (int)rank, cus);
    p.sums = static_cast<float*>(ws);
    return sfc::launch_lora_down(p, layout == SFC_B_NK, as_stream(stream));
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "adapters, down");
}

int sfc_lora_up(int64_t rows, int64_t N, int64_t rank, int adapters, const float* V, int64_t ldv, const void* B, int64_t ldb,
                int64_t stride_b, int layout, const int32_t* ids, const void* base, int64_t ld_base, void* Y, int64_t ldy,
                int type, void* stream) {
  const Checked c = sfc::check_lora_up(rows, N, rank, adapters, sfc::kMaxRank, V, ldv, B, ldb, stride_b, layout, ids, base,
                                       ld_base, Y, ldy, type);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || N == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const int64_t size = sfc::type_size(type);
  const hipError_t e = lora_parts(rows, N, [&](int64_t first, int64_t count, int64_t col, int64_t width) {
    sfc::LoraParams p = {};
    p.rows = count;
    p.cols = width;
    p.rank = (int)rank;
    p.adapters = adapters;
    p.ids = ids + first;
    p.W = bf16(B) + (layout == SFC_B_NK ? col * ldb : col);
    p.ldw = ldb;
    p.stride_w = stride_b;
    p.V = const_cast<float*>(V) + first * ldv;
    p.ldv = ldv;
    p.base = base ? static_cast<const char*>(base) + (first * ld_base + col) * size : nullptr;
    p.ld_base = ld_base;
    p.Y = static_cast<char*>(Y) + (first * ldy + col) * size;
    p.ldy = ldy;
    return sfc::launch_lora_up(p, layout == SFC_B_NK, type == SFC_OUT_BF16, cus, as_stream(stream));
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "adapters, up");
}

size_t sfc_lora_wgrad_ws_size(int64_t rows, int64_t columns, int64_t rank, int adapters) {
  if (sfc::check_lora_sizes(rows, columns, rank, adapters, sfc::kMaxRank, SFC_B_NK).code != SFC_OK || columns == 0 || rank == 0)
    return 0;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  if (sfc::host_num_cus(&cus) != SFC_OK) return 0;
  return lora_sums(sfc::lora_wgrad_splits(rows, columns, (int)rank, adapters, cus), columns, rank, adapters);
}

int sfc_lora_wgrad(int64_t rows, int64_t columns, int64_t rank, int adapters, const void* Z, int64_t ldz, const float* V,
                   int64_t ldv, const int32_t* ids, void* G, int64_t ldg, int64_t stride_g, int layout, int out_type,
                   void* ws, size_t ws_bytes, void* stream) {
  Checked c = sfc::check_lora_wgrad(rows, columns, rank, adapters, sfc::kMaxRank, Z, ldz, V, ldv, ids, G, ldg, stride_g,
                                    layout, out_type);
  if (c.code == SFC_OK) c = sfc::check_workspace(ws);
  if (c.code != SFC_OK) return reject(c);
  if (columns == 0 || rank == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::LoraParams p = {};
  p.splits = sfc::lora_wgrad_splits(rows, columns, (int)rank, adapters, cus);
  const size_t need = lora_sums(p.splits, columns, rank, adapters);
  if (ws && ws_bytes < need) return sfc::host_error(SFC_ERR_WORKSPACE, "workspace smaller than sfc_lora_wgrad_ws_size()");
  if (need && !ws) {
    rc = sfc::host_workspace(as_stream(stream), need, &ws);
    if (rc != SFC_OK) return rc;
  }
  if (p.splits > 1) {
    p.parts = static_cast<int32_t*>(ws);
    p.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + lora_table(adapters));
  }
  p.rows = rows;
  p.cols = columns;
  p.rank = (int)rank;
  p.adapters = adapters;
  p.ids = ids;
  p.X = bf16(Z);
  p.ldx = ldz;
  p.V = const_cast<float*>(V);
  p.ldv = ldv;
  p.Y = G;
  p.ldy = ldg;
  p.stride_y = stride_g;
  const hipError_t e = sfc::launch_lora_wgrad(p, layout == SFC_B_NK, out_type == SFC_OUT_BF16, as_stream(stream));
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "adapters, weight gradient");
}

}  // extern "C"
