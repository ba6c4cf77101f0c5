// C ABI of the 4-bit (MX) and expert operators (declarations and contracts in
// include/sfcgemm.h): argument checks, the choice of kernel, workspaces and launches.
// No entry point synchronises the device or a stream.
#include <hip/hip_runtime.h>

#include <mutex>

#include "sfc_host.h"
#include "sfc_ops_params.h"
#include "sfc_ops_validate.h"
#include "sfc_params.h"
#include "sfcgemm.h"

namespace {

using sfc::Checked;

int reject(const Checked& c) { return sfc::host_error(c.code, c.msg); }
hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
const uint8_t* bytes(const void* p) { return static_cast<const uint8_t*>(p); }
int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// Whether a C of so many elements goes past the caches: from 32 MB on, as for the row operators
// (us, through / past: bf16 4096x4096x1024 18.7 / 17.3, 4096x14336x4096 141 / 139; fp32
// 2048x4096x1024 14.7 / 12.9, 4096x14336x1024 77.7 / 67.4, 8192^3 276 / 268, the weight gradients of
// 8 experts 2048x4096 with 8192 rows 113 / 89), and what is read next is still cached.
bool past_caches(int64_t elements, int out_type) { return elements * (out_type == SFC_OUT_BF16 ? 2 : 4) >= (int64_t)32 << 20; }

// How a dense product runs.
struct Mx4Plan {
  bool few = false;                    // up to 16 rows: A stays in registers
  int fm = 0;                          // > 0: the streaming kernel, 16 * fm rows at a time
  bool large = false;                  // 256x256 blocks, else 128x128
  int layers = 1;
};

// Microseconds of `tasks` blocks over `stages` 256-deep stages on the tile kernels, fitted to
// timings of random operands (M, N from 100 to 14336, K from 1024 to 16384; mostly within 10 %):
// 256x256 blocks take 1.9 us a stage on a full chip (1.5 on few CUs: the clock), 128x128
// blocks 0.6 alone on a CU and 1.15 for the two that share one; then the store of a round.
double mx4_tile_us(bool large, double tasks, double stages, bool out_f32, int num_cus) {
  const double slots = large ? num_cus : 2 * num_cus;
  const double full = (double)(int64_t)(tasks / slots), part = tasks / slots - full;
  double us = full * (large ? 1.9 * stages + (out_f32 ? 11.0 : 5.5) : 1.15 * stages + (out_f32 ? 4.5 : 2.5));
  if (part > 0) {
    if (large) us += (1.5 + 0.4 * part) * stages + 2.0 + (out_f32 ? 9.0 : 3.5) * part;
    else if (part <= 0.5) us += (0.55 + 0.2 * part) * stages + 0.4 + (out_f32 ? 4.5 : 2.2) * part;
    else us += (0.3 + 0.85 * part) * stages + (out_f32 ? 4.0 : 2.5);
  }
  return us;
}

Mx4Plan mx4_plan(int64_t M, int64_t N, int64_t K, bool out_f32, int num_cus) {
  Mx4Plan pl;
  if (M <= 16) {
    // (one block of columns to a workgroup and several turns to a wave: no loads ahead to gain.
    // 1x4096x14336: 10.2 us, streaming 8.4; 1x16384x16384: 26.8, streaming 30.7)
    pl.few = K <= 16 * 512 || (K <= sfc::kFewDepth && N > 16 * (int64_t)num_cus);
    pl.fm = pl.few ? 0 : 1;
    return pl;
  }
  // Up to 64 rows: the streaming kernel reads A once for every 32 columns, which pays while a
  // wave has one turn of K (us, streaming against 128x128 blocks with their best layers:
  // 32x4096x4096 7.6 / 10.6, 32x14336x4096 13.7 / 14.5, 32x4096x14336 20.5 / 16.0; 64x4096x4096
  // 10.3 / 11.7, 64x1024x1024 4.4 / 6.2, 64x14336x4096 21.0 / 15.5).  (2^28: 512 threads for every 32
  // columns have to fit a launch.)
  if (M <= 64 && K <= 8 * 512 && (M <= 32 ? N < (int64_t)1 << 28 : N <= 4096)) {
    pl.fm = M <= 32 ? 2 : 4;
    return pl;
  }
  // block shape and layers of the least estimated time; copies are written, and read back by a
  // second launch (2.5 us and 0.3 a layer), at 6 TB/s
  double best = 0;
  for (int large = 1; large >= 0; --large) {
    const int64_t b = large ? 256 : 128, blocks = sfc::ceil_div(M, b) * sfc::ceil_div(N, b);
    const int64_t stages = K > 0 ? sfc::ceil_div(K, 256) : 1;
    for (int c = 1; c <= sfc::kAutoLayers && (c == 1 || 2 * c <= stages); c *= 2) {
      double us = mx4_tile_us(large, (double)(blocks * c), (double)sfc::ceil_div(stages, c), out_f32 || c > 1, num_cus);
      if (c > 1) us += 2.5 + 0.3 * c + 8.0 * (double)c * (double)M * (double)N / 6.0e6;
      if (best == 0 || us < best) {
        best = us;
        pl.large = large != 0;
        pl.layers = c;
      }
    }
  }
  return pl;
}

// Bytes of layer copies that the plan needs.
size_t mx4_copies(const Mx4Plan& pl, int64_t M, int64_t N) {
  return pl.layers > 1 ? (size_t)pl.layers * (size_t)M * (size_t)N * 4u : 0;
}

// How a linear layer runs: its product, and the memory for X's codes and scales, then the product's
// layer copies.
struct LinearPlan {
  Mx4Plan product;
  bool fused = false;                  // X brought to 4 bits by the product's own launch
  int64_t blocks = 0, ldq = 0, lds = 0;
  size_t codes = 0, scales = 0, copies = 0;
  size_t bytes() const { return codes + scales + copies; }
};

LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, bool out_f32, int num_cus) {
  LinearPlan pl;
  pl.blocks = sfc::mx4_blocks(K);
  pl.product = mx4_plan(M, N, 32 * pl.blocks, out_f32, num_cus);
  // Few rows brought to 4 bits by the product's own launch: every workgroup converts them, which
  // costs less than a launch while they or the workgroups are few (us in a graph, both
  // launches against one: 1x4096x4096 7.2 / 5.6, 16x4096x4096 7.4 / 8.0 but 3.5 us less host time,
  // 8x14336x4096 11.6 / 11.6, 16x14336x4096 11.7 / 13.0).
  pl.fused = pl.product.few && K > 0 && K <= sfc::kConvertDepth && (M <= 8 || N <= 32 * (int64_t)num_cus);
  if (pl.fused) return pl;
  pl.ldq = 16 * pl.blocks;
  pl.lds = round_up(pl.blocks, 4);
  pl.codes = (size_t)M * (size_t)pl.ldq;
  pl.scales = (size_t)round_up(M * pl.lds, 16);
  pl.copies = mx4_copies(pl.product, M, N);
  return pl;
}

// `need` bytes at *ws: the caller's, if there are any, else the stream's.  With the lock held.
int memory(hipStream_t stream, size_t need, size_t ws_bytes, const char* too_small, void** ws) {
  if (*ws) return ws_bytes < need ? sfc::host_error(SFC_ERR_WORKSPACE, too_small) : SFC_OK;
  return need ? sfc::host_workspace(stream, need, ws) : SFC_OK;
}

// For the queries of sizes: the number of CUs, if the sizes are good and not empty.
bool ws_device(const Checked& c, int64_t M, int64_t N, int* num_cus) {
  if (c.code != SFC_OK || M == 0 || N == 0) return false;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  return sfc::host_num_cus(num_cus) == SFC_OK;
}

// Launches a dense product; `copies` holds its layer copies.  With the lock held.
int mx4_dense(const Mx4Plan& pl, sfc::Mx4GemmParams& p, bool ob, int num_cus, float* copies, hipStream_t stream) {
  if (pl.few || pl.fm) {
    const hipError_t e = pl.few ? sfc::launch_mx4_few(p, sfc::kRowsCodes, num_cus, ob, stream)
                                : sfc::launch_mx4_rows(p, sfc::kMxDense, pl.fm, sfc::ceil_div(p.N, 32) < num_cus, ob, stream);
    return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "4-bit product of few rows");
  }
  const int b = pl.large ? 256 : 128;
  p.gm = (int)sfc::ceil_div(p.M, b);
  p.gn = (int)sfc::ceil_div(p.N, b);
  p.layers = pl.layers;
  p.experts = 0;
  const int rc = sfc::host_table(p.gm, p.gn, stream, &p.table);
  if (rc != SFC_OK) return rc;
  void* C = p.C;
  const int64_t ldc = p.ldc;
  if (pl.layers > 1) {
    p.C = copies;
    p.ldc = p.N;
    p.stride_c = p.M * p.N;
    p.past = false;                    // (read next)
  }
  const int64_t tasks = (int64_t)p.gm * p.gn * pl.layers, slots = pl.large ? num_cus : 2 * num_cus;
  const int grid = (int)(tasks < slots ? tasks : slots);
  const bool bf16 = ob && pl.layers == 1;
  hipError_t e = pl.large ? sfc::launch_mx4_256x256(p, sfc::kMxDense, bf16, grid, stream)
                          : sfc::launch_mx4_128x128(p, sfc::kMxDense, bf16, grid, stream);
  if (e != hipSuccess) return sfc::host_hip_error(e, "4-bit product");
  if (pl.layers > 1) {
    e = sfc::launch_reduce(copies, pl.layers, p.M, p.N, C, ldc, ob, stream);
    if (e != hipSuccess) return sfc::host_hip_error(e, "sum of the layer copies");
  }
  return SFC_OK;
}

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }
const char* at(const void* p, int64_t offset) { return p ? static_cast<const char*>(p) + offset : nullptr; }
uint8_t* at(uint8_t* p, int64_t offset) { return p ? p + offset : nullptr; }

// Rows first .. first + count - 1 of X for every launch that `rows` of them take.
template <class F>
hipError_t row_launches(int64_t rows, F launch) {
  for (int64_t first = 0; first < rows; first += sfc::kLaunchRows) {
    const hipError_t e = launch(first, least(sfc::kLaunchRows, rows - first));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// A part of a quantisation: `count` rows from row `first` (a multiple of 256) and `width` columns from
// column `col` (a multiple of 128).
hipError_t quant_part(const sfc::Mx4QuantParams& all, int64_t first, int64_t count, int64_t col, int64_t width, bool bf16,
                      int num_cus, hipStream_t stream) {
  sfc::Mx4QuantParams p = all;
  p.rows = count;
  p.cols = width;
  p.X = at(all.X, ((all.order ? 0 : first * all.ldx) + col) * (bf16 ? 2 : 4));
  if (all.order) p.order += first;
  else p.x_rows = count;
  p.Q = at(all.Q, first * all.ldq + col / 2);
  p.S = at(all.S, first * all.lds + col / 32);
  p.Qt = at(all.Qt, col * all.ldqt + first / 2);
  p.St = at(all.St, col * all.ldst + first / 32);
  return sfc::launch_mx4_quant(p, bf16, num_cus, stream);
}

int quant_launch(const sfc::Mx4QuantParams& p, bool bf16, int num_cus, hipStream_t stream) {
  // along the columns as many whole blocks of 128 columns as a launch has workgroups for
  const int64_t row_groups = sfc::ceil_div(least(p.rows, sfc::kLaunchRows), 128);
  const int64_t cols = p.Qt ? sfc::kLaunchBlocks / row_groups * 128 : p.cols;
  const hipError_t e = row_launches(p.rows, [&](int64_t first, int64_t count) {
    for (int64_t c = 0; c < p.cols; c += cols) {
      const hipError_t part = quant_part(p, first, count, c, least(cols, p.cols - c), bf16, num_cus, stream);
      if (part != hipSuccess) return part;
    }
    return hipSuccess;
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "4-bit quantisation");
}

}  // namespace

extern "C" {

int sfc_mx4_quant(int64_t rows, int64_t cols, const void* X, int64_t ldx, int in_type, const int32_t* order,
                  int64_t x_rows, int topk, void* Q, int64_t ldq, void* S, int64_t lds, void* Qt, int64_t ldqt,
                  void* St, int64_t ldst, void* stream) {
  const Checked c = sfc::check_mx4_quant(rows, cols, X, ldx, in_type, order, x_rows, topk, Q, ldq, S, lds, Qt, ldqt, St,
                                         ldst);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || cols == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::Mx4QuantParams p;
  p.rows = rows;
  p.cols = cols;
  p.X = X;
  p.ldx = ldx;
  p.order = order;
  p.x_rows = order ? x_rows : rows;
  p.topk = order ? topk : 1;
  p.Q = static_cast<uint8_t*>(Q);
  p.ldq = ldq;
  p.S = static_cast<uint8_t*>(S);
  p.lds = lds;
  p.Qt = static_cast<uint8_t*>(Qt);
  p.ldqt = ldqt;
  p.St = static_cast<uint8_t*>(St);
  p.ldst = ldst;
  return quant_launch(p, in_type == SFC_OUT_BF16, cus, as_stream(stream));
}

int sfc_mx4_dequant(int64_t rows, int64_t cols, const void* Q, int64_t ldq, const void* S, int64_t lds, void* Y,
                    int64_t ldy, int out_type, void* stream) {
  const Checked c = sfc::check_mx4_dequant(rows, cols, Q, ldq, S, lds, Y, ldy, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || cols == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const hipError_t e = row_launches(rows, [&](int64_t first, int64_t count) {
    const sfc::Mx4DequantParams p = {count, cols, bytes(Q) + first * ldq, bytes(S) + first * lds, ldq, lds,
                                     static_cast<char*>(Y) + first * ldy * sfc::type_size(out_type), ldy};
    return sfc::launch_mx4_dequant(p, out_type == SFC_OUT_BF16, cus, as_stream(stream));
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "4-bit dequantisation");
}

int sfc_gemm_mx4_ex(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* As, int64_t ldas,
                    const void* B, int64_t ldb, const void* Bs, int64_t ldbs, void* C, int64_t ldc, int out_type,
                    void* stream) {
  return sfc_gemm_mx4_ws_ex(M, N, K, A, lda, As, ldas, B, ldb, Bs, ldbs, C, ldc, out_type, nullptr, 0, stream);
}

size_t sfc_gemm_mx4_ws_size(int64_t M, int64_t N, int64_t K, int out_type) {
  int cus = 0;
  if (!ws_device(sfc::check_gemm_mx4_sizes(M, N, K, out_type), M, N, &cus)) return 0;
  return mx4_copies(mx4_plan(M, N, K, out_type == SFC_OUT_F32, cus), M, N);
}

int sfc_gemm_mx4_ws_ex(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* As, int64_t ldas,
                       const void* B, int64_t ldb, const void* Bs, int64_t ldbs, void* C, int64_t ldc, int out_type,
                       void* ws, size_t ws_bytes, void* stream) {
  Checked c = sfc::check_gemm_mx4(M, N, K, A, lda, As, ldas, B, ldb, Bs, ldbs, C, ldc, out_type);
  if (c.code == SFC_OK) c = sfc::check_workspace(ws);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const Mx4Plan pl = mx4_plan(M, N, K, out_type == SFC_OUT_F32, cus);
  rc = memory(st, mx4_copies(pl, M, N), ws_bytes, "workspace smaller than sfc_gemm_mx4_ws_size()", &ws);
  if (rc != SFC_OK) return rc;
  sfc::Mx4GemmParams p = {M, N, K, bytes(A), bytes(As), bytes(B), bytes(Bs), lda, ldas, ldb, ldbs, 0, 0, C, ldc, 0,
                          nullptr, 0, 0, 0, nullptr, 1, past_caches(M * N, out_type), nullptr, 0, 0};
  return mx4_dense(pl, p, out_type == SFC_OUT_BF16, cus, static_cast<float*>(ws), st);
}

int sfc_mx4_linear(int64_t M, int64_t N, int64_t K, const void* X, int64_t ldx, int in_type, const void* W, int64_t ldw,
                   const void* Ws, int64_t ldws, void* Y, int64_t ldy, int out_type, void* stream) {
  return sfc_mx4_linear_ws(M, N, K, X, ldx, in_type, W, ldw, Ws, ldws, Y, ldy, out_type, nullptr, 0, stream);
}

size_t sfc_mx4_linear_ws_size(int64_t M, int64_t N, int64_t K, int out_type) {
  int cus = 0;
  if (!ws_device(sfc::check_mx4_linear_sizes(M, N, K, out_type, out_type), M, N, &cus)) return 0;
  const LinearPlan pl = linear_plan(M, N, K, out_type == SFC_OUT_F32, cus);
  return pl.bytes();
}

int sfc_mx4_linear_ws(int64_t M, int64_t N, int64_t K, const void* X, int64_t ldx, int in_type, const void* W, int64_t ldw,
                      const void* Ws, int64_t ldws, void* Y, int64_t ldy, int out_type, void* ws, size_t ws_bytes,
                      void* stream) {
  Checked c = sfc::check_mx4_linear(M, N, K, X, ldx, in_type, W, ldw, Ws, ldws, Y, ldy, out_type);
  if (c.code == SFC_OK) c = sfc::check_workspace(ws);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const LinearPlan pl = linear_plan(M, N, K, out_type == SFC_OUT_F32, cus);
  if (pl.fused) {
    const sfc::Mx4GemmParams p = {M, N, 32 * pl.blocks, nullptr, nullptr, bytes(W), bytes(Ws), 0, 0, ldw, ldws, 0, 0, Y, ldy,
                                  0, nullptr, 0, 0, 0, nullptr, 1, false, X, ldx, K};
    const hipError_t e = sfc::launch_mx4_few(p, in_type == SFC_OUT_BF16 ? sfc::kRowsBf16 : sfc::kRowsF32, cus,
                                             out_type == SFC_OUT_BF16, st);
    return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "4-bit product of few rows");
  }
  rc = memory(st, pl.bytes(), ws_bytes, "workspace smaller than sfc_mx4_linear_ws_size()", &ws);
  if (rc != SFC_OK) return rc;
  uint8_t* q = static_cast<uint8_t*>(ws);
  if (K > 0) {
    sfc::Mx4QuantParams x = {M, K, X, ldx, nullptr, M, 1, q, q + pl.codes, pl.ldq, pl.lds, nullptr, nullptr, 0, 0};
    rc = quant_launch(x, in_type == SFC_OUT_BF16, cus, st);
    if (rc != SFC_OK) return rc;
  }
  sfc::Mx4GemmParams p = {M, N, 32 * pl.blocks, q, q + pl.codes, bytes(W), bytes(Ws), pl.ldq, pl.lds, ldw, ldws, 0, 0, Y, ldy,
                          0, nullptr, 0, 0, 0, nullptr, 1, past_caches(M * N, out_type), nullptr, 0, 0};
  return mx4_dense(pl.product, p, out_type == SFC_OUT_BF16, cus, reinterpret_cast<float*>(q + pl.codes + pl.scales), st);
}

int sfc_moe_gemm_mx4_ex(int64_t rows, int64_t N, int64_t K, int experts, const void* A, int64_t lda, const void* As,
                        int64_t ldas, const void* B, int64_t ldb, int64_t stride_b, const void* Bs, int64_t ldbs,
                        int64_t stride_bs, const int32_t* offsets, void* C, int64_t ldc, int out_type, void* stream) {
  const Checked c = sfc::check_moe_gemm_mx4(rows, N, K, experts, sfc::kMaxExperts, A, lda, As, ldas, B, ldb, stride_b, Bs,
                                            ldbs, stride_bs, offsets, C, ldc, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::Mx4GemmParams p = {rows, N, K, bytes(A), bytes(As), bytes(B), bytes(Bs), lda, ldas, ldb, ldbs, stride_b,
                          stride_bs, C, ldc, 0, nullptr, 0, 0, experts, offsets, 1, past_caches(rows * N, out_type), nullptr, 0, 0};
  const bool ob = out_type == SFC_OUT_BF16;
  hipError_t e;
  const double stages = (double)sfc::ceil_div(K > 0 ? K : 1, 256);
  // blocks of rows: every expert's last one is on average half full
  auto tasks = [&](int64_t b) { return ((double)rows / (double)b + 0.5 * experts) * (double)sfc::ceil_div(N, b); };
  if (rows <= 32 * (int64_t)experts && experts * sfc::ceil_div(N, 128) < cus) {
    // Few rows to an expert, and too few blocks of columns to fill the chip (us, the streaming
    // kernel / 128x128 blocks, 2 rows to an expert: 8 experts 2048x4096 11.1 / 15.2, 4 experts
    // 4096x4096 10.7 / 15.3; 64 experts 2048x4096 66 / 58, 16 rows to one of 16 experts
    // 2048x4096 33 / 17: an expert's rows past 16 fm read its weights again)
    e = sfc::launch_mx4_rows(p, sfc::kMxRows, rows <= 8 * (int64_t)experts ? 1 : 2, false, ob, st);
  } else {
    const bool big = mx4_tile_us(true, tasks(256), stages, !ob, cus) < mx4_tile_us(false, tasks(128), stages, !ob, cus);
    const int b = big ? 256 : 128;
    p.gn = (int)sfc::ceil_div(N, b);
    const int64_t most = (sfc::ceil_div(rows, b) + experts) * p.gn, slots = big ? cus : 2 * cus;
    const int grid = (int)(most < slots ? most : slots);
    e = big ? sfc::launch_mx4_256x256(p, sfc::kMxRows, ob, grid, st) : sfc::launch_mx4_128x128(p, sfc::kMxRows, ob, grid, st);
  }
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "experts' 4-bit product");
}

int sfc_moe_wgrad_mx4_ex(int64_t M, int64_t N, int64_t rows, int experts, const void* A, int64_t lda, const void* As,
                         int64_t ldas, const void* B, int64_t ldb, const void* Bs, int64_t ldbs, const int32_t* offsets,
                         void* C, int64_t ldc, int64_t stride_c, int out_type, void* stream) {
  const Checked c = sfc::check_moe_wgrad_mx4(M, N, rows, experts, sfc::kMaxExperts, A, lda, As, ldas, B, ldb, Bs, ldbs,
                                             offsets, C, ldc, stride_c, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::Mx4GemmParams p = {M, N, rows, bytes(A), bytes(As), bytes(B), bytes(Bs), lda, ldas, ldb, ldbs, 0, 0, C, ldc,
                          stride_c, nullptr, 0, 0, experts, offsets, 1, past_caches(M * N * experts, out_type), nullptr, 0, 0};
  const bool ob = out_type == SFC_OUT_BF16;
  const double stages = (double)sfc::ceil_div(rows > 0 ? rows : 1, 256 * (int64_t)experts);
  auto us = [&](int64_t b) {
    return mx4_tile_us(b == 256, (double)(sfc::ceil_div(M, b) * sfc::ceil_div(N, b) * experts), stages, !ob, cus);
  };
  const bool big = us(256) < us(128);
  const int b = big ? 256 : 128;
  p.gm = (int)sfc::ceil_div(M, b);
  p.gn = (int)sfc::ceil_div(N, b);
  rc = sfc::host_table(p.gm, p.gn, st, &p.table);
  if (rc != SFC_OK) return rc;
  const int64_t tasks = (int64_t)p.gm * p.gn * experts, slots = big ? cus : 2 * cus;
  const int grid = (int)(tasks < slots ? tasks : slots);
  const hipError_t e = big ? sfc::launch_mx4_256x256(p, sfc::kMxDepth, ob, grid, st)
                           : sfc::launch_mx4_128x128(p, sfc::kMxDepth, ob, grid, st);
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "experts' 4-bit weight gradient");
}

size_t sfc_moe_sort_ws_size(int64_t slots, int experts) {
  if (slots < 0 || slots >= sfc::kMaxDim || experts < 1 || experts > sfc::kMaxExperts) return 0;
  const int64_t chunks = sfc::ceil_div(slots, sfc::kSortChunk);
  return chunks > 1 ? (size_t)(chunks > sfc::kSortScan ? chunks + 1 : chunks) * (size_t)experts * 4u : 0;
}

int sfc_moe_sort(int64_t slots, int experts, int align, const int32_t* ids, int64_t rows, int32_t* offsets,
                 int32_t* order, int32_t* pos, void* ws, size_t ws_bytes, void* stream) {
  const Checked c = sfc::check_moe_sort(slots, experts, sfc::kMaxExperts, align, ids, rows, offsets, order, pos);
  if (c.code != SFC_OK) return reject(c);
  const size_t need = sfc_moe_sort_ws_size(slots, experts);
  if (ws && ws_bytes < need) return sfc::host_error(SFC_ERR_WORKSPACE, "workspace smaller than sfc_moe_sort_ws_size()");
  if (ws && (uintptr_t)ws % 4) return sfc::host_error(SFC_ERR_UNSUPPORTED, "workspace must be 4-byte aligned");
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  if (need && !ws) {
    const int rc = sfc::host_workspace(st, need, &ws);
    if (rc != SFC_OK) return rc;
  }
  const sfc::MoeSortParams p = {slots, experts, align, ids, rows, offsets, order, pos, static_cast<int32_t*>(ws)};
  const hipError_t e = sfc::launch_moe_sort(p, st);
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "sort by expert");
}

int sfc_moe_dispatch(int64_t rows, int64_t cols, int64_t tokens, int topk, const void* X, int64_t ldx, int type,
                     const int32_t* order, const float* weights, void* Xs, int64_t ldxs, void* stream) {
  Checked c = sfc::check_moe_sizes(tokens, rows, cols, topk, type);
  if (c.code == SFC_OK && rows > 0 && cols > 0) {
    c = sfc::check_rows(X, tokens, cols, ldx, type, "X is NULL", "ldx < cols");
    if (c.code == SFC_OK) c = sfc::check_rows(Xs, rows, cols, ldxs, type, "Xs is NULL", "ldxs < cols");
    if (c.code == SFC_OK) c = sfc::check_index(order, "order is NULL");
    if (c.code == SFC_OK) c = sfc::check_weights(weights);
  }
  if (c.code != SFC_OK) return reject(c);
  if (rows == 0 || cols == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const hipError_t e = row_launches(rows, [&](int64_t first, int64_t count) {
    const sfc::MoeRowsParams p = {tokens, count, cols, topk, X, ldx, nullptr, 0, order + first, nullptr, weights,
                                  static_cast<char*>(Xs) + first * ldxs * sfc::type_size(type), ldxs, nullptr, 0, 0, 0, 0};
    return sfc::launch_moe_dispatch(p, type == SFC_OUT_BF16, cus, as_stream(stream));
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "dispatch");
}

int sfc_moe_combine(int64_t tokens, int64_t cols, int64_t rows, int topk, const void* Ys, int64_t ldys, int type,
                    const int32_t* pos, const float* weights, void* Y, int64_t ldy, void* stream) {
  Checked c = sfc::check_moe_sizes(tokens, rows, cols, topk, type);
  if (c.code == SFC_OK && tokens > 0 && cols > 0) {
    c = sfc::check_rows(Ys, rows, cols, ldys, type, "Ys is NULL", "ldys < cols");
    if (c.code == SFC_OK) c = sfc::check_rows(Y, tokens, cols, ldy, type, "Y is NULL", "ldy < cols");
    if (c.code == SFC_OK) c = sfc::check_index(pos, "pos is NULL");
    if (c.code == SFC_OK) c = sfc::check_weights(weights);
  }
  if (c.code != SFC_OK) return reject(c);
  if (tokens == 0 || cols == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const hipError_t e = row_launches(tokens, [&](int64_t first, int64_t count) {
    const sfc::MoeRowsParams p = {count, rows, cols, topk, Ys, ldys, nullptr, 0, nullptr, pos + first * topk,
                                  weights ? weights + first * topk : nullptr,
                                  static_cast<char*>(Y) + first * ldy * sfc::type_size(type), ldy, nullptr, 0, 0, 0, 0};
    return sfc::launch_moe_combine(p, type == SFC_OUT_BF16, cus, as_stream(stream));
  });
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "combine");
}

int sfc_moe_combine_grad(int64_t tokens, int64_t cols, int64_t rows, int topk, const void* dY, int64_t lddy,
                         const void* Ys, int64_t ldys, int type, const int32_t* order, const int32_t* pos,
                         const float* weights, void* dYs, int64_t lddys, float* dW, void* stream) {
  Checked c = sfc::check_moe_sizes(tokens, rows, cols, topk, type);
  if (c.code == SFC_OK) c = sfc::check_rows(dY, tokens, cols, lddy, type, "dY is NULL", "lddy < cols");
  if (c.code == SFC_OK) c = sfc::check_rows(Ys, rows, cols, ldys, type, "Ys is NULL", "ldys < cols");
  if (c.code == SFC_OK) c = sfc::check_rows(dYs, rows, cols, lddys, type, "dYs is NULL", "lddys < cols");
  if (c.code == SFC_OK && rows > 0) c = sfc::check_index(order, "order is NULL");
  if (c.code == SFC_OK && tokens > 0) c = sfc::check_index(pos, "pos is NULL");
  if (c.code == SFC_OK && tokens > 0) c = sfc::check_index(dW, "dW is NULL");
  if (c.code == SFC_OK) c = sfc::check_weights(weights);
  if (c.code != SFC_OK) return reject(c);
  if (tokens == 0 && rows == 0) return SFC_OK;
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  const int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  sfc::MoeRowsParams p = {tokens, rows, cols, topk, dY, lddy, Ys, ldys, order, pos, weights, dYs, lddys, dW, 0, 0, 0, 0};
  hipError_t e = hipSuccess;
  while (e == hipSuccess && (p.end_token < tokens || p.end_row < rows)) {
    p.first_token = p.end_token;
    p.end_token = least(p.first_token + sfc::kLaunchRows, tokens);
    p.first_row = p.end_row;
    p.end_row = least(p.first_row + 8 * sfc::kLaunchRows, rows);
    e = sfc::launch_moe_combine_grad(p, type == SFC_OUT_BF16, cus, as_stream(stream));
  }
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "gradient of combine");
}

}  // extern "C"
