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

// How a dense product runs.
struct Mx4Plan {
  int fm = 0, fn = 0, waves = 0;       // fm > 0: the kernel for few rows
  bool large = false;                  // 256x256 blocks, else 128x128
  int layers = 1;
};

Mx4Plan mx4_plan(int64_t M, int64_t N, int64_t K, int num_cus) {
  Mx4Plan pl;
  const int64_t turns = sfc::ceil_div(K, 512);
  if (M <= 64) {
    pl.fm = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    pl.fn = pl.fm == 1 && sfc::ceil_div(N, 32) < num_cus ? 1 : 2;
    pl.waves = turns >= 8 ? 8 : 4;
    return pl;
  }
  const int64_t large = sfc::ceil_div(M, 256) * sfc::ceil_div(N, 256);
  pl.large = 2 * large >= num_cus;
  const int64_t tasks = pl.large ? large : sfc::ceil_div(M, 128) * sfc::ceil_div(N, 128);
  const int64_t slots = pl.large ? num_cus : 2 * num_cus;
  while (pl.layers < sfc::kAutoLayers && 2 * tasks * pl.layers <= slots && turns >= 4 * pl.layers) pl.layers *= 2;
  return pl;
}

// Bytes of layer copies that the plan needs.
size_t mx4_copies(const Mx4Plan& pl, int64_t M, int64_t N) {
  return pl.layers > 1 ? (size_t)pl.layers * (size_t)M * (size_t)N * 4u : 0;
}

// Launches a dense product; `copies` holds its layer copies.  With the lock held.
int mx4_dense(const Mx4Plan& pl, sfc::Mx4GemmParams& p, bool ob, int num_cus, float* copies, hipStream_t stream) {
  if (pl.fm) {
    const hipError_t e = sfc::launch_mx4_rows(p, sfc::kMxDense, pl.fm, pl.fn, pl.waves, ob, stream);
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

int quant_launch(const sfc::Mx4QuantParams& p, bool bf16, int num_cus, hipStream_t stream) {
  const hipError_t e = sfc::launch_mx4_quant(p, bf16, num_cus, stream);
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
  const sfc::Mx4DequantParams p = {rows, cols, bytes(Q), bytes(S), ldq, lds, Y, ldy};
  const hipError_t e = sfc::launch_mx4_dequant(p, out_type == SFC_OUT_BF16, cus, as_stream(stream));
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "4-bit dequantisation");
}

int sfc_gemm_mx4_ex(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* As, int64_t ldas,
                    const void* B, int64_t ldb, const void* Bs, int64_t ldbs, void* C, int64_t ldc, int out_type,
                    void* stream) {
  const Checked c = sfc::check_gemm_mx4(M, N, K, A, lda, As, ldas, B, ldb, Bs, ldbs, C, ldc, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const Mx4Plan pl = mx4_plan(M, N, K, cus);
  void* ws = nullptr;
  const size_t need = mx4_copies(pl, M, N);
  if (need) rc = sfc::host_workspace(st, need, &ws);
  if (rc != SFC_OK) return rc;
  sfc::Mx4GemmParams p = {M, N, K, bytes(A), bytes(As), bytes(B), bytes(Bs), lda, ldas, ldb, ldbs, 0, 0, C, ldc, 0,
                          nullptr, 0, 0, 0, nullptr, 1};
  return mx4_dense(pl, p, out_type == SFC_OUT_BF16, cus, static_cast<float*>(ws), st);
}

int sfc_mx4_linear(int64_t M, int64_t N, int64_t K, const void* X, int64_t ldx, int in_type, const void* W, int64_t ldw,
                   const void* Ws, int64_t ldws, void* Y, int64_t ldy, int out_type, void* stream) {
  const Checked c = sfc::check_mx4_linear(M, N, K, X, ldx, in_type, W, ldw, Ws, ldws, Y, ldy, out_type);
  if (c.code != SFC_OK) return reject(c);
  if (M == 0 || N == 0) return SFC_OK;
  const hipStream_t st = as_stream(stream);
  std::lock_guard<std::mutex> lock(sfc::host_mutex());
  int cus = 0;
  int rc = sfc::host_num_cus(&cus);
  if (rc != SFC_OK) return rc;
  const int64_t blocks = sfc::mx4_blocks(K), ldq = 16 * blocks, lds = round_up(blocks, 4);
  const Mx4Plan pl = mx4_plan(M, N, 32 * blocks, cus);
  // the stream's workspace: codes and scales of X, then the layer copies
  const size_t code_bytes = (size_t)M * (size_t)ldq, scale_bytes = (size_t)round_up(M * lds, 16);
  void* ws = nullptr;
  if (K > 0 || pl.layers > 1) rc = sfc::host_workspace(st, code_bytes + scale_bytes + mx4_copies(pl, M, N), &ws);
  if (rc != SFC_OK) return rc;
  uint8_t* q = static_cast<uint8_t*>(ws);
  if (K > 0) {
    sfc::Mx4QuantParams x = {M, K, X, ldx, nullptr, M, 1, q, q + code_bytes, ldq, lds, nullptr, nullptr, 0, 0};
    rc = quant_launch(x, in_type == SFC_OUT_BF16, cus, st);
    if (rc != SFC_OK) return rc;
  }
  sfc::Mx4GemmParams p = {M, N, 32 * blocks, q, q + code_bytes, bytes(W), bytes(Ws), ldq, lds, ldw, ldws, 0, 0, Y, ldy,
                          0, nullptr, 0, 0, 0, nullptr, 1};
  return mx4_dense(pl, p, out_type == SFC_OUT_BF16, cus, reinterpret_cast<float*>(q + code_bytes + scale_bytes), st);
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
                          stride_bs, C, ldc, 0, nullptr, 0, 0, experts, offsets, 1};
  const bool ob = out_type == SFC_OUT_BF16;
  hipError_t e;
  if (rows <= 32 * (int64_t)experts) {
    const int64_t turns = sfc::ceil_div(K, 512);
    e = sfc::launch_mx4_rows(p, sfc::kMxRows, rows <= 16 * (int64_t)experts ? 1 : 2, 2, turns >= 8 ? 8 : 4, ob, st);
  } else {
    const int64_t large = (rows / 256 + experts) * sfc::ceil_div(N, 256);
    const bool big = rows >= 192 * (int64_t)experts && 2 * large >= cus;
    const int b = big ? 256 : 128;
    p.gn = (int)sfc::ceil_div(N, b);
    const int64_t tasks = (sfc::ceil_div(rows, b) + experts) * p.gn, slots = big ? cus : 2 * cus;
    const int grid = (int)(tasks < slots ? tasks : slots);
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
                          stride_c, nullptr, 0, 0, experts, offsets, 1};
  const bool ob = out_type == SFC_OUT_BF16;
  const int64_t large = sfc::ceil_div(M, 256) * sfc::ceil_div(N, 256) * experts;
  const bool big = 2 * large >= cus;
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
  return chunks > 1 ? (size_t)chunks * (size_t)experts * 4u : 0;
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
  const sfc::MoeRowsParams p = {tokens, rows, cols, topk, X, ldx, nullptr, 0, order, nullptr, weights, Xs, ldxs, nullptr};
  const hipError_t e = sfc::launch_moe_dispatch(p, type == SFC_OUT_BF16, cus, as_stream(stream));
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
  const sfc::MoeRowsParams p = {tokens, rows, cols, topk, Ys, ldys, nullptr, 0, nullptr, pos, weights, Y, ldy, nullptr};
  const hipError_t e = sfc::launch_moe_combine(p, type == SFC_OUT_BF16, cus, as_stream(stream));
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
  const sfc::MoeRowsParams p = {tokens, rows, cols, topk, dY, lddy, Ys, ldys, order, pos, weights, dYs, lddys, dW};
  const hipError_t e = sfc::launch_moe_combine_grad(p, type == SFC_OUT_BF16, cus, as_stream(stream));
  return e == hipSuccess ? SFC_OK : sfc::host_hip_error(e, "gradient of combine");
}

}  // extern "C"
