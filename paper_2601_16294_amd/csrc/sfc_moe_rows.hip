// Experts' bf16 products of few rows, C[p] = A[r(p)] B[e]^T (weights N x K), for gfx950.
//
// A workgroup streams 16 FN rows of one expert's weights past that expert's rows, 16 FM at a time: its 8 waves
// deal K out in blocks of 64, several of whose loads are in flight, straight into MFMA fragments, and add up
// through LDS in the order of the waves.  Bound: one read of the weights; the rows come from the caches.  32 tokens,
// 4 of 64 experts 2048x4096: 151 us, 6 to 7 TB/s of the weights of experts that have rows (as many as have any); 1 token, 2 of 8 experts
// 4096x4096: 17 to 20 us, 3.6 TB/s, half of it the launch and the first loads.  16 weight rows a workgroup where an expert has few
// rows: most workgroups and loads in flight; 32 where its rows are read for several fragments.
#include "sfc_launch.h"
#include "sfc_moe_gemm_kernel.h"
#include "sfc_row_io.h"

namespace sfc {

namespace {

constexpr int kWaves = 8;

__device__ __forceinline__ bf16x8 as_bf16x8(const row_u32x4& v) { return __builtin_bit_cast(bf16x8, v); }

template <int FM, int FN, bool GATHER, bool OB>
__global__ __launch_bounds__(kWaves * 64) void moe_rows_kernel(MoeGemmParams p) {
  constexpr int U = FM + FN <= 2 ? 4 : FM + FN <= 4 ? 2 : 1;             // blocks of K in flight
  __shared__ __attribute__((aligned(16))) float sums[kWaves][16 * FM][16 * FN + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * FN);
  const int e = blockIdx.y;
  const Segments seg = {p.offsets, p.experts, p.M};
  int64_t lo, hi;
  seg.bounds(e, lo, hi);
  const uint16_t* b[FN];                       // this lane's rows of the weights (past N: any, not kept)
#pragma unroll
  for (int j = 0; j < FN; ++j)
    b[j] = p.B + e * p.stride_b + (n0 + 16 * j + col < p.N ? n0 + 16 * j + col : p.N - 1) * p.ldb + 8 * g;
  for (int64_t m0 = lo; m0 < hi; m0 += 16 * FM) {
    const uint16_t* a[FM];                     // its rows of A (past the segment: any, not kept)
    bool none[FM];                             // a row of no slot: zeros
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t row = m0 + 16 * i + col < hi ? m0 + 16 * i + col : hi - 1;
      int64_t source = row;
      if constexpr (GATHER) {
        const int s = p.order[row];
        source = s < 0 ? -1 : s / p.topk;
        if (source >= p.a_rows) source = -1;
      }
      none[i] = source < 0;
      a[i] = p.A + (none[i] ? 0 : source) * p.lda + 8 * g;
    }
    f32x4 acc[FM][FN] = {};
    auto multiply = [&](const row_u32x4 (&av)[FM], const row_u32x4 (&bv)[FN]) {
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const row_u32x4 x = GATHER && none[i] ? row_u32x4{} : av[i];
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(bv[j]), as_bf16x8(x), acc[i][j], 0, 0, 0);
      }
    };
    auto blocks = [&](int64_t k, auto count) {
      constexpr int n = count;
      row_u32x4 av[n][2][FM], bv[n][2][FN];
#pragma unroll
      for (int u = 0; u < n; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int64_t at = k + u * (kWaves * 64) + 32 * s;
#pragma unroll
          for (int j = 0; j < FN; ++j) bv[u][s][j] = reinterpret_cast<const Any16<2>*>(b[j] + at)->v;
#pragma unroll
          for (int i = 0; i < FM; ++i) av[u][s][i] = reinterpret_cast<const Any16<2>*>(a[i] + at)->v;
        }
      __builtin_amdgcn_sched_barrier(0);       // (all loads are on their way first)
#pragma unroll
      for (int u = 0; u < n; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s) multiply(av[u][s], bv[u][s]);
    };
    int64_t k = (int64_t)wave * 64;
    if (p.a_rows > 0 || !GATHER) {
      for (; k + (U - 1) * (kWaves * 64) + 64 <= p.K; k += U * (kWaves * 64)) blocks(k, std::integral_constant<int, U>{});
      for (; k + 64 <= p.K; k += kWaves * 64) blocks(k, std::integral_constant<int, 1>{});
      if (k < p.K)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          row_u32x4 av[FM], bv[FN];
          const int64_t at = k + 32 * s + 8 * g;
#pragma unroll
          for (int j = 0; j < FN; ++j) bv[j] = load8<true>(b[j] - 8 * g, at, p.K).w[0];
#pragma unroll
          for (int i = 0; i < FM; ++i) av[i] = load8<true>(a[i] - 8 * g, at, p.K).w[0];
          multiply(av, bv);
        }
    }
    // lane: row l % 16, columns 4 (l / 16) .. + 3 of a fragment
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(&sums[wave][16 * i + col][16 * j + 4 * g]) = acc[i][j];
    __syncthreads();
    for (int i = tid; i < 16 * FM * 16 * FN; i += kWaves * 64) {
      const int row = i / (16 * FN), c = i % (16 * FN);
      if (m0 + row >= hi || n0 + c >= p.N) continue;
      float v = sums[0][row][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += sums[w][row][c];
      if constexpr (OB) reinterpret_cast<__bf16*>(p.C)[(m0 + row) * p.ldc + n0 + c] = (__bf16)v;
      else reinterpret_cast<float*>(p.C)[(m0 + row) * p.ldc + n0 + c] = v;
    }
    __syncthreads();
  }
  if (e != 0) return;
  // rows of no expert
  int used;
  seg.blocks<16>(lane, used);
  for (int64_t i = tid; i < (p.M - used) * (16 * FN); i += kWaves * 64) {
    const int64_t row = used + i / (16 * FN), c = n0 + i % (16 * FN);
    if (c >= p.N) continue;
    if constexpr (OB) reinterpret_cast<uint16_t*>(p.C)[row * p.ldc + c] = 0;
    else reinterpret_cast<uint32_t*>(p.C)[row * p.ldc + c] = 0;
  }
}

template <int FM, int FN>
hipError_t launch(const MoeGemmParams& p, bool ob, hipStream_t stream) {
  const dim3 grid((unsigned)((p.N + 16 * FN - 1) / (16 * FN)), (unsigned)p.experts), block(kWaves * 64);
  if (p.order) return launch_kernel(ob ? moe_rows_kernel<FM, FN, true, true> : moe_rows_kernel<FM, FN, true, false>, grid, block, 0, stream, p);
  return launch_kernel(ob ? moe_rows_kernel<FM, FN, false, true> : moe_rows_kernel<FM, FN, false, false>, grid, block, 0, stream, p);
}

}  // namespace

hipError_t launch_moe_rows(const MoeGemmParams& p, int fm, int fn, bool out_bf16, hipStream_t stream) {
  if (fm == 1 && fn == 1) return launch<1, 1>(p, out_bf16, stream);
  if (fm == 2 && fn == 2) return launch<2, 2>(p, out_bf16, stream);
  if (fm == 4 && fn == 2) return launch<4, 2>(p, out_bf16, stream);
  return hipErrorInvalidValue;
}

}  // namespace sfc
