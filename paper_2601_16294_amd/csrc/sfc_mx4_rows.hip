// Products of few rows with 4-bit weights, C = A B^T (a decode step's tokens, or the few
// rows of each expert): the calls whose time is one read of B.
//
// A workgroup computes 16*FN columns (rows of B) for 16*FM rows of A at a time.  Its waves
// deal K out between them, 512 values a turn: a turn reads 256 bytes of codes and 16 bytes
// of scales of every row straight into registers, all loads of a turn in flight at once,
// then runs 4 MFMA 16x16x128 per fragment pair.  The waves' partial blocks are added in
// LDS, ascending, in fp32.  Lane l holds row l%16 and block l/16 of a 128-value step.
//
// Rows and blocks outside the matrices load zeros (lanes past the descriptors' range);
// their scale bytes are masked to code 0, because a NaN scale makes even zeros NaN.
#include "sfc_gemm_kernel.h"
#include "sfc_ops_params.h"

namespace sfc {

constexpr int kTurn = 512;           // values of K that a wave takes at a time

__device__ __forceinline__ i32x4 load16_range(__amdgpu_buffer_rsrc_t rsrc, int voffset) {
  return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, voffset, 0, 0));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* base, int range) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, range, 0x00020000);
}
__device__ __forceinline__ i32x8 rows_wide(const i32x4& v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}

template <int FM, int FN, bool OB>
__device__ __forceinline__ void rows_block(const Mx4GemmParams& p, const uint8_t* B, const uint8_t* Bs, int64_t a_row,
                                           int m_valid, int64_t n0, float* part) {
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;
  const int n_valid = p.N - n0 < 16 * FN ? (int)(p.N - n0) : 16 * FN;
  const int blocks = (int)(p.K >> 5), turns = (blocks + 15) >> 4;
  const int s_end = (blocks + 3) & ~3;
  const __amdgpu_buffer_rsrc_t qa = rows_rsrc(p.A + a_row * p.lda, kOobOffset);
  const __amdgpu_buffer_rsrc_t qb = rows_rsrc(B + n0 * p.ldb, kOobOffset);
  const __amdgpu_buffer_rsrc_t ca = rows_rsrc(p.As + a_row * p.ldas, (int)((m_valid - 1) * p.ldas) + s_end);
  const __amdgpu_buffer_rsrc_t cb = rows_rsrc(Bs + n0 * p.ldbs, (int)((n_valid - 1) * p.ldbs) + s_end);
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int turn = wave; turn < turns; turn += waves) {
    i32x4 fb[FN][4], fa[FM][4], sb[FN], sa[FM];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int r = 16 * j + r16;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int blk = 16 * turn + 4 * u + g;
        fb[j][u] = load16_range(qb, r < n_valid && blk < blocks ? (int)(r * p.ldb) + 16 * blk : kOobOffset);
      }
      sb[j] = load16_range(cb, r < n_valid ? (int)(r * p.ldbs) + 16 * turn : kOobOffset);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int r = 16 * i + r16;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int blk = 16 * turn + 4 * u + g;
        fa[i][u] = load16_range(qa, r < m_valid && blk < blocks ? (int)(r * p.lda) + 16 * blk : kOobOffset);
      }
      sa[i] = load16_range(ca, r < m_valid ? (int)(r * p.ldas) + 16 * turn : kOobOffset);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int mask = 16 * turn + 4 * u + g < blocks ? 0xFF : 0;
      int xa[FM], xb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) xa[i] = (int)((uint32_t)sa[i][u] >> (8 * g)) & mask;
#pragma unroll
      for (int j = 0; j < FN; ++j) xb[j] = (int)((uint32_t)sb[j][u] >> (8 * g)) & mask;
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(rows_wide(fb[j][u]), rows_wide(fa[i][u]), acc[i][j],
                                                                       4, 4, 0, xb[j], 0, xa[i]);
    }
  }

  // the waves' partial blocks: [wave][row of A][16 * FN columns]
  constexpr int ROWS = 16 * FM, COLS = 16 * FN;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<f32x4*>(part + ((wave * ROWS + 16 * i + r16) * COLS + 16 * j + 4 * g)) = acc[i][j];
  __syncthreads();
  for (int e = threadIdx.x; e < ROWS * COLS / 4; e += blockDim.x) {
    const int row = e / (COLS / 4), col = (e % (COLS / 4)) * 4;
    f32x4 s = *reinterpret_cast<const f32x4*>(part + row * COLS + col);
    for (int w = 1; w < waves; ++w) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(part + (w * ROWS + row) * COLS + col);
      s[0] += v[0]; s[1] += v[1]; s[2] += v[2]; s[3] += v[3];
    }
    if (row < m_valid) {
      const int64_t at = (a_row + row) * p.ldc + n0 + col;
      if constexpr (OB) {
        struct __attribute__((packed, aligned(2))) Any { bf16x4 v; };
        __bf16* dst = reinterpret_cast<__bf16*>(p.C) + at;
        const bf16x4 b = {(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
        if (col + 4 <= n_valid) reinterpret_cast<Any*>(dst)->v = b;
        else
#pragma unroll
          for (int k = 0; k < 3; ++k)
            if (col + k < n_valid) dst[k] = b[k];
      } else {
        struct __attribute__((packed, aligned(4))) Any { f32x4 v; };
        float* dst = reinterpret_cast<float*>(p.C) + at;
        if (col + 4 <= n_valid) reinterpret_cast<Any*>(dst)->v = s;
        else
#pragma unroll
          for (int k = 0; k < 3; ++k)
            if (col + k < n_valid) dst[k] = s[k];
      }
    }
  }
}

template <int FM, int FN, bool OB, bool GROUPED>
__global__ __launch_bounds__(512) void mx4_rows_kernel(Mx4GemmParams p) {
  extern __shared__ __attribute__((aligned(16))) float part[];
  if constexpr (!GROUPED) {
    const int64_t n0 = (int64_t)blockIdx.x * 16 * FN;
    for (int64_t m0 = 0; m0 < p.M; m0 += 16 * FM) {
      if (m0 > 0) __syncthreads();
      rows_block<FM, FN, OB>(p, p.B, p.Bs, m0, p.M - m0 < 16 * FM ? (int)(p.M - m0) : 16 * FM, n0, part);
    }
  } else {
    const int e = blockIdx.x / p.gn, in = blockIdx.x - e * p.gn;
    int64_t lo = p.offsets[e], hi = p.offsets[e + 1];
    lo = lo < 0 ? 0 : lo > p.M ? p.M : lo;
    hi = hi < lo ? lo : hi > p.M ? p.M : hi;
    for (int64_t m0 = lo; m0 < hi; m0 += 16 * FM) {
      if (m0 > lo) __syncthreads();
      rows_block<FM, FN, OB>(p, p.B + (int64_t)e * p.stride_b, p.Bs + (int64_t)e * p.stride_bs, m0,
                             hi - m0 < 16 * FM ? (int)(hi - m0) : 16 * FM, (int64_t)in * 16 * FN, part);
    }
    // rows of no expert, cleared by the workgroups of the last one: from the end of the last
    // segment on
    if (e == p.experts - 1) {
      int* end_at = reinterpret_cast<int*>(part);
      __syncthreads();
      if (threadIdx.x == 0) *end_at = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < p.experts; i += blockDim.x) {
        int64_t from = p.offsets[i], to = p.offsets[i + 1];
        from = from < 0 ? 0 : from > p.M ? p.M : from;
        to = to < from ? from : to > p.M ? p.M : to;
        atomicMax(end_at, (int)to);
      }
      __syncthreads();
      for (int64_t r = (int64_t)*end_at + in; r < p.M; r += p.gn)
        for (int64_t c = threadIdx.x; c < p.N; c += blockDim.x) {
          if constexpr (OB) reinterpret_cast<uint16_t*>(p.C)[r * p.ldc + c] = 0;
          else reinterpret_cast<uint32_t*>(p.C)[r * p.ldc + c] = 0;
        }
    }
  }
}

template <int FM, int FN>
static hipError_t rows_launch(const Mx4GemmParams& p, Mx4Mode mode, int waves, bool ob, hipStream_t stream) {
  Mx4GemmParams q = p;
  q.gn = (int)((p.N + 16 * FN - 1) / (16 * FN));
  const bool grouped = mode == kMxRows;
  const void* k = grouped ? (ob ? reinterpret_cast<const void*>(&mx4_rows_kernel<FM, FN, true, true>)
                                : reinterpret_cast<const void*>(&mx4_rows_kernel<FM, FN, false, true>))
                          : (ob ? reinterpret_cast<const void*>(&mx4_rows_kernel<FM, FN, true, false>)
                                : reinterpret_cast<const void*>(&mx4_rows_kernel<FM, FN, false, false>));
  const unsigned grid = (unsigned)q.gn * (grouped ? (unsigned)p.experts : 1u);
  void* args[] = {&q};
  return hipLaunchKernel(k, dim3(grid), dim3(64u * (unsigned)waves), args, (size_t)waves * 256 * FM * FN * 4, stream);
}

hipError_t launch_mx4_rows(const Mx4GemmParams& p, Mx4Mode mode, int fm, int fn, int waves, bool out_bf16,
                           hipStream_t stream) {
  if (fm == 1) return fn == 1 ? rows_launch<1, 1>(p, mode, waves, out_bf16, stream)
                              : rows_launch<1, 2>(p, mode, waves, out_bf16, stream);
  if (fm == 2) return rows_launch<2, 2>(p, mode, waves, out_bf16, stream);
  return rows_launch<4, 2>(p, mode, waves, out_bf16, stream);
}

}  // namespace sfc
