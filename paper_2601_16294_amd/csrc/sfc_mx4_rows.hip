// Products of few rows with 4-bit weights, C = A B^T (a decode step's tokens, or the few
// rows of each expert): the calls whose time is one read of B.  16x14336x4096: 9.0 us
// (3.5 TB/s: 2 us of launch and the first loads' way, then 31 MB), 16x16384x16384 26.8 (5.3,
// about the rate at which memory is read here at best).
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
#include "sfc_mx4_convert.h"
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

// Columns col .. col + 3 of a row of C, of which `left` are inside it.
template <bool OB>
__device__ __forceinline__ void rows_store(const Mx4GemmParams& p, int64_t row, int64_t col, int left, const f32x4& s) {
  const int64_t at = row * p.ldc + col;
  if constexpr (OB) {
    struct __attribute__((packed, aligned(2))) Any { bf16x4 v; };
    __bf16* dst = reinterpret_cast<__bf16*>(p.C) + at;
    const bf16x4 b = {(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
    if (left >= 4) reinterpret_cast<Any*>(dst)->v = b;
    else
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < left) dst[k] = b[k];
  } else {
    struct __attribute__((packed, aligned(4))) Any { f32x4 v; };
    float* dst = reinterpret_cast<float*>(p.C) + at;
    if (left >= 4) reinterpret_cast<Any*>(dst)->v = s;
    else
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < left) dst[k] = s[k];
  }
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
    if (row < m_valid) rows_store<OB>(p, a_row + row, n0 + col, n_valid - col, s);
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

// ---- up to 16 rows ---------------------------------------------------------------------------
// As above for one fragment of A, which stays: a wave keeps its TPW turns of A in
// registers, as codes or brought to 4 bits on the way in (a lane's 32 values of a block are
// its own), and the workgroup runs over several blocks of columns, the loads of the next one
// going out as the registers of this one are used.
// The block of 32 values from column `col` of a row (null: zeros) as codes and a scale code.
template <bool BF16>
__device__ __forceinline__ i32x4 rows_convert(const Raw8<BF16> (&r)[4], int& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = top8<BF16>(r[i]);
    top = top > m ? top : m;
  }
  const uint32_t s = scale_code(top);
  i32x4 q;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = (int)codes8<BF16>(r[i], scale_value(s));
  scale = (int)s;
  return q;
}

template <int FN, bool OB, int XT, int TPW>
__global__ __launch_bounds__(512) void mx4_few_kernel(Mx4GemmParams p, int blocks_per_group) {
  extern __shared__ __attribute__((aligned(16))) float part[];       // [2][waves][16][16 * FN]
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;
  const int blocks = (int)((p.K + 31) >> 5), s_end = (blocks + 3) & ~3;
  constexpr int COLS = 16 * FN;
  constexpr bool XB = XT == kRowsBf16;
  const int64_t all = (p.N + COLS - 1) / COLS;
  const int64_t nb0 = (int64_t)blockIdx.x * blocks_per_group;
  const int64_t nb1 = nb0 + blocks_per_group < all ? nb0 + blocks_per_group : all;

  i32x4 fb[TPW][FN][4], sb[TPW][FN];
  auto load_b = [&](int64_t nb, int k) {
    const int64_t n0 = nb * COLS;
    const int n_valid = nb < nb1 ? (p.N - n0 < COLS ? (int)(p.N - n0) : COLS) : 0;
    const int64_t row0 = nb < nb1 ? n0 : 0;
    const __amdgpu_buffer_rsrc_t qb = rows_rsrc(p.B + row0 * p.ldb, kOobOffset);
    const __amdgpu_buffer_rsrc_t cb = rows_rsrc(p.Bs + row0 * p.ldbs, n_valid > 0 ? (int)((n_valid - 1) * p.ldbs) + s_end : 0);
    const int turn = wave + k * waves;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int r = 16 * j + r16;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int blk = 16 * turn + 4 * u + g;
        fb[k][j][u] = load16_range(qb, r < n_valid && blk < blocks ? (int)(r * p.ldb) + 16 * blk : kOobOffset);
      }
      sb[k][j] = load16_range(cb, r < n_valid && 16 * turn < blocks ? (int)(r * p.ldbs) + 16 * turn : kOobOffset);
    }
  };
  // A before B: loads return in order, and A comes from nearby
  i32x4 fa[TPW][4];
  int xa[TPW];               // scale bytes (byte u: this lane's block of step u; 0 outside the range)
  if constexpr (XT == kRowsCodes) {
    const __amdgpu_buffer_rsrc_t qa = rows_rsrc(p.A, kOobOffset);
    const __amdgpu_buffer_rsrc_t ca = rows_rsrc(p.As, (int)((p.M - 1) * p.ldas) + s_end);
    i32x4 s[TPW];
#pragma unroll
    for (int k = 0; k < TPW; ++k) {
      const int turn = wave + k * waves;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int blk = 16 * turn + 4 * u + g;
        fa[k][u] = load16_range(qa, r16 < p.M && blk < blocks ? (int)(r16 * p.lda) + 16 * blk : kOobOffset);
      }
      s[k] = load16_range(ca, r16 < p.M && 16 * turn < blocks ? (int)(r16 * p.ldas) + 16 * turn : kOobOffset);
    }
#pragma unroll
    for (int k = 0; k < TPW; ++k) load_b(nb0, k);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < TPW; ++k) {
      xa[k] = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (16 * (wave + k * waves) + 4 * u + g < blocks) xa[k] |= (int)(((uint32_t)s[k][u] >> (8 * g)) & 0xFF) << (8 * u);
    }
  } else {
    static_assert(TPW == 1, "rows are brought to 4 bits a turn at a time");
    constexpr int ES = XB ? 2 : 4;
    Raw8<XB> raw[4][4];
    const int64_t reach = 15 * p.ldx * ES + p.x_cols * ES;
    if (p.x_cols % 8 == 0 && reach < kOobOffset) {
      // whole chunks: one load each, zeros past the descriptor's range
      const __amdgpu_buffer_rsrc_t qx = rows_rsrc(reinterpret_cast<const uint8_t*>(p.X), kOobOffset);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int col = 32 * (16 * wave + 4 * u + g);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int at = r16 < p.M && col + 8 * c < p.x_cols ? (int)(r16 * p.ldx * ES) + (col + 8 * c) * ES : kOobOffset;
          raw[u][c].w[0] = __builtin_bit_cast(row_u32x4, load16_range(qx, at));
          if constexpr (!XB) raw[u][c].w[1] = __builtin_bit_cast(row_u32x4, load16_range(qx, at == kOobOffset ? at : at + 16));
        }
      }
    } else {
      const char* row = reinterpret_cast<const char*>(p.X) + r16 * p.ldx * ES;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t col = 32 * (int64_t)(16 * wave + 4 * u + g);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          raw[u][c] = r16 < p.M && col + 8 * c < p.x_cols ? load8<XB>(row, col + 8 * c, p.x_cols) : zero8<XB>();
      }
    }
    load_b(nb0, 0);
    __builtin_amdgcn_sched_barrier(0);
    xa[0] = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      int s;
      fa[0][u] = rows_convert<XB>(raw[u], s);
      xa[0] |= s << (8 * u);
    }
  }

  int flip = 0;
  for (int64_t nb = nb0; nb < nb1; ++nb, flip ^= 1) {
    f32x4 acc[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < TPW; ++k) {
      const int turn = wave + k * waves;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int mask = 16 * turn + 4 * u + g < blocks ? 0xFF : 0;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int xb = (int)((uint32_t)sb[k][j][u] >> (8 * g)) & mask;
          const i32x8 b = rows_wide(fb[k][j][u]), a = rows_wide(fa[k][u]);
          if (u == 0) acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc[j], 4, 4, 0, xb, 0, xa[k]);
          if (u == 1) acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc[j], 4, 4, 0, xb, 1, xa[k]);
          if (u == 2) acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc[j], 4, 4, 0, xb, 2, xa[k]);
          if (u == 3) acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc[j], 4, 4, 0, xb, 3, xa[k]);
        }
      }
      load_b(nb + 1, k);
    }
    // the waves' partial blocks, ascending; two buffers in turn: one barrier a block
    float* mine = part + flip * waves * 16 * COLS;
#pragma unroll
    for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(mine + (wave * 16 + r16) * COLS + 16 * j + 4 * g) = acc[j];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int64_t n0 = nb * COLS;
    const int row = threadIdx.x / (COLS / 4), col = (threadIdx.x % (COLS / 4)) * 4;
    if (row < p.M && row < 16) {
      f32x4 s = *reinterpret_cast<const f32x4*>(mine + row * COLS + col);
      for (int w = 1; w < waves; ++w) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(mine + (w * 16 + row) * COLS + col);
        s[0] += v[0]; s[1] += v[1]; s[2] += v[2]; s[3] += v[3];
      }
      rows_store<OB>(p, row, n0 + col, (int)(p.N - n0 < COLS ? p.N - n0 : COLS) - col, s);
    }
  }
}

template <int FN, bool OB>
static const void* few_kernel(Mx4Rows rows, int tpw) {
  if (rows == kRowsBf16) return reinterpret_cast<const void*>(&mx4_few_kernel<FN, OB, kRowsBf16, 1>);
  if (rows == kRowsF32) return reinterpret_cast<const void*>(&mx4_few_kernel<FN, OB, kRowsF32, 1>);
  if constexpr (FN == 1)
    if (tpw == 4) return reinterpret_cast<const void*>(&mx4_few_kernel<FN, OB, kRowsCodes, 4>);
  return tpw == 1 ? reinterpret_cast<const void*>(&mx4_few_kernel<FN, OB, kRowsCodes, 1>)
                  : reinterpret_cast<const void*>(&mx4_few_kernel<FN, OB, kRowsCodes, 2>);
}

// Whole blocks of columns to a workgroup, as few as put at most one workgroup on a CU: 14336 columns
// are 224 workgroups of two blocks each, and 32 CUs have none.  (us, that / up to two workgroups to a CU,
// 448 there, weights in rotation: 16x14336x4096 9.3 / 11.0, 16x11008x4096 10.0 / 10.8, 16x28672x4096
// 16.6 / 18.2.)
template <int FN>
static hipError_t few_launch(const Mx4GemmParams& p, Mx4Rows rows, int num_cus, bool ob, hipStream_t stream) {
  const int64_t turns = (p.K + kTurn - 1) / kTurn;
  const int waves = turns <= 4 ? 4 : 8;
  const int tpw = turns <= waves ? 1 : turns <= 2 * waves ? 2 : 4;
  const void* k = ob ? few_kernel<FN, true>(rows, tpw) : few_kernel<FN, false>(rows, tpw);
  const int64_t all = (p.N + 16 * FN - 1) / (16 * FN);
  int per = (int)((all + num_cus - 1) / num_cus);
  Mx4GemmParams q = p;
  void* args[] = {&q, &per};
  return hipLaunchKernel(k, dim3((unsigned)((all + per - 1) / per)), dim3(64u * (unsigned)waves), args,
                         (size_t)2 * waves * 256 * FN * 4, stream);
}

hipError_t launch_mx4_few(const Mx4GemmParams& p, Mx4Rows rows, int num_cus, bool out_bf16, hipStream_t stream) {
  // blocks of 32 columns where they fill the chip (and the turns of one wave leave the registers)
  const bool wide = (p.N + 31) / 32 >= num_cus && p.K <= 16 * kTurn;
  return wide ? few_launch<2>(p, rows, num_cus, out_bf16, stream) : few_launch<1>(p, rows, num_cus, out_bf16, stream);
}

// ---- launches ----------------------------------------------------------------------------------
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

hipError_t launch_mx4_rows(const Mx4GemmParams& p, Mx4Mode mode, int fm, bool narrow, bool out_bf16, hipStream_t stream) {
  const int waves = p.K >= 8 * kTurn ? 8 : 4;
  if (fm == 1) return narrow ? rows_launch<1, 1>(p, mode, waves, out_bf16, stream)
                             : rows_launch<1, 2>(p, mode, waves, out_bf16, stream);
  if (fm == 2) return rows_launch<2, 2>(p, mode, waves, out_bf16, stream);
  return rows_launch<4, 2>(p, mode, waves, out_bf16, stream);
}

}  // namespace sfc
