// Microscaled 4-bit floating point: to 4 bits and back.
//
// A block of 32 values that lie side by side along the contraction shares one power
// of two, its scale code being s = max(field - 2, 0) where `field` is the exponent
// field of the largest magnitude as fp32 (that is 2^(floor(log2 max) - 2), at least
// 2^-127); an infinity or NaN in the block gives s = 255, which makes every value of
// the block NaN.  Elements are x / 2^(s-127) rounded to the nearest E2M1 value, ties
// to the even code, at most 6 in magnitude: the conversion instruction does the
// scaling, rounding and saturation (subnormal inputs and the scale 2^-127 included).
//
// Bound: memory.  Every value is read once, 17/32 byte written.
#include "sfc_ops_params.h"
#include "sfc_row_io.h"

namespace sfc {

typedef __bf16 qbf16x2 __attribute__((ext_vector_type(2)));
typedef float qf32x2 __attribute__((ext_vector_type(2)));

// The maximum over the 4 lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const uint32_t a = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
  v = v > a ? v : a;
  const uint32_t b = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);   // lanes 2 3 0 1
  return v > b ? v : b;
}

// Scale code of a block whose largest magnitude has the fp32 bits `top` (sign bit clear).
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
  const int field = (int)(top >> 23);
  return field == 255 ? 255u : (uint32_t)(field > 2 ? field - 2 : 0);
}
// The scale as fp32.  255: any finite number (the block is NaN whatever its codes).
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __builtin_bit_cast(float, s == 255 ? 127u << 23 : s == 0 ? 1u << 22 : s << 23);
}

// Largest magnitude (as fp32 bits) of eight elements: magnitudes order as their bits do,
// NaN above all.
template <bool BF16>
__device__ __forceinline__ uint32_t top8(const Raw8<BF16>& r) {
  uint32_t m = 0;
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = (r.w[0][i] << 16) & 0x7FFFFFFFu, hi = r.w[0][i] & 0x7FFF0000u;
      m = m > lo ? m : lo;
      m = m > hi ? m : hi;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t v = r.w[i >> 2][i & 3] & 0x7FFFFFFFu;
      m = m > v ? m : v;
    }
  }
  return m;
}

// Codes of eight elements, the first in the low bits.
template <bool BF16>
__device__ __forceinline__ uint32_t codes8(const Raw8<BF16>& r, float scale) {
  uint32_t q = 0;
  if constexpr (BF16) {
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][0]), scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][1]), scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][2]), scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][3]), scale, 3);
  } else {
    float f[8];
    to_float<BF16>(r, f);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[0], f[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[2], f[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[4], f[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[6], f[7], scale, 3);
  }
  return q;
}

// Row p of the matrix to quantise, or null: a row of zeros.
template <bool BF16>
__device__ __forceinline__ const char* source_row(const Mx4QuantParams& p, int64_t row) {
  int64_t r = row;
  if (p.order) {
    const int32_t slot = p.order[row];
    r = slot < 0 ? -1 : (int64_t)((uint32_t)slot / (uint32_t)p.topk);
  }
  if (r < 0 || r >= p.x_rows) return nullptr;
  return reinterpret_cast<const char*>(p.X) + r * p.ldx * (BF16 ? 2 : 4);
}

// Blocks along the columns.  A lane takes eight values, four lanes a block.
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quant_rows_kernel(Mx4QuantParams p, RowShape sh) {
  const int tx = 1 << sh.tx_log2;
  const int64_t rb = blockIdx.x / sh.splits;
  const int split = (int)(blockIdx.x - rb * sh.splits);
  const int64_t row = rb * (256 >> sh.tx_log2) + (threadIdx.x >> sh.tx_log2);
  if (row >= p.rows) return;
  const int64_t blocks = (p.cols + 31) >> 5, chunks = blocks * 4;
  const int64_t first = (int64_t)split * sh.per;
  const int64_t last = first + sh.per < chunks ? first + sh.per : chunks;
  const char* src = source_row<BF16>(p, row);
  uint8_t* q = p.Q + row * p.ldq;
  uint8_t* s = p.S + row * p.lds;
  const int lane_tx = threadIdx.x & (tx - 1);
  // the first and last chunk are multiples of 4, so a block's four lanes stay together
  for (int64_t c = first + lane_tx; c < last; c += tx) {
    const Raw8<BF16> r = src ? load8<BF16>(src, c * 8, p.cols) : zero8<BF16>();
    const uint32_t sc = scale_code(quad_max(top8<BF16>(r)));
    *reinterpret_cast<uint32_t*>(q + c * 4) = codes8<BF16>(r, scale_value(sc));
    if ((lane_tx & 3) == 0) s[c >> 2] = (uint8_t)sc;
  }
}

// Blocks along the rows, the result transposed.  A workgroup takes 256 rows x 128
// columns: a lane holds 32 rows of two columns in registers, so a block's maximum needs
// no other lane; the codes of eight blocks of a column meet in LDS and leave as one
// 128-byte line of the transposed matrix.
constexpr int kQtCols = 128, kQtStride = 144;        // LDS bytes from one column to the next
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quant_cols_kernel(Mx4QuantParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t codes[kQtCols * kQtStride];
  __shared__ __attribute__((aligned(16))) uint8_t scales[kQtCols * 8];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t col_blocks = (p.cols + kQtCols - 1) / kQtCols;
  const int64_t rg = blockIdx.x / col_blocks, cb = blockIdx.x - rg * col_blocks;
  const int64_t c0 = cb * kQtCols, c = c0 + 2 * lane;
  const int64_t blocks = (p.rows + 31) >> 5;
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    const int b = 2 * wave + half;
    const int64_t r0 = rg * 256 + 32 * b;
    uint32_t v[2][32];                   // fp32 bits of the two columns
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      v[0][i] = 0;
      v[1][i] = 0;
      const char* src = r0 + i < p.rows ? source_row<BF16>(p, r0 + i) : nullptr;
      if (src) {
        if constexpr (BF16) {
          const uint16_t* e = reinterpret_cast<const uint16_t*>(src) + c;
          if (c + 1 < p.cols) {
            struct __attribute__((packed, aligned(2))) Pair { uint32_t v; };
            const uint32_t w = reinterpret_cast<const Pair*>(e)->v;
            v[0][i] = w << 16;
            v[1][i] = w & 0xFFFF0000u;
          } else if (c < p.cols) {
            v[0][i] = (uint32_t)e[0] << 16;
          }
        } else {
          const uint32_t* e = reinterpret_cast<const uint32_t*>(src) + c;
          if (c + 1 < p.cols) {
            struct __attribute__((packed, aligned(4))) Pair { uint32_t v[2]; };
            const Pair w = *reinterpret_cast<const Pair*>(e);
            v[0][i] = w.v[0];
            v[1][i] = w.v[1];
          } else if (c < p.cols) {
            v[0][i] = e[0];
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const uint32_t m = v[k][i] & 0x7FFFFFFFu;
        top = top > m ? top : m;
      }
      const uint32_t sc = scale_code(top);
      const float scale = scale_value(sc);
      row_u32x4 q;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t x = 0;
#define SFC_CVT(n)                                                                                                  \
  x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, __builtin_bit_cast(float, v[k][8 * w + 2 * n]),                   \
                                               __builtin_bit_cast(float, v[k][8 * w + 2 * n + 1]), scale, n)
        SFC_CVT(0);
        SFC_CVT(1);
        SFC_CVT(2);
        SFC_CVT(3);
#undef SFC_CVT
        q[w] = x;
      }
      *reinterpret_cast<row_u32x4*>(codes + (2 * lane + k) * kQtStride + 16 * b) = q;
      scales[(2 * lane + k) * 8 + b] = (uint8_t)sc;
    }
  }
  __syncthreads();
  const int64_t b0 = rg * 8;
  for (int i = tid; i < kQtCols * 8; i += 256) {
    const int col = i >> 3, b = i & 7;
    if (c0 + col < p.cols && b0 + b < blocks) {
      *reinterpret_cast<row_u32x4*>(p.Qt + (c0 + col) * p.ldqt + (b0 + b) * 16) =
          *reinterpret_cast<const row_u32x4*>(codes + col * kQtStride + 16 * b);
      p.St[(c0 + col) * p.ldst + b0 + b] = scales[col * 8 + b];
    }
  }
}

hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool in_bf16, int num_cus, hipStream_t stream) {
  if (p.Q) {
    const RowShape sh = row_shape(p.rows, (p.cols + 31) / 32 * 4, num_cus);
    const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
    if (in_bf16) hipLaunchKernelGGL((mx4_quant_rows_kernel<true>), g, b, 0, stream, p, sh);
    else hipLaunchKernelGGL((mx4_quant_rows_kernel<false>), g, b, 0, stream, p, sh);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.Qt) {
    const dim3 g((unsigned)(((p.rows + 255) / 256) * ((p.cols + kQtCols - 1) / kQtCols))), b(256);
    if (in_bf16) hipLaunchKernelGGL((mx4_quant_cols_kernel<true>), g, b, 0, stream, p);
    else hipLaunchKernelGGL((mx4_quant_cols_kernel<false>), g, b, 0, stream, p);
    return hipGetLastError();
  }
  return hipSuccess;
}

// ---- back to fp32 or bf16 ----------------------------------------------------------------

// Eight codes (low bits first) times the scale.
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> values8(uint32_t q, uint32_t s) {
  Raw8<BF16> r;
  if (s == 255) {
    r.w[0] = BF16 ? row_u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u}
                  : row_u32x4{0x7FC00000u, 0x7FC00000u, 0x7FC00000u, 0x7FC00000u};
    if constexpr (!BF16) r.w[1] = r.w[0];
    return r;
  }
  const float scale = scale_value(s);
  qf32x2 f[4];
  f[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 0);
  f[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 1);
  f[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 2);
  f[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 3);
  const float v[8] = {f[0][0], f[0][1], f[1][0], f[1][1], f[2][0], f[2][1], f[3][0], f[3][1]};
  return from_float<BF16>(v);
}

template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequant_kernel(Mx4DequantParams p, RowShape sh) {
  const int tx = 1 << sh.tx_log2;
  const int64_t rb = blockIdx.x / sh.splits;
  const int split = (int)(blockIdx.x - rb * sh.splits);
  const int64_t row = rb * (256 >> sh.tx_log2) + (threadIdx.x >> sh.tx_log2);
  if (row >= p.rows) return;
  const int64_t chunks = (p.cols + 7) >> 3;
  const int64_t first = (int64_t)split * sh.per;
  const int64_t last = first + sh.per < chunks ? first + sh.per : chunks;
  const uint8_t* q = p.Q + row * p.ldq;
  const uint8_t* s = p.S + row * p.lds;
  char* y = reinterpret_cast<char*>(p.Y) + row * p.ldy * (BF16 ? 2 : 4);
  for (int64_t c = first + (threadIdx.x & (tx - 1)); c < last; c += tx)
    store8<BF16>(y, c * 8, p.cols, values8<BF16>(*reinterpret_cast<const uint32_t*>(q + c * 4), s[c >> 2]));
}

hipError_t launch_mx4_dequant(const Mx4DequantParams& p, bool out_bf16, int num_cus, hipStream_t stream) {
  const RowShape sh = row_shape(p.rows, (p.cols + 7) / 8, num_cus);
  const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
  if (out_bf16) hipLaunchKernelGGL((mx4_dequant_kernel<true>), g, b, 0, stream, p, sh);
  else hipLaunchKernelGGL((mx4_dequant_kernel<false>), g, b, 0, stream, p, sh);
  return hipGetLastError();
}

}  // namespace sfc
