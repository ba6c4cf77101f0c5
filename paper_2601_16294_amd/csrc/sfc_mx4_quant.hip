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
#include "sfc_mx4_convert.h"

namespace sfc {

// The maximum over the 4 lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const uint32_t a = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
  v = v > a ? v : a;
  const uint32_t b = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);   // lanes 2 3 0 1
  return v > b ? v : b;
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

// Blocks along the rows of X.  A lane takes eight values, four lanes a block.
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quant_rows_kernel(Mx4QuantParams p, RowShape sh) {
  const RowPlace at = row_place(sh, (p.cols + 31) / 32 * 4);
  if (at.row >= p.rows) return;
  const char* src = source_row<BF16>(p, at.row);
  uint8_t* q = p.Q + at.row * p.ldq;
  uint8_t* s = p.S + at.row * p.lds;
  // the first and last chunk are multiples of 4, so a block's four lanes stay together
  constexpr int U = 4;
  Raw8<BF16> r[U];
  row_loop<U>(
      at, [&](int u, int64_t c) { r[u] = src ? load8<BF16>(src, c * 8, p.cols) : zero8<BF16>(); },
      [&](int u, int64_t c) {
        const uint32_t sc = scale_code(quad_max(top8<BF16>(r[u])));
        *reinterpret_cast<uint32_t*>(q + c * 4) = codes8<BF16>(r[u], scale_value(sc));
        if ((at.lane_tx & 3) == 0) s[c >> 2] = (uint8_t)sc;
      });
}

// Blocks along the columns, the result transposed, and (BOTH) blocks along the rows from
// the same read.  A workgroup of 8 waves takes 256 rows x 128 columns: a lane holds 32 rows
// of two columns in registers, so a column block's maximum needs no other lane, and a row
// block is 16 lanes.  Codes and scales meet in LDS and leave as 128-byte (64-byte: rows)
// pieces.
constexpr int kQtCols = 128, kQtStride = 144;        // LDS bytes from one column to the next

typedef uint16_t q_u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(q_u16x2, a), __builtin_bit_cast(q_u16x2, b)));
}
// The maxima of both halves over the 16 lanes of a row of lanes.
__device__ __forceinline__ uint32_t row16_max16x2(uint32_t v) {
  v = max16x2(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
  v = max16x2(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1
  v = max16x2(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true));     // mirrored in 8
  return max16x2(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true));  // mirrored in 16
}
// Scale code from the upper 16 bits of the largest magnitude (its exponent field is all that counts).
__device__ __forceinline__ uint32_t scale_code16(uint32_t top) { return scale_code(top << 16); }

template <bool BF16, bool BOTH>
__global__ __launch_bounds__(512, 4) void mx4_quant_cols_kernel(Mx4QuantParams p, int row_groups) {
  __shared__ __attribute__((aligned(16))) uint8_t codes[kQtCols * kQtStride];
  __shared__ __attribute__((aligned(16))) uint8_t scales[kQtCols * 8];
  __shared__ __attribute__((aligned(16))) uint32_t row_codes[BOTH ? 64 * 64 : 4];    // [4 rows][2 columns]: a byte a row
  __shared__ __attribute__((aligned(16))) uint8_t row_scales[BOTH ? 256 * 4 : 16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col_groups = gridDim.x / (unsigned)row_groups;
  const int rg = blockIdx.x / (unsigned)col_groups, cb = blockIdx.x - rg * col_groups;
  const int64_t c0 = (int64_t)cb * kQtCols, c = c0 + 2 * lane;
  const int64_t r0 = (int64_t)rg * 256 + 32 * wave;
  // the wave's 32 source rows (-1: zeros), all loads before any use
  int source = -1;
  if (lane < 32 && r0 + lane < p.rows) {
    source = (int)(r0 + lane);
    if (p.order) {
      const int32_t slot = p.order[r0 + lane];
      source = slot < 0 ? -1 : (int)((uint32_t)slot / (uint32_t)p.topk);
    }
    if (source >= p.x_rows) source = -1;
  }
  constexpr int ES = BF16 ? 2 : 4;
  // as stored: both columns of a row in a word, or (fp32) a word each
  uint32_t raw[BF16 ? 1 : 2][32];
#pragma unroll
  for (int i = 0; i < 32; ++i) raw[0][i] = raw[BF16 ? 0 : 1][i] = 0;
  if (p.x_rows > 0 && c < p.cols) {
    const char* x = reinterpret_cast<const char*>(p.X) + c * ES;
    if (c + 1 < p.cols) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int r = __builtin_amdgcn_readlane(source, i);
        struct __attribute__((packed, aligned(ES))) Pair { uint32_t v[BF16 ? 1 : 2]; };
        const Pair w = *reinterpret_cast<const Pair*>(x + (int64_t)(r < 0 ? 0 : r) * p.ldx * ES);
        raw[0][i] = w.v[0];
        if constexpr (!BF16) raw[1][i] = w.v[1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int r = __builtin_amdgcn_readlane(source, i);
        const char* e = x + (int64_t)(r < 0 ? 0 : r) * p.ldx * ES;
        raw[0][i] = BF16 ? *reinterpret_cast<const uint16_t*>(e) : *reinterpret_cast<const uint32_t*>(e);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const bool zero = __builtin_amdgcn_readlane(source, i) < 0;
#pragma unroll
    for (int k = 0; k < (BF16 ? 1 : 2); ++k) raw[k][i] = zero ? 0u : raw[k][i];
  }
  // row i of column k as fp32, and the upper halves of the row's magnitudes
  auto value = [&](int k, int i) {
    return __builtin_bit_cast(float, !BF16 ? raw[BF16 ? 0 : k][i] : k ? raw[0][i] & 0xFFFF0000u : raw[0][i] << 16);
  };
  auto mag = [&](int i) {
    return (BF16 ? raw[0][i] : (raw[0][i] >> 16) | (raw[BF16 ? 0 : 1][i] & 0xFFFF0000u)) & 0x7FFF7FFFu;
  };
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max16x2(top, mag(i));
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t sc = scale_code16(k ? top >> 16 : top & 0xFFFFu);
    const float scale = scale_value(sc);
    row_u32x4 q;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t o = 0;
#define SFC_CVT(n)                                                                                                  \
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, value(k, 8 * w + 2 * n), value(k, 8 * w + 2 * n + 1), scale, n)
      SFC_CVT(0);
      SFC_CVT(1);
      SFC_CVT(2);
      SFC_CVT(3);
#undef SFC_CVT
      q[w] = o;
    }
    *reinterpret_cast<row_u32x4*>(codes + (2 * lane + k) * kQtStride + 16 * wave) = q;
    scales[(2 * lane + k) * 8 + wave] = (uint8_t)sc;
  }
  if constexpr (BOTH) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      uint32_t q = 0;
#pragma unroll
      for (int u = 0; u < 4; u += 2) {
        // the two rows' maxima over the lane's columns, then over 16 lanes
        const uint32_t a = mag(i + u), b = mag(i + u + 1);
        const uint32_t m = row16_max16x2(max16x2((a & 0xFFFFu) | (b << 16), (a >> 16) | (b & 0xFFFF0000u)));
        const uint32_t s0 = scale_code16(m & 0xFFFFu), s1 = scale_code16(m >> 16);
        // (the conversion's byte selector is a constant)
        const float x0 = value(0, i + u), y0 = value(1, i + u), x1 = value(0, i + u + 1), y1 = value(1, i + u + 1);
        if (u == 0) {
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x0, y0, scale_value(s0), 0);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x1, y1, scale_value(s1), 1);
        } else {
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x0, y0, scale_value(s0), 2);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x1, y1, scale_value(s1), 3);
        }
        if ((lane & 15) == 0) {
          row_scales[(32 * wave + i + u) * 4 + (lane >> 4)] = (uint8_t)s0;
          row_scales[(32 * wave + i + u + 1) * 4 + (lane >> 4)] = (uint8_t)s1;
        }
      }
      row_codes[(8 * wave + i / 4) * 64 + lane] = q;
    }
  }
  __syncthreads();
  const int64_t blocks = (p.rows + 31) >> 5, b0 = (int64_t)rg * 8;
  for (int i = tid; i < kQtCols * 8; i += 512) {
    const int col = i >> 3, b = i & 7;
    if (c0 + col < p.cols && b0 + b < blocks) {
      *reinterpret_cast<row_u32x4*>(p.Qt + (c0 + col) * p.ldqt + (b0 + b) * 16) =
          *reinterpret_cast<const row_u32x4*>(codes + col * kQtStride + 16 * b);
      p.St[(c0 + col) * p.ldst + b0 + b] = scales[col * 8 + b];
    }
  }
  if constexpr (BOTH) {
    const int64_t row_blocks = (p.cols + 31) >> 5, cb0 = c0 >> 5, top_row = (int64_t)rg * 256;
    // a thread takes a block of four rows: 16 words of a byte per row, turned into 4 x 16 bytes
    if (tid < 256) {
      const int quad = tid >> 2, b = tid & 3;
      row_u32x4 in[4], out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) in[j] = *reinterpret_cast<const row_u32x4*>(row_codes + quad * 64 + 16 * b + 4 * j);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w0 = in[j][0], w1 = in[j][1], w2 = in[j][2], w3 = in[j][3];
        const uint32_t a0 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), a1 = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
        const uint32_t b0 = __builtin_amdgcn_perm(w3, w2, 0x05010400u), b1 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
        out[0][j] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
        out[1][j] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
        out[2][j] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
        out[3][j] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
      }
      if (cb0 + b < row_blocks) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = 4 * quad + u;
          if (top_row + r < p.rows) {
            *reinterpret_cast<row_u32x4*>(p.Q + (top_row + r) * p.ldq + (cb0 + b) * 16) = out[u];
            p.S[(top_row + r) * p.lds + cb0 + b] = row_scales[r * 4 + b];
          }
        }
      }
    }
  }
}

hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool in_bf16, int num_cus, hipStream_t stream) {
  if (!p.Qt) {
    const RowShape sh = row_shape(p.rows, (p.cols + 31) / 32 * 4, num_cus);
    const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
    if (in_bf16) hipLaunchKernelGGL((mx4_quant_rows_kernel<true>), g, b, 0, stream, p, sh);
    else hipLaunchKernelGGL((mx4_quant_rows_kernel<false>), g, b, 0, stream, p, sh);
    return hipGetLastError();
  }
  const int rg = (int)((p.rows + 255) / 256);
  const dim3 g((unsigned)(rg * ((p.cols + kQtCols - 1) / kQtCols))), b(512);
  if (in_bf16 && p.Q) hipLaunchKernelGGL((mx4_quant_cols_kernel<true, true>), g, b, 0, stream, p, rg);
  else if (in_bf16) hipLaunchKernelGGL((mx4_quant_cols_kernel<true, false>), g, b, 0, stream, p, rg);
  else if (p.Q) hipLaunchKernelGGL((mx4_quant_cols_kernel<false, true>), g, b, 0, stream, p, rg);
  else hipLaunchKernelGGL((mx4_quant_cols_kernel<false, false>), g, b, 0, stream, p, rg);
  return hipGetLastError();
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

template <bool BF16, bool PAST>
__global__ __launch_bounds__(256) void mx4_dequant_kernel(Mx4DequantParams p, RowShape sh) {
  const RowPlace at = row_place(sh, (p.cols + 7) >> 3);
  if (at.row >= p.rows) return;
  const uint8_t* q = p.Q + at.row * p.ldq;
  const uint8_t* s = p.S + at.row * p.lds;
  char* y = reinterpret_cast<char*>(p.Y) + at.row * p.ldy * (BF16 ? 2 : 4);
  constexpr int U = 4;
  uint32_t code[U], scale[U];
  row_loop<U>(
      at,
      [&](int u, int64_t c) {
        code[u] = *reinterpret_cast<const uint32_t*>(q + c * 4);
        scale[u] = s[c >> 2];
      },
      [&](int u, int64_t c) { store8<BF16, PAST>(y, c * 8, p.cols, values8<BF16>(code[u], scale[u])); });
}

hipError_t launch_mx4_dequant(const Mx4DequantParams& p, bool out_bf16, int num_cus, hipStream_t stream) {
  const RowShape sh = row_shape(p.rows, (p.cols + 7) / 8, num_cus);
  const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
  const bool past = streams_past_caches(p.rows * p.cols * (out_bf16 ? 2 : 4));
  if (out_bf16 && past) hipLaunchKernelGGL((mx4_dequant_kernel<true, true>), g, b, 0, stream, p, sh);
  else if (out_bf16) hipLaunchKernelGGL((mx4_dequant_kernel<true, false>), g, b, 0, stream, p, sh);
  else if (past) hipLaunchKernelGGL((mx4_dequant_kernel<false, true>), g, b, 0, stream, p, sh);
  else hipLaunchKernelGGL((mx4_dequant_kernel<false, false>), g, b, 0, stream, p, sh);
  return hipGetLastError();
}

}  // namespace sfc
