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
// Bound: memory.  Every value is read once, 17/32 byte written.  8192 x 4096 bf16: along the
// rows 17.5 us (4.8 TB/s), back 13.4 (6.3; the codes are still cached); a copy of as many
// values 25.9 (5.2).  Three such matrices in turn, which the caches hold in part: bf16 14.1 along the
// rows, 14.7 along the columns, 24.6 both ways; fp32 27.9 (5.5 TB/s), 33.2 and 37.7.
#include "sfc_launch.h"
#include "sfc_mx4_convert.h"
#include "sfc_ops_params.h"

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
// the same read.  A workgroup of W = 8 (4) waves takes 256 (128) rows x 128 columns: a lane holds 32 rows
// of two columns in registers, so a column block's maximum needs no other lane, and a row
// block is 16 lanes.  Codes and scales meet in LDS and leave as 128-byte (64-byte: rows)
// pieces.  Stores go through the caches, since a product reads them next: past them this
// kernel takes 2-3 us less and the weight gradients 14 us more.
// 8192 x 4096 bf16: 20.3 us (4.2 TB/s), both ways 27.4 (3.75; two calls 38); bounded by memory
// and, both ways, by a workgroup's phases (load, convert, store) with two workgroups to a CU:
// three (80 registers) spill and take 36 us.
constexpr int kQtCols = 128;

typedef uint16_t q_u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(q_u16x2, a), __builtin_bit_cast(q_u16x2, b)));
}
// Of 16 words a lane (two rows' maxima each), lane j of a row of 16 lanes is left with the
// maximum of word row_pair(j) over the row: every step halves the words and doubles the lanes
// that they cover (60 instructions; the maximum of each word in every lane took 128).
__device__ __forceinline__ int row_pair(int lane) {
  return ((lane >> 2) & 1) * 8 + (lane & 1) * 4 + ((lane >> 1) & 1) * 2 + ((lane >> 3) & 1);
}
// The lane that holds word i.
constexpr int row_pair_lane(int i) { return ((i >> 3) & 1) * 4 + ((i >> 2) & 1) + ((i >> 1) & 1) * 2 + (i & 1) * 8; }
template <int DPP>
__device__ __forceinline__ void row_halve(uint32_t* m, int n, bool upper) {
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const uint32_t keep = upper ? m[i + n] : m[i], give = upper ? m[i] : m[i + n];
    m[i] = max16x2(keep, __builtin_amdgcn_update_dpp(0, give, DPP, 0xF, 0xF, true));
  }
}
__device__ __forceinline__ uint32_t row_maxima(uint32_t (&m)[16], int lane) {
  row_halve<0x141>(m, 8, lane & 4);      // lanes mirrored in 8
  row_halve<0xB1>(m, 4, lane & 1);       // lanes 1 0 3 2
  row_halve<0x4E>(m, 2, lane & 2);       // lanes 2 3 0 1
  row_halve<0x128>(m, 1, lane & 8);      // lanes 8 further in 16
  return m[0];
}
// Word I's value in every lane of the row.
template <int I>
__device__ __forceinline__ uint32_t row_word(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x150 + row_pair_lane(I), 0xF, 0xF, true);
}
// Scale code from the upper 16 bits of the largest magnitude (its exponent field is all that counts).
__device__ __forceinline__ uint32_t scale_code16(uint32_t top) { return scale_code(top << 16); }

template <bool BF16, bool BOTH, int W>
__global__ __launch_bounds__(64 * W, 4) void mx4_quant_cols_kernel(Mx4QuantParams p, int row_groups) {
  // column 2 i + k of the block lies in place 64 k + i: lanes that write neighbouring even (odd)
  // columns meet 36 banks apart
  constexpr int kRows = 32 * W, kStride = 16 * W + 16;         // kStride: LDS bytes from one column to the next
  __shared__ __attribute__((aligned(16))) uint8_t codes[kQtCols * kStride];
  __shared__ __attribute__((aligned(16))) uint8_t scales[kQtCols * W];
  __shared__ __attribute__((aligned(16))) uint32_t row_codes[BOTH ? kRows / 4 * 64 : 4];    // [4 rows][2 columns]: a byte a row
  __shared__ __attribute__((aligned(16))) uint8_t row_scales[BOTH ? kRows * 4 : 16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col_groups = gridDim.x / (unsigned)row_groups;
  // BOTH: two neighbouring column blocks, whose 64-byte pieces of rows make a line, go to one XCD
  // (8192 x 4096 bf16: 27.4 us, neighbours on different ones 28.9)
  unsigned task = blockIdx.x;
  if (BOTH && task < (gridDim.x & ~15u)) task = (task & ~15u) + 2 * (task & 7) + ((task >> 3) & 1);
  const int rg = task / (unsigned)col_groups, cb = task - rg * col_groups;
  const int64_t c0 = (int64_t)cb * kQtCols, c = c0 + 2 * lane;
  const int64_t r0 = (int64_t)rg * kRows + 32 * wave;
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
    const char* x = reinterpret_cast<const char*>(p.X) + c0 * ES;
    const uint32_t off = 2 * lane * ES;
    if (c + 1 < p.cols) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int r = __builtin_amdgcn_readlane(source, i);
        struct __attribute__((packed, aligned(ES))) Pair { uint32_t v[BF16 ? 1 : 2]; };
        const Pair w = *reinterpret_cast<const Pair*>(x + (int64_t)(r < 0 ? 0 : r) * p.ldx * ES + off);
        raw[0][i] = w.v[0];
        if constexpr (!BF16) raw[1][i] = w.v[1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int r = __builtin_amdgcn_readlane(source, i);
        const char* e = x + (int64_t)(r < 0 ? 0 : r) * p.ldx * ES + off;
        raw[0][i] = BF16 ? *reinterpret_cast<const uint16_t*>(e) : *reinterpret_cast<const uint32_t*>(e);
      }
    }
  }
  if (__ballot(source < 0) & 0xFFFFFFFFull) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const bool zero = __builtin_amdgcn_readlane(source, i) < 0;
#pragma unroll
      for (int k = 0; k < (BF16 ? 1 : 2); ++k) raw[k][i] = zero ? 0u : raw[k][i];
    }
  }
  // rows 2 i and 2 i + 1 of column k: the values as bf16 (the upper halves of fp32)
  auto upper = [&](int k, int i) {
    return __builtin_amdgcn_perm(raw[BF16 ? 0 : k][2 * i + 1], raw[BF16 ? 0 : k][2 * i], BF16 && k == 0 ? 0x05040100u : 0x07060302u);
  };
  // rows 2 i and 2 i + 1 of column k, or both columns of row i, to codes: byte n of q
#define SFC_CVT_COL(q, k, i, n)                                                                                        \
  q = BF16 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, upper(k, i)), scale, n)          \
           : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_bit_cast(float, raw[BF16 ? 0 : k][2 * (i)]),        \
                                                      __builtin_bit_cast(float, raw[BF16 ? 0 : k][2 * (i) + 1]), scale, n)
#define SFC_CVT_ROW(q, i, scale, n)                                                                                    \
  q = BF16 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, raw[0][i]), scale, n)            \
           : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_bit_cast(float, raw[0][i]),                         \
                                                      __builtin_bit_cast(float, raw[BF16 ? 0 : 1][i]), scale, n)
  uint32_t rows2[16], top[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t a = upper(0, i) & 0x7FFF7FFFu, b = upper(1, i) & 0x7FFF7FFFu;
    top[0] = max16x2(top[0], a);
    top[1] = max16x2(top[1], b);
    rows2[i] = max16x2(a, b);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t t = max16x2(top[k], top[k] >> 16);
    const uint32_t sc = scale_code16(t & 0xFFFFu);
    const float scale = scale_value(sc);
    row_u32x4 q;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t o = 0;
      SFC_CVT_COL(o, k, 4 * w, 0);
      SFC_CVT_COL(o, k, 4 * w + 1, 1);
      SFC_CVT_COL(o, k, 4 * w + 2, 2);
      SFC_CVT_COL(o, k, 4 * w + 3, 3);
      q[w] = o;
    }
    *reinterpret_cast<row_u32x4*>(codes + (64 * k + lane) * kStride + 16 * wave) = q;
    scales[(64 * k + lane) * W + wave] = (uint8_t)sc;
  }
  if constexpr (BOTH) {
    // a lane makes the scales of two rows, whose upper halves (all that is not 0 in them) the
    // others take from it
    const uint32_t m = row_maxima(rows2, lane);
    const uint32_t s0 = scale_code16(m & 0xFFFFu), s1 = scale_code16(m >> 16);
    const int row = 32 * wave + 2 * row_pair(lane);
    row_scales[row * 4 + (lane >> 4)] = (uint8_t)s0;
    row_scales[(row + 1) * 4 + (lane >> 4)] = (uint8_t)s1;
    const uint32_t both = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, scale_value(s1)),
                                                __builtin_bit_cast(uint32_t, scale_value(s0)), 0x07060302u);
    uint32_t* out = row_codes + 8 * wave * 64 + lane;
#define SFC_FOUR_ROWS(w)                                                         \
  {                                                                              \
    const uint32_t sa = row_word<2 * w>(both), sb = row_word<2 * w + 1>(both);   \
    uint32_t q = 0;                                                              \
    SFC_CVT_ROW(q, 4 * w, __builtin_bit_cast(float, sa << 16), 0);               \
    SFC_CVT_ROW(q, 4 * w + 1, __builtin_bit_cast(float, sa & 0xFFFF0000u), 1);   \
    SFC_CVT_ROW(q, 4 * w + 2, __builtin_bit_cast(float, sb << 16), 2);           \
    SFC_CVT_ROW(q, 4 * w + 3, __builtin_bit_cast(float, sb & 0xFFFF0000u), 3);   \
    out[w * 64] = q;                                                             \
  }
    SFC_FOUR_ROWS(0)
    SFC_FOUR_ROWS(1)
    SFC_FOUR_ROWS(2)
    SFC_FOUR_ROWS(3)
    SFC_FOUR_ROWS(4)
    SFC_FOUR_ROWS(5)
    SFC_FOUR_ROWS(6)
    SFC_FOUR_ROWS(7)
#undef SFC_FOUR_ROWS
  }
#undef SFC_CVT_COL
#undef SFC_CVT_ROW
  __syncthreads();
  const int64_t blocks = (p.rows + 31) >> 5, b0 = (int64_t)rg * W;
#pragma unroll
  for (int i = tid; i < kQtCols * W; i += 64 * W) {
    const int col = i / W, b = i % W, place = 64 * (col & 1) + (col >> 1);
    if (c0 + col < p.cols && b0 + b < blocks) {
      *reinterpret_cast<row_u32x4*>(p.Qt + (c0 + col) * p.ldqt + (b0 + b) * 16) =
          *reinterpret_cast<const row_u32x4*>(codes + place * kStride + 16 * b);
    }
  }
  if (tid < kQtCols && c0 + tid < p.cols) {
    const uint8_t* from = scales + (64 * (tid & 1) + (tid >> 1)) * W;
    uint8_t* to = p.St + (c0 + tid) * p.ldst + b0;
    if (b0 + W <= blocks) {
#pragma unroll
      for (int k = 0; k < W / 4; ++k) reinterpret_cast<uint32_t*>(to)[k] = reinterpret_cast<const uint32_t*>(from)[k];
    } else {
      for (int b = 0; b0 + b < blocks; ++b) to[b] = from[b];
    }
  }
  if constexpr (BOTH) {
    const int64_t row_blocks = (p.cols + 31) >> 5, cb0 = c0 >> 5, top_row = (int64_t)rg * kRows;
    // half of the threads take a block of four rows each: 16 words of a byte per row, turned into
    // 4 x 16 bytes; the others a row's scales
    if (tid < kRows) {
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
          if (top_row + r < p.rows)
            *reinterpret_cast<row_u32x4*>(p.Q + (top_row + r) * p.ldq + (cb0 + b) * 16) = out[u];
        }
      }
    } else if (top_row + tid - kRows < p.rows) {
      const uint8_t* from = row_scales + (tid - kRows) * 4;
      uint8_t* to = p.S + (top_row + tid - kRows) * p.lds + cb0;
      if (cb0 + 4 <= row_blocks) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
      else
        for (int b = 0; cb0 + b < row_blocks; ++b) to[b] = from[b];
    }
  }
}

template <int W>
static hipError_t launch_cols(const Mx4QuantParams& p, bool in_bf16, dim3 g, dim3 b, int rg, hipStream_t stream) {
  if (in_bf16 && p.Q) return launch_kernel(mx4_quant_cols_kernel<true, true, W>, g, b, 0, stream, p, rg);
  if (in_bf16) return launch_kernel(mx4_quant_cols_kernel<true, false, W>, g, b, 0, stream, p, rg);
  if (p.Q) return launch_kernel(mx4_quant_cols_kernel<false, true, W>, g, b, 0, stream, p, rg);
  return launch_kernel(mx4_quant_cols_kernel<false, false, W>, g, b, 0, stream, p, rg);
}

hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool in_bf16, int num_cus, hipStream_t stream) {
  if (!p.Qt) {
    const RowShape sh = row_shape(p.rows, (p.cols + 31) / 32 * 4, num_cus);
    const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
    if (in_bf16) return launch_kernel(mx4_quant_rows_kernel<true>, g, b, 0, stream, p, sh);
    return launch_kernel(mx4_quant_rows_kernel<false>, g, b, 0, stream, p, sh);
  }
  const int col_groups = (int)((p.cols + kQtCols - 1) / kQtCols);
  // 256 rows to a workgroup, 128 while that leaves half of the CUs without one (us, 256 / 128 rows, both
  // ways: bf16 128x4096 5.4 / 4.3, 1024x1024 5.0 / 4.3, 2048x2048 6.2 / 5.7, 4096x4096 15.2 / 16.5,
  // 16384x4096 48.1 / 49.8; fp32 along the columns 128x4096 5.0 / 3.5, 2048x4096 10.2 / 10.7)
  const bool wide = (p.rows + 255) / 256 * col_groups * 2 > num_cus;
  const int rows = wide ? 256 : 128, rg = (int)((p.rows + rows - 1) / rows);
  const dim3 g((unsigned)(rg * col_groups)), b(2 * rows);
  return wide ? launch_cols<8>(p, in_bf16, g, b, rg, stream) : launch_cols<4>(p, in_bf16, g, b, rg, stream);
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
  // (fp32: a lane's two stores leave holes in a line, which only the caches fill: 8192x4096 51 us past
  // them, 26 through)
  const bool past = out_bf16 && streams_past_caches(p.rows * p.cols * 2);
  if (past) return launch_kernel(mx4_dequant_kernel<true, true>, g, b, 0, stream, p, sh);
  if (out_bf16) return launch_kernel(mx4_dequant_kernel<true, false>, g, b, 0, stream, p, sh);
  return launch_kernel(mx4_dequant_kernel<false, false>, g, b, 0, stream, p, sh);
}

}  // namespace sfc
