// Rows of fp32 or bf16 values, eight at a time, at any element alignment.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sfc {

typedef uint32_t row_u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at the alignment of an element: the access mode of ROCm takes such loads and
// stores as one instruction.
template <int ES>
struct __attribute__((packed, aligned(ES))) Any16 { row_u32x4 v; };

__device__ __forceinline__ float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }

// Two fp32 values rounded to bf16, to nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Eight consecutive elements as stored: BF16 one 16-byte word, else two.
template <bool BF16>
struct Raw8 {
  row_u32x4 w[BF16 ? 1 : 2];
};

// Elements c .. c+7 of a row of `cols`; those past its end are 0.
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load8(const void* row, int64_t c, int64_t cols) {
  Raw8<BF16> r;
  if constexpr (BF16) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + c;
    if (c + 8 <= cols) {
      r.w[0] = reinterpret_cast<const Any16<2>*>(p)->v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = c + 2 * i < cols ? p[2 * i] : 0, hi = c + 2 * i + 1 < cols ? p[2 * i + 1] : 0;
        r.w[0][i] = lo | (hi << 16);
      }
    }
  } else {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + c;
    if (c + 8 <= cols) {
      r.w[0] = reinterpret_cast<const Any16<4>*>(p)->v;
      r.w[1] = reinterpret_cast<const Any16<4>*>(p + 4)->v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = c + i < cols ? p[i] : 0;
    }
  }
  return r;
}

template <bool BF16>
__device__ __forceinline__ Raw8<BF16> zero8() {
  Raw8<BF16> r;
  r.w[0] = row_u32x4{0u, 0u, 0u, 0u};
  if constexpr (!BF16) r.w[1] = row_u32x4{0u, 0u, 0u, 0u};
  return r;
}

template <bool BF16>
__device__ __forceinline__ void store8(void* row, int64_t c, int64_t cols, const Raw8<BF16>& r) {
  if constexpr (BF16) {
    uint16_t* p = reinterpret_cast<uint16_t*>(row) + c;
    if (c + 8 <= cols) {
      reinterpret_cast<Any16<2>*>(p)->v = r.w[0];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = (uint16_t)(r.w[0][i >> 1] >> (16 * (i & 1)));
    }
  } else {
    uint32_t* p = reinterpret_cast<uint32_t*>(row) + c;
    if (c + 8 <= cols) {
      reinterpret_cast<Any16<4>*>(p)->v = r.w[0];
      reinterpret_cast<Any16<4>*>(p + 4)->v = r.w[1];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = r.w[i >> 2][i & 3];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void to_float(const Raw8<BF16>& r, float* f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (BF16) f[i] = (i & 1) ? bf16_high(r.w[0][i >> 1]) : bf16_low(r.w[0][i >> 1]);
    else f[i] = __builtin_bit_cast(float, (uint32_t)r.w[i >> 2][i & 3]);
  }
}

template <bool BF16>
__device__ __forceinline__ Raw8<BF16> from_float(const float* f) {
  Raw8<BF16> r;
#pragma unroll
  for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
    if constexpr (BF16) r.w[0][i] = bf16_pair(f[2 * i], f[2 * i + 1]);
    else r.w[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, f[i]);
  }
  return r;
}

// How a workgroup of 256 threads covers rows of `chunks` eight-element chunks: tx threads
// (a power of two, at least 4) side by side, 256 / tx rows, and each row's chunks dealt to
// `splits` workgroups, `per` chunks (a multiple of tx) each.
struct RowShape {
  int tx_log2, splits;
  int64_t per, row_blocks;
};
inline RowShape row_shape(int64_t rows, int64_t chunks, int num_cus) {
  RowShape s;
  s.tx_log2 = 2;
  while (s.tx_log2 < 8 && (int64_t)1 << s.tx_log2 < chunks) ++s.tx_log2;
  const int64_t tx = (int64_t)1 << s.tx_log2, ty = 256 / tx;
  s.row_blocks = (rows + ty - 1) / ty;
  const int64_t passes = (chunks + tx - 1) / tx;         // of a workgroup over a whole row
  // few rows: a row is shared out until there are 8 workgroups for each CU
  int64_t splits = (8 * (int64_t)num_cus) / (s.row_blocks > 0 ? s.row_blocks : 1);
  if (splits < 1) splits = 1;
  if (splits > passes) splits = passes < 1 ? 1 : passes;
  const int64_t each = (passes + splits - 1) / splits;
  s.per = each * tx;
  s.splits = (int)((passes + each - 1) / each);
  if (s.splits < 1) s.splits = 1;
  return s;
}

}  // namespace sfc
