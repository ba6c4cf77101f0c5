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

// Whether a kernel's output of `bytes` goes past the caches: it will not be found there, and
// the rows that are read stay.  8192 x 4096 bf16 rows: dispatch 45.6 -> 40.8 us, combine
// 39.4 -> 36.6, its gradient 66.9 -> 64.5, dequantisation 17.4 -> 13.5; below 32 MB the next
// kernel may find the output in the caches.  fp32 rows, two stores a lane, gain less or lose: each
// kernel's launch says which.
inline bool streams_past_caches(int64_t bytes) { return bytes >= (int64_t)32 << 20; }

typedef row_u32x4 any_u32x4 __attribute__((aligned(2)));
// (PAST is a template argument: the compiler joins a branch's two stores into one)
template <bool PAST>
__device__ __forceinline__ void store16(void* p, const row_u32x4& v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<any_u32x4*>(p));
  else *reinterpret_cast<any_u32x4*>(p) = v;
}

template <bool BF16, bool PAST>
__device__ __forceinline__ void store8(void* row, int64_t c, int64_t cols, const Raw8<BF16>& r) {
  if constexpr (BF16) {
    uint16_t* p = reinterpret_cast<uint16_t*>(row) + c;
    if (c + 8 <= cols) {
      store16<PAST>(p, r.w[0]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = (uint16_t)(r.w[0][i >> 1] >> (16 * (i & 1)));
    }
  } else {
    uint32_t* p = reinterpret_cast<uint32_t*>(row) + c;
    if (c + 8 <= cols) {
      store16<PAST>(p, r.w[0]);
      store16<PAST>(p + 4, r.w[1]);
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
// (a power of two, 4 .. 256, half the chunks if that is fewer: two loads or more to a
// thread) side by side, 256 / tx rows, and each row's chunks dealt to `splits` workgroups,
// `per` chunks (a multiple of tx) each.  Rows of 4096 bf16: 256 threads 39.5 us for a combine
// of 8192 tokens, 64 threads 54; rows of 1024: 128 threads 25.2 us for 16384, 64 threads 21.6.
struct RowShape {
  int tx_log2, splits;
  int64_t per, row_blocks;
};
inline RowShape row_shape(int64_t rows, int64_t chunks, int num_cus) {
  RowShape s;
  s.tx_log2 = 2;
  while (s.tx_log2 < 8 && (int64_t)2 << s.tx_log2 < chunks) ++s.tx_log2;
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

// A thread's place in a RowShape launch, and a loop over its chunks, U at a time: `load(u, c)`
// for all of them, then `use(u, c)`, so that U loads are in flight (the stores of one chunk
// could alias the loads of the next: the compiler would not do it by itself).
struct RowPlace {
  int64_t row, first, last;
  int lane_tx, tx;
};
__device__ __forceinline__ RowPlace row_place(const RowShape& sh, int64_t chunks) {
  RowPlace p;
  p.tx = 1 << sh.tx_log2;
  const int64_t rb = blockIdx.x / (unsigned)sh.splits;
  const int split = (int)(blockIdx.x - rb * sh.splits);
  p.row = rb * (256 >> sh.tx_log2) + (threadIdx.x >> sh.tx_log2);
  p.first = (int64_t)split * sh.per;
  p.last = p.first + sh.per < chunks ? p.first + sh.per : chunks;
  p.lane_tx = threadIdx.x & (p.tx - 1);
  return p;
}
template <int U, typename Load, typename Use>
__device__ __forceinline__ void row_loop(const RowPlace& p, Load load, Use use) {
  for (int64_t c = p.first + p.lane_tx; c < p.last; c += U * p.tx) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c + u * p.tx < p.last) load(u, c + u * p.tx);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c + u * p.tx < p.last) use(u, c + u * p.tx);
  }
}

}  // namespace sfc
