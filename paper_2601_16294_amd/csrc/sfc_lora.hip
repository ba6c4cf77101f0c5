// Low-rank adapters of many requests beside a shared projection, for gfx950.
//
//   down      V[t] = s[a] X[t] A[a]^T            a = ids[t], zeros where there is none
//   up        Y[t] = base[t] + V[t] B[a]^T       base[t] where there is none
//   gradient  G[a] = sum over t with ids[t] = a of Z[t]^T V[t]
//
// with ranks of a few to a few hundred: X, base and Y are read and written once, and that
// traffic is what bounds them; the products are small beside it.  V is fp32.  Where it meets bf16 weights in
// MFMAs it is taken apart into bf16 terms, each the leading 8 bits of what the ones before
// leave, the last one rounded: two are off by at most 2^-16 of it (bf16 results, which are rounded to 2^-8),
// three hold every bit of it (fp32 results), down to 2^-134.
//
// Measured: up of 4096 rows x 14336, rank 64 57 us = 4.2 TB/s, of 8192 x 4096, rank 16 26 us = 5.2 TB/s; 32 rows x 4096 of 16
// adapters, rank 16, 3.7 us down and 3.7 up, a launch and a chain of loads each.
//
// Two forms of down and up.  Where rows x rank x columns is small, as in decode steps, every row is taken by
// itself and reads its adapter's weights (from the L2 where another row has): no order of the rows is
// slow.  Else a wave takes tiles of 16 rows on MFMAs.  They may belong to up to 16 adapters: it computes with one adapter
// after the other and keeps the results of that adapter's rows, so no row sees another adapter's
// weights, infinities and NaN among them.
//
// An infinite weight (in the gradient: Z) times a term of V that is 0, as the second of 1 is, would be NaN where the formula has an
// infinity.  The first term is 0 only where V is, so up adds up the others by themselves and puts a number in the place of a
// NaN before the two meet; the gradient forms sums that end as NaN once more, from V as it is.
#include "sfc_gemm_kernel.h"
#include "sfc_launch.h"
#include "sfc_lora_params.h"
#include "sfc_row_io.h"

namespace sfc {

namespace {

__device__ __forceinline__ bf16x8 as_bf16x8(const row_u32x4& v) { return __builtin_bit_cast(bf16x8, v); }

// 8 elements at p.
__device__ __forceinline__ row_u32x4 load_any(const uint16_t* p) { return reinterpret_cast<const Any16<2>*>(p)->v; }
// Element i + n of v as element i, zeros behind.
__device__ __forceinline__ row_u32x4 moved_down(const row_u32x4& v, int64_t n) {
  const uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  const int s = n < 4 ? 16 * (int)n : n < 8 ? 16 * (int)n - 64 : 0;
  const uint64_t low = n >= 8 ? 0 : n >= 4 ? hi >> s : s ? lo >> s | hi << (64 - s) : lo, high = n >= 4 ? 0 : hi >> s;
  return row_u32x4{(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
}
// 8 elements of a row from column c on; CHECKED: those that lie before `cols`, and zeros.
template <bool CHECKED>
__device__ __forceinline__ row_u32x4 load_part(const uint16_t* row, int64_t c, int64_t cols) {
  if constexpr (!CHECKED) {
    return load_any(row + c);
  } else if (cols < 8) {
    return c < cols ? load8<true>(row, c, cols).w[0] : row_u32x4{};
  } else {
    // the 8 elements that end with the row, moved down (no branch: a load waits for no other)
    const int64_t at = c + 8 <= cols ? c : cols - 8;
    return moved_down(load_any(row + at), c - at);
  }
}
__device__ __forceinline__ row_u32x4 keep_if(bool on, const row_u32x4& v) {
  return row_u32x4{on ? v[0] : 0u, on ? v[1] : 0u, on ? v[2] : 0u, on ? v[3] : 0u};
}
__device__ __forceinline__ void floats_of(const row_u32x4& v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (i & 1) ? bf16_high(v[i >> 1]) : bf16_low(v[i >> 1]);
}

// The adapter of row t, or -1.
__device__ __forceinline__ int adapter_of(const LoraParams& p, int64_t t) {
  const int a = p.ids[t < p.rows ? t : p.rows - 1];
  return t < p.rows && a >= 0 && a < p.adapters ? a : -1;
}

// bf16 terms of 8 fp32 values.  (Halves of two words in one: a byte permutation.)  The first is the value's leading 8
// bits, the last of them set where a bit behind them is: so it is 0 only where the value is, a NaN stays one whatever its
// payload, and what is left is less than its last bit.  An infinity leaves NaN.
__device__ __forceinline__ uint32_t halves(float lo, float hi, uint32_t which) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), which);
}
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&v)[8], bf16x8 (&out)[TERMS]) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u32x4 w[TERMS];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = v[2 * i], hi = v[2 * i + 1];
    const u16x2 behind = __builtin_elementwise_min(__builtin_bit_cast(u16x2, halves(lo, hi, 0x05040100u)), u16x2{1, 1});
    w[0][i] = halves(lo, hi, 0x07060302u) | __builtin_bit_cast(uint32_t, behind);
    lo -= bf16_low(w[0][i]);
    hi -= bf16_high(w[0][i]);
#pragma unroll
    for (int k = 1; k + 1 < TERMS; ++k) {
      w[k][i] = halves(lo, hi, 0x07060302u);
      lo -= bf16_low(w[k][i]);
      hi -= bf16_high(w[k][i]);
    }
    w[TERMS - 1][i] = bf16_pair(lo, hi);
  }
#pragma unroll
  for (int k = 0; k < TERMS; ++k) out[k] = __builtin_bit_cast(bf16x8, w[k]);
}

// v, or the nearest number for an infinity, and some number for NaN.
__device__ __forceinline__ float number(float v) { return __builtin_amdgcn_fmed3f(v, -__FLT_MAX__, __FLT_MAX__); }

// Ranks r .. r + 7 of a row of V; zeros past the rank (which is at least 1).
__device__ __forceinline__ void load_ranks(const float* row, int r, int rank, float (&v)[8]) {
  if (rank % 8 == 0) {
    const float* q = row + (r < rank ? r : 0);
    const f32x4 lo = __builtin_bit_cast(f32x4, reinterpret_cast<const Any16<4>*>(q)->v);
    const f32x4 hi = __builtin_bit_cast(f32x4, reinterpret_cast<const Any16<4>*>(q + 4)->v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = r < rank ? lo[e] : 0.f;
      v[4 + e] = r < rank ? hi[e] : 0.f;
    }
  } else {
    // (8 places for every chunk of ranks: kept from row to row, they made up of ranks over 128 spill 81 to 100 registers, 4096x4096,
    // rank 256, bf16 74 us, else 54)
    asm volatile("" : "+v"(r));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = row[r + e < rank ? r + e : rank - 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r + e < rank ? v[e] : 0.f;
  }
}
// Loads before it are on their way before anything behind it (the compiler would put them next to their
// uses, a few at a time, to save registers).
__device__ __forceinline__ void loads_first() { __builtin_amdgcn_sched_barrier(0); }

// Transposing read of 32 rows x 16 columns: lane l gets column column0(l % 16) of rows 8 (l / 16) .. + 7,
// from LDS rows `pitch` bytes apart; `at` is this lane's address, row 8 (l / 16) + (l % 16) / 4 and the
// first of 4 columns.
__device__ __forceinline__ bf16x8 read_transposed(uint32_t at, int pitch) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)at);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)(at + (uint32_t)(4 * pitch)));
  const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

// ---- row by row ----------------------------------------------------------------------------------

// A wave takes RW ranks of a row; lanes deal K out, 8 elements at a time.
template <int RW>
__global__ __launch_bounds__(256) void lora_row_down_nk(LoraParams p) {
  const int lane = threadIdx.x & 63;
  const int groups = (p.rank + RW - 1) / RW;
  const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = job / groups;
  const int r0 = (int)(job - t * groups) * RW;
  if (t >= p.rows) return;
  const int a = __builtin_amdgcn_readfirstlane(adapter_of(p, t));
  float sum[RW] = {};
  if (a >= 0) {
    const uint16_t* x = p.X + t * p.ldx;
    const uint16_t* w[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) w[i] = p.W + a * p.stride_w + (int64_t)(r0 + i < p.rank ? r0 + i : p.rank - 1) * p.ldw;
    auto add = [&](const row_u32x4& xv, const row_u32x4 (&wv)[RW]) {
      float xf[8], wf[8];
      floats_of(xv, xf);
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        floats_of(wv[i], wf);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[i] = __builtin_fmaf(xf[e], wf[e], sum[i]);
      }
    };
    constexpr int U = RW == 1 ? 8 : 4;         // loads of a row in flight
    int64_t k = 0;
    auto turns = [&](auto many) {
      constexpr int n = many;
      for (; k + n * 512 <= p.cols; k += n * 512) {
        row_u32x4 xv[n], wv[n][RW];
#pragma unroll
        for (int u = 0; u < n; ++u) {
          xv[u] = load_any(x + k + u * 512 + 8 * lane);
#pragma unroll
          for (int i = 0; i < RW; ++i) wv[u][i] = load_any(w[i] + k + u * 512 + 8 * lane);
        }
        loads_first();
#pragma unroll
        for (int u = 0; u < n; ++u) add(xv[u], wv[u]);
      }
    };
    turns(std::integral_constant<int, U>{});
    turns(std::integral_constant<int, 1>{});
    if (k + 8 * lane < p.cols) {
      row_u32x4 wv[RW];
#pragma unroll
      for (int i = 0; i < RW; ++i) wv[i] = load_part<true>(w[i], k + 8 * lane, p.cols);
      add(load_part<true>(x, k + 8 * lane, p.cols), wv);
    }
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) sum[i] += __shfl_xor(sum[i], d);
  }
  const float scale = a >= 0 && p.scales ? p.scales[a] : 1.f;
#pragma unroll
  for (int i = 0; i < RW; ++i)
    if (lane == 0 && r0 + i < p.rank) p.V[t * p.ldv + r0 + i] = scale * sum[i];
}

// Weights of K x rank: a workgroup takes a row.  A lane holds 8 ranks, LPR lanes a row of weights; the rows
// go round the lanes and waves, whose sums meet by lane exchanges, then through LDS.
constexpr int kRowWaves = 8;
template <int LPR>
__global__ __launch_bounds__(kRowWaves * 64) void lora_row_down_kn(LoraParams p) {
  constexpr int STEP = kRowWaves * 64 / LPR, U = 8;
  __shared__ float sums[kRowWaves][LPR * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int a = __builtin_amdgcn_readfirstlane(adapter_of(p, t));
  const int r = 8 * (lane % LPR), first = tid / LPR;
  float sum[8] = {};
  if (a >= 0 && r < p.rank) {
    const uint16_t* x = p.X + t * p.ldx;
    const uint16_t* w = p.W + a * p.stride_w;
    auto add = [&](uint16_t xv, const row_u32x4& wv) {
      float wf[8];
      floats_of(wv, wf);
      const float xf = bf16_low(xv);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf(xf, wf[e], sum[e]);
    };
    auto run = [&](auto checked) {
      int64_t k = first;
      for (; k + (U - 1) * STEP < p.cols; k += U * STEP) {
        uint16_t xv[U];
        row_u32x4 wv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          xv[u] = x[k + u * STEP];
          wv[u] = load_part<checked>(w + (k + u * STEP) * p.ldw, r, p.rank);
        }
        loads_first();
#pragma unroll
        for (int u = 0; u < U; ++u) add(xv[u], wv[u]);
      }
      for (; k < p.cols; k += STEP) add(x[k], load_part<checked>(w + k * p.ldw, r, p.rank));
    };
    if (p.rank % 8 == 0) run(std::false_type{});
    else run(std::true_type{});
  }
#pragma unroll
  for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += __shfl_xor(sum[e], d);
  if (lane < LPR)
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][r + e] = sum[e];
  __syncthreads();
  const float scale = a >= 0 && p.scales ? p.scales[a] : 1.f;
  if (tid < p.rank) {
    float v = sums[0][tid];
#pragma unroll
    for (int k = 1; k < kRowWaves; ++k) v += sums[k][tid];
    p.V[t * p.ldv + tid] = scale * v;
  }
}

template <bool OB>
__device__ __forceinline__ float load_base(const LoraParams& p, int64_t t, int64_t n) {
  if (!p.base) return 0.f;
  if constexpr (OB) return bf16_low(reinterpret_cast<const uint16_t*>(p.base)[t * p.ld_base + n]);
  else return reinterpret_cast<const float*>(p.base)[t * p.ld_base + n];
}

// A wave takes a row and 4 x 64 / LPC columns; LPC lanes share a column, 8 ranks at a time each.
template <int LPC, bool OB>
__global__ __launch_bounds__(256) void lora_row_up_nk(LoraParams p) {
  constexpr int Q = 4, PER = 64 / LPC;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = blockIdx.y, n0 = ((int64_t)blockIdx.x * 4 + wave) * (Q * PER);
  if (n0 >= p.cols) return;
  const int a = __builtin_amdgcn_readfirstlane(adapter_of(p, t));
  float sum[Q], base[Q];
  int64_t n[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    sum[q] = 0.f;
    n[q] = n0 + q * PER + lane / LPC;
    base[q] = n[q] < p.cols ? load_base<OB>(p, t, n[q]) : 0.f;
  }
  if (a >= 0) {
    const uint16_t* w = p.W + a * p.stride_w;
    const float* v = p.V + t * p.ldv;
    auto run = [&](auto checked) {
      for (int r = 8 * (lane % LPC); r < p.rank; r += 8 * LPC) {
        row_u32x4 wv[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) wv[q] = load_part<checked>(w + (n[q] < p.cols ? n[q] : p.cols - 1) * p.ldw, r, p.rank);
        float vf[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) vf[e] = !checked || r + e < p.rank ? v[r + e] : 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          float wf[8];
          floats_of(wv[q], wf);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[q] = __builtin_fmaf(vf[e], wf[e], sum[q]);
        }
      }
    };
    if (p.rank % 8 == 0) run(std::false_type{});
    else run(std::true_type{});
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int d = 1; d < LPC; d <<= 1) sum[q] += __shfl_xor(sum[q], d);
  }
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (lane % LPC == 0 && n[q] < p.cols) {
      const float y = base[q] + sum[q];
      if constexpr (OB) reinterpret_cast<__bf16*>(p.Y)[t * p.ldy + n[q]] = (__bf16)y;
      else reinterpret_cast<float*>(p.Y)[t * p.ldy + n[q]] = y;
    }
}

// Weights of rank x N: a lane takes 8 columns of a row.
template <bool OB>
__global__ __launch_bounds__(256) void lora_row_up_kn(LoraParams p) {
  const int64_t t = blockIdx.y, n = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (n >= p.cols) return;
  const int a = __builtin_amdgcn_readfirstlane(adapter_of(p, t));
  float y[8] = {};
  if (a >= 0) {
    const uint16_t* w = p.W + a * p.stride_w;
    const float* v = p.V + t * p.ldv;
    auto add = [&](float vf, const row_u32x4& wv) {
      float wf[8];
      floats_of(wv, wf);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(vf, wf[e], y[e]);
    };
    auto run = [&](auto checked) {
      int r = 0;
      for (; r + 8 <= p.rank; r += 8) {
        row_u32x4 wv[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) wv[u] = load_part<checked>(w + (int64_t)(r + u) * p.ldw, n, p.cols);
        loads_first();
#pragma unroll
        for (int u = 0; u < 8; ++u) add(v[r + u], wv[u]);
      }
      for (; r < p.rank; ++r) add(v[r], load_part<checked>(w + (int64_t)r * p.ldw, n, p.cols));
    };
    if (n + 8 <= p.cols) run(std::false_type{});
    else run(std::true_type{});
  }
  constexpr int ES = OB ? 2 : 4;
  if (p.base) {
    float b[8];
    to_float<OB>(load8<OB>(static_cast<const char*>(p.base) + t * p.ld_base * ES, n, p.cols), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] += b[e];
  }
  store8<OB, false>(static_cast<char*>(p.Y) + t * p.ldy * ES, n, p.cols, from_float<OB>(y));
}

// ---- up, in tiles --------------------------------------------------------------------------------

// The first n of 8 bf16 elements, to a whole word's address.
__device__ __forceinline__ void store_words(char* to, const row_u32x4& v, int n) {
  typedef row_u32x4 word_u32x4 __attribute__((aligned(4)));
  typedef uint32_t word_u32x2 __attribute__((ext_vector_type(2), aligned(4)));
  if (n >= 8) {
    *reinterpret_cast<word_u32x4*>(to) = v;
  } else if (n > 0) {
    if (n & 4) *reinterpret_cast<word_u32x2*>(to) = word_u32x2{v[0], v[1]};
    if (n & 2) *reinterpret_cast<uint32_t*>(to + 2 * (n & 4)) = n & 4 ? v[2] : v[0];
    if (n & 1) *reinterpret_cast<uint16_t*>(to + 2 * (n & 6)) = (uint16_t)(n & 4 ? (n & 2 ? v[3] : v[2]) : n & 2 ? v[1] : v[0]);
  }
}

// Column of 64 that lane n of fragment j computes, so that a lane, which ends with 4 columns of every
// fragment, has 16 bytes of a row at a time, and 4 lanes 64: bf16 8 columns of two fragments, fp32 4 of one.
template <bool OB>
__device__ __forceinline__ int up_column(int j, int n) {
  return OB ? 32 * (j >> 1) + 8 * (n >> 2) + 4 * (j & 1) + (n & 3) : 16 * j + n;
}

// A workgroup takes 64 Q rows, Q tiles for each of its 4 waves, and a block of columns, one adapter after the other:
// the block's weights of that adapter go into LDS, and the waves take the tiles that hold rows of it, of which they load and
// store these rows alone.  A last turn copies the rows of no adapter.  Column blocks run fastest over the
// workgroups: those in flight cover whole rows.
template <int Q, int NC, bool NK, bool OB>
__global__ __launch_bounds__(256, (NC == 1 ? 3 : 2)) void lora_up_kernel(LoraParams p) {
  constexpr int TERMS = OB ? 2 : 3, ES = OB ? 2 : 4, CB = lora_up_columns(NC, OB), UNITS = CB / 64;
  constexpr int PITCH = NK ? NC * 64 + 16 : CB * 2 + 16;     // NK: [column][rank], else [rank][column]
  constexpr int PIECES = OB ? 2 : 4;           // 16-byte pieces of 64 columns of a row that a lane has
  __shared__ __attribute__((aligned(16))) unsigned char smem[NK ? CB * PITCH : 32 * NC * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int64_t t0 = (int64_t)blockIdx.y * (64 * Q), n0 = (int64_t)blockIdx.x * CB;
  const uint32_t lds0 = lds_addr(smem);
  const bool inside = n0 + CB <= p.cols;       // the block lies inside the columns
  const bool whole = inside && p.rank % 8 == 0;
  // rows of bf16 that start inside a word (16 bytes a lane at odd elements: 2001 rows x 4097, rank 40 24 us, 19 from the next word on)
  const bool odd = OB && ((reinterpret_cast<uint64_t>(p.Y) | (uint64_t)(p.ldy * 2)) & 2);
  int id[Q];
  uint64_t pending[Q], none[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    id[q] = adapter_of(p, t0 + 64 * q + lane);
    pending[q] = __ballot(id[q] >= 0);
    none[q] = __ballot(id[q] < 0 && t0 + 64 * q + lane < p.rows);
  }

  // rows `bits` of tile k: base (+ V times the weights in LDS), to Y
  auto tile = [&](int k, uint32_t bits, auto product, auto in) {
    const int64_t t = t0 + 16 * k + col;
    const bool mine = bits >> col & 1;
    const int64_t row = mine ? t : t0 + 16 * k + __builtin_ctz(bits);
    const int piece = 16 / ES * g;             // of this lane's pieces, from the first column of each
    constexpr int APART = 64 / PIECES;         // columns from piece to piece
    const char* base = static_cast<const char*>(p.base) + (row * p.ld_base + n0 + piece) * ES;
    char* out = static_cast<char*>(p.Y) + (row * p.ldy + n0 + piece) * ES;
    const int left = in ? 0 : (int)(p.cols - n0 - piece);              // columns from the lane's first on
    row_u32x4 bv[in ? UNITS : 1][PIECES];
    // at: column from the block's first on
    auto load_base_piece = [&](int at) -> row_u32x4 {
      if (!p.base) return row_u32x4{};
      if constexpr (in) {
        return reinterpret_cast<const Any16<ES>*>(base + at * ES)->v;
      } else if constexpr (OB) {
        return load_part<true>(reinterpret_cast<const uint16_t*>(base) - piece, at + piece, p.cols - n0);
      } else {
        row_u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = reinterpret_cast<const uint32_t*>(base)[at + e < left ? at + e : -piece];
        return v;
      }
    };
    if constexpr (in) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int q = 0; q < PIECES; ++q) bv[u][q] = load_base_piece(64 * u + APART * q);
    }
    bf16x8 vf[NC][TERMS];
    if constexpr (product) {
      constexpr int AHEAD = NC < 2 ? NC : 2;   // chunks whose loads are on their way at a time
#pragma unroll
      for (int c = 0; c < NC; c += AHEAD) {
        float v[AHEAD][8];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load_ranks(p.V + row * p.ldv, 32 * (c + i) + 8 * g, p.rank, v[i]);
        loads_first();
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) split_terms<TERMS>(v[i], vf[c + i]);
      }
    }
    auto unit = [&](int u, const row_u32x4 (&b)[PIECES]) {
      f32x4 y[4];
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        if constexpr (OB) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t w = b[q][e >> 1];
            y[2 * q + (e >> 2)][e & 3] = (e & 1) ? bf16_high(w) : bf16_low(w);
          }
        } else {
          y[q] = __builtin_bit_cast(f32x4, b[q]);
        }
      }
      if constexpr (product) {
        // The sums of all terms but the first, made numbers before they meet the first's.  Up to 2 chunks: these come on
        // top of them, from the same weights in registers.  More would be read from LDS twice (8192x4096, rank 128,
        // bf16 50 us), so the two sums have registers of their own (45 us).
        constexpr bool FIRST = NC <= 2;
        f32x4 acc[4] = {}, low[4] = {};
        bf16x8 wf[FIRST ? NC : 1][4];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (NC > 2 && 32 * c >= p.rank) break;
          bf16x8 (&w)[4] = wf[FIRST ? c : 0];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (NK)
              w[j] = *(lds_bf16x8*)(uintptr_t)(lds0 + (uint32_t)((64 * u + up_column<OB>(j, col)) * PITCH + 64 * c + 16 * g));
            else
              w[j] = read_transposed(lds0 + (uint32_t)((32 * c + 8 * g + (col >> 2)) * PITCH + 2 * (64 * u + up_column<OB>(j, 4 * (col & 3)))), PITCH);
          }
          constexpr int SOME = FIRST ? TERMS - 1 : TERMS;
#pragma unroll
          for (int m = 0; m < 4 * SOME; ++m) {
            const int j = m % 4, k2 = TERMS - SOME + m / 4;
            f32x4& to = k2 ? low[j] : acc[j];
            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], vf[c][k2], to, 0, 0, 0);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = FIRST ? number(low[j][e]) : acc[j][e] + number(low[j][e]);
        if constexpr (FIRST) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c][j], vf[c][0], acc[j], 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[j][e] += acc[j][e];
      }
      Raw8<true> results[PIECES];
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        if constexpr (OB) {
          const f32x4 lo = y[2 * q], hi = y[2 * q + 1];
          results[q].w[0] = row_u32x4{bf16_pair(lo[0], lo[1]), bf16_pair(lo[2], lo[3]), bf16_pair(hi[0], hi[1]), bf16_pair(hi[2], hi[3])};
        } else {
          results[q].w[0] = __builtin_bit_cast(row_u32x4, y[q]);
        }
      }
      if constexpr (OB) {
        if (odd) {
          // from the next word on: elements 1 .. 7 and the next lane's first; the unit's first element alone
          const int first = (int)(reinterpret_cast<uint64_t>(out) >> 1) & 1;
          const uint32_t w0 = results[0].w[0][0], w1 = results[1].w[0][0];
          const uint32_t next[2] = {(uint32_t)__shfl((int)(g == 0 ? w1 : w0), (lane + 16) & 63),
                                    (uint32_t)__shfl((int)w1, (lane + 16) & 63)};
          if (!mine) return;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int at = 64 * u + APART * q, most = q == 1 && g == 3 ? 8 : 9;
            const int end = in ? most : left - at < most ? left - at : most;
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t w = results[q].w[0][e], up = e < 3 ? results[q].w[0][e + 1] : next[q];
              o[e] = first ? w >> 16 | up << 16 : w;
            }
            store_words(out + 2 * (at + first), o, end - first);
            if (first && q == 0 && g == 0 && end > 0) *reinterpret_cast<uint16_t*>(out + 2 * at) = (uint16_t)w0;
          }
          return;
        }
      }
      if (mine) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
          const int at = 64 * u + APART * q;
          const Raw8<true>& o = results[q];
          if constexpr (in) store16<false>(out + at * ES, o.w[0]);
          else if constexpr (OB) store8<true, false>(out, at, left, o);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (at + e < left) reinterpret_cast<uint32_t*>(out)[at + e] = o.w[0][e];
        }
      }
    };
    if constexpr (in) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        loads_first();                         // (and one unit after the other, for registers)
        unit(u, bv[u]);
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < UNITS && n0 + 64 * u < p.cols; ++u) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) bv[0][q] = load_base_piece(64 * u + APART * q);
        unit(u, bv[0]);
      }
    }
  };
  auto tiles = [&](const uint64_t (&rows)[Q], auto product) {
    // (tiles 4 q .. 4 q + 3, one a wave: 16 bits of each)
    uint64_t own = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) own |= (rows[q] >> (16 * wave) & 0xFFFFu) << (16 * q);
#pragma unroll 1
    for (int k = wave; own; k += 4, own >>= 16) {
      const uint32_t bits = (uint32_t)own & 0xFFFFu;
      if (!bits) continue;
      if (inside) tile(k, bits, product, std::true_type{});
      else tile(k, bits, product, std::false_type{});
    }
  };

  for (;;) {
    int a = -1;
#pragma unroll
    for (int q = Q - 1; q >= 0; --q)
      if (pending[q]) a = __builtin_amdgcn_readlane(id[q], __builtin_ctzll(pending[q]));
    if (a < 0 || p.rank == 0) break;
    uint64_t match[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      match[q] = __ballot(id[q] == a);
      pending[q] &= ~match[q];
    }
    const uint16_t* w = p.W + (int64_t)a * p.stride_w;
    // 16-byte pieces of the block's weights, consecutive ones a lane after the other
    constexpr int LINE = NK ? NC * 4 : CB / 8, COUNT = (NK ? CB : 32 * NC) * LINE / 256;
    row_u32x4 piece[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int line = (tid + 256 * i) / LINE, at = 8 * ((tid + 256 * i) % LINE);
      if constexpr (NK) {
        if (whole) piece[i] = load_any(w + (n0 + line) * p.ldw + (at < p.rank ? at : 0));
        else piece[i] = load_part<true>(w + (n0 + line < p.cols ? n0 + line : p.cols - 1) * p.ldw, at, p.rank);
      } else {
        if (inside) piece[i] = load_any(w + (int64_t)(line < p.rank ? line : 0) * p.ldw + n0 + at);
        else piece[i] = load_part<true>(w + (int64_t)(line < p.rank ? line : 0) * p.ldw, n0 + at, p.cols);
      }
    }
    loads_first();
    __syncthreads();                           // the last turn's readers are done
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int line = (tid + 256 * i) / LINE, at = 8 * ((tid + 256 * i) % LINE);
      lds_write16(lds0 + (uint32_t)(line * PITCH + 2 * at), keep_if((NK ? at : line) < p.rank, piece[i]));
    }
    __syncthreads();
    tiles(match, std::true_type{});
  }
  if (p.rank == 0) {
#pragma unroll
    for (int q = 0; q < Q; ++q) none[q] |= pending[q];
  }
  tiles(none, std::false_type{});
}

// ---- gradient of the weights -------------------------------------------------------------------

constexpr int kGradList = 2048;        // chunks of 32 rows that are looked through at a time

// Parts of an adapter with `count` of `total` rows: `extra` of them are dealt out over all adapters by their
// rows; less than two are one, which needs no sum.
__device__ __forceinline__ int grad_parts(int64_t count, int64_t total, int extra) {
  const int n = total > 0 ? (int)(count * extra / total) : 0;
  return n > 1 ? n : 1;
}

__device__ __forceinline__ void store4(float* to, const f32x4& v, int64_t inside) {
  if (inside >= 4) {
    reinterpret_cast<Any16<4>*>(to)->v = __builtin_bit_cast(row_u32x4, v);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < inside) to[e] = v[e];
  }
}

// A workgroup takes 256 columns of Z, 64 a wave, 16 FR ranks, an adapter and a part of its rows.  Parts go by
// the adapters' numbers of rows, which every workgroup counts for itself, so that an adapter with most of the
// rows keeps the chip busy too; the workgroup then lists the chunks of 32 rows that hold rows of its
// adapter and takes its part of the list.  A chunk's V is taken apart once for all waves; chunks lie in one of two
// slots of LDS, the next one written while one is computed with, three more on their way.  In a
// chunk, rows of other adapters are zeros in both operands.  Bound: one read of Z for every 64 ranks, 13 us for 8192
// rows x 4096, rank 16; with 4 adapters it takes 26 and the sum 4: the pass over the ids, the list and the first loads come before
// a workgroup's 8 chunks (2001 rows x 4097, rank 40, 4 chunks each: 19).  That is for rows in runs: a chunk is loaded once for every
// adapter that has a row in it (both launches, 8192 rows x 4096, rank 16, runs / at random: 4 adapters 27 / 62, 32 adapters 27 / 198).
// NARROW: rows of Z or V of fewer than 8 elements, which are loaded one by one.
template <int FR, bool NARROW, bool NK, bool OB>
__global__ __launch_bounds__(kGradWaves * 64) void lora_wgrad_kernel(LoraParams p) {
  constexpr int WAVES = kGradWaves, TERMS = 3;
  constexpr int ZP = 64 * 2 + 16, VP = 16 * FR * 2 + 16;                 // bytes from row to row
  constexpr int VSLOT = TERMS * 32 * VP;
  constexpr int VL = (32 * 2 * FR + WAVES * 64 - 1) / (WAVES * 64);      // pieces of 8 ranks of a thread
  constexpr int SLOT = WAVES * 32 * ZP + VSLOT;                          // a chunk's Z and V
  __shared__ __attribute__((aligned(16))) unsigned char smem[2 * SLOT];
  __shared__ uint16_t list[kGradList];
  __shared__ int found[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int64_t c0 = (int64_t)blockIdx.x * kGradColumns + 64 * wave;
  const int r0 = (int)blockIdx.y * 16 * FR;
  const uint32_t z_own = lds_addr(smem) + (uint32_t)(wave * 32 * ZP), v_all = lds_addr(smem) + WAVES * 32 * ZP;
  const bool whole = c0 + 64 <= p.cols, live = c0 < p.cols;
  f32x4 acc[4][FR] = {};

  const int64_t chunks = (p.rows + 31) >> 5;
  // What a chunk's rows belong to: the adapter that all of them have, -1 for none, -2 for several.  With
  // `counts`, adds up the adapters' rows there.
  int* const kinds = reinterpret_cast<int*>(smem);                       // of kGradList chunks from `from` on
  int* const counts = kinds + kGradList;                                 // of kGradAdapters
  auto look_through = [&](int64_t from, int n, bool count) {
    for (int c = tid; c < n; c += WAVES * 64) {
      const int64_t t = (from + c) * 32;
      int ids[32];
      if (t + 32 <= p.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const row_u32x4 v = reinterpret_cast<const Any16<4>*>(p.ids + t + 4 * i)->v;
#pragma unroll
          for (int e = 0; e < 4; ++e) ids[4 * i + e] = (int)v[e];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) ids[i] = t + i < p.rows ? p.ids[t + i] : -1;
      }
      loads_first();
#pragma unroll
      for (int i = 0; i < 32; ++i) ids[i] = ids[i] >= 0 && ids[i] < p.adapters ? ids[i] : -1;
      bool one = true;
#pragma unroll
      for (int i = 1; i < 32; ++i) one = one && ids[i] == ids[0];
      kinds[c] = one ? ids[0] : -2;
      if (count && one) {
        if (ids[0] >= 0) atomicAdd(&counts[ids[0]], 32);
      } else if (count) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (ids[i] >= 0) atomicAdd(&counts[ids[i]], 1);
      }
    }
  };
  // this workgroup's adapter, which part of how many, and the first of them among all parts that are summed
  int a = p.first_adapter + (int)blockIdx.z, part = 0, parts = 1, first_part = 0;
  if (p.splits > 1 && p.adapters == 1) {
    part = a;
    parts = p.splits;
    a = 0;
    if (tid == 0 && part == 0 && blockIdx.x == 0 && blockIdx.y == 0) {
      p.parts[0] = 0;
      p.parts[1] = parts;
    }
  } else if (p.splits > 1) {
    for (int i = tid; i < p.adapters; i += WAVES * 64) counts[i] = 0;
    __syncthreads();
    for (int64_t from = 0; from < chunks; from += kGradList)
      look_through(from, (int)(chunks - from < kGradList ? chunks - from : kGradList), true);
    __syncthreads();
    int64_t total = 0;
    for (int i = lane; i < p.adapters; i += 64) total += counts[i];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
    // adapters in order, 64 at a time, until their parts pass this workgroup's number
    int before = 0, summed = 0;
    a = -1;
    for (int base = 0; base < p.adapters; base += 64) {
      const int own = base + lane < p.adapters ? grad_parts(counts[base + lane], total, p.splits) : 0;
      int end = own, sums = own > 1 ? own : 0;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int e = __shfl_up(end, d), q = __shfl_up(sums, d);
        end += lane >= d ? e : 0;
        sums += lane >= d ? q : 0;
      }
      if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && wave == 0 && base + lane < p.adapters) {
        p.parts[2 * (base + lane)] = summed + sums - (own > 1 ? own : 0);
        p.parts[2 * (base + lane) + 1] = own;
      }
      const uint64_t past = __ballot(before + end > (int)blockIdx.z);
      if (past && a < 0) {
        const int l = __ffsll((unsigned long long)past) - 1;
        a = base + l;
        parts = __shfl(own, l);
        part = (int)blockIdx.z - (before + __shfl(end, l) - parts);
        first_part = summed + __shfl(sums, l) - (parts > 1 ? parts : 0);
      }
      before += __shfl(end, 63);
      summed += __shfl(sums, 63);
    }
    a = __builtin_amdgcn_readfirstlane(a);
    parts = __builtin_amdgcn_readfirstlane(parts);
    part = __builtin_amdgcn_readfirstlane(part);
    first_part = __builtin_amdgcn_readfirstlane(first_part);
    __syncthreads();
    if (a < 0) return;                         // more workgroups than parts
  }

  constexpr int DEEP = 3;                      // chunks whose loads are on their way
  struct Chunk {
    int id;                    // of row l % 32
    row_u32x4 z[4];
    float v[VL][8];
  };
  // lane: row 8 i + l / 8 and 8 columns of load i of Z; thread: row and 8 ranks of piece i of V.  Pieces that
  // the end of a row cuts are the 8 elements that end with it, moved down before they are written; nothing in
  // `load` depends on a branch, so that a chunk waits for its own loads alone.
  const int zc = 8 * (lane & 7);
  const int64_t z_at = c0 + zc + 8 <= p.cols ? c0 + zc : p.cols - 8;
  auto v_place = [&](int i, int& t, int& r) {
    const int at = tid + i * (WAVES * 64) < 32 * 2 * FR ? tid + i * (WAVES * 64) : 32 * 2 * FR - 1;
    t = at / (2 * FR);
    r = r0 + 8 * (at % (2 * FR));
  };
  auto load = [&](int64_t t0, Chunk& k) {
    k.id = p.ids[t0 + (lane & 31) < p.rows ? t0 + (lane & 31) : p.rows - 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = t0 + 8 * i + (lane >> 3) < p.rows ? t0 + 8 * i + (lane >> 3) : p.rows - 1;
      if constexpr (NARROW) k.z[i] = load_part<true>(p.X + t * p.ldx, c0 + zc, p.cols);
      else k.z[i] = load_any(p.X + t * p.ldx + z_at);
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      int tv, r;
      v_place(i, tv, r);
      const int64_t t = t0 + tv < p.rows ? t0 + tv : p.rows - 1;
      if constexpr (NARROW) {
        load_ranks(p.V + t * p.ldv, r, p.rank, k.v[i]);
      } else {
        const float* q = p.V + t * p.ldv + (r + 8 <= p.rank ? r : p.rank - 8);
        const row_u32x4 lo = reinterpret_cast<const Any16<4>*>(q)->v, hi = reinterpret_cast<const Any16<4>*>(q + 4)->v;
#pragma unroll
        for (int e = 0; e < 8; ++e) k.v[i][e] = __builtin_bit_cast(float, (uint32_t)(e < 4 ? lo[e] : hi[e - 4]));
      }
    }
  };
  auto write = [&](const Chunk& k, int64_t t0, uint32_t slot) {
    const uint32_t mine = (uint32_t)__ballot(k.id == a && t0 + (lane & 31) < p.rows);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 8 * i + (lane >> 3);
      const row_u32x4 z = NARROW || whole ? k.z[i] : moved_down(k.z[i], c0 + zc - z_at);
      lds_write16(z_own + slot + (uint32_t)(t * ZP + 2 * zc), keep_if(mine >> t & 1, z));
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      int t, r;
      v_place(i, t, r);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = k.v[i][e];
      if (!NARROW && r0 + 16 * FR > p.rank) {
        const int n = r + 8 <= p.rank ? 0 : r - (p.rank - 8);
#pragma unroll
        for (int d = 4; d >= 1; d >>= 1)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = (n & d) || n >= 8 ? (e + d < 8 && n < 8 ? v[e + d] : 0.f) : v[e];
      }
      bf16x8 terms[TERMS];
      split_terms<TERMS>(v, terms);
      if (tid + i * (WAVES * 64) < 32 * 2 * FR) {
#pragma unroll
        for (int q = 0; q < TERMS; ++q)
          lds_write16(v_all + slot + (uint32_t)(q * 32 * VP + t * VP + 2 * (r - r0)),
                      keep_if(mine >> t & 1, __builtin_bit_cast(row_u32x4, terms[q])));
      }
    }
  };
  auto compute = [&](uint32_t slot) {
    const uint32_t lane_row = (uint32_t)(8 * g + (col >> 2));
    bf16x8 zf[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) zf[c] = read_transposed(z_own + slot + lane_row * ZP + (uint32_t)(32 * c + 8 * (col & 3)), ZP);
#pragma unroll
    for (int q = 0; q < TERMS; ++q)
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        const bf16x8 vf = read_transposed(v_all + slot + (uint32_t)(q * 32 * VP) + lane_row * VP + (uint32_t)(32 * f + 8 * (col & 3)), VP);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[c][f] = NK ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, zf[c], acc[c][f], 0, 0, 0)
                         : __builtin_amdgcn_mfma_f32_16x16x32_bf16(zf[c], vf, acc[c][f], 0, 0, 0);
      }
  };

  for (int64_t from = 0; from < chunks; from += kGradList) {
    const int n = (int)(chunks - from < kGradList ? chunks - from : kGradList);
    if (p.splits == 1 || p.adapters == 1 || chunks > kGradList) look_through(from, n, false);
    __syncthreads();
    // the list: a thread to a chunk, 64 chunks a wave at a time
    int total = 0;
    for (int b = 0; b < n; b += WAVES * 64) {
      const int c = b + tid;
      bool any = c < n && kinds[c] == a;
      if (c < n && kinds[c] == -2)
        for (int i = 0; i < 32; ++i) any |= adapter_of(p, (from + c) * 32 + i) == a;
      const uint64_t m = __ballot(any);
      if (lane == 0) found[wave] = __popcll(m);
      __syncthreads();
      int at = total;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        at += w < wave ? found[w] : 0;
        total += found[w];
      }
      if (any) list[at + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)c;
      __syncthreads();
    }
    total = __builtin_amdgcn_readfirstlane(total);
    const int lo = (int)((int64_t)total * part / parts), hi = (int)((int64_t)total * (part + 1) / parts);
    if (lo == hi) continue;                    // (for the whole workgroup; the list is not used again)
    Chunk k[DEEP];
    auto first_row = [&](int i) { return (from + __builtin_amdgcn_readfirstlane(list[i < hi ? i : hi - 1])) * 32; };
    auto fetch = [&](int i, Chunk& c) {
      load(first_row(i), c);
      loads_first();
    };
#pragma unroll
    for (int d = 0; d < DEEP; ++d) fetch(lo + d, k[d]);
    write(k[0], first_row(lo), 0);
    fetch(lo + DEEP, k[0]);
    wait_lds_all();
    __builtin_amdgcn_s_barrier();
    uint32_t slot = 0;
    for (int i = lo; i < hi; i += DEEP)
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        if (i + d >= hi) break;
        // the next chunk goes into the other slot while this one is computed with (behind the last one: once more)
        write(k[(d + 1) % DEEP], first_row(i + d + 1), SLOT - slot);
        fetch(i + d + 1 + DEEP, k[(d + 1) % DEEP]);
        compute(slot);
        slot = SLOT - slot;
        wait_lds_all();
        __builtin_amdgcn_s_barrier();
      }
    __syncthreads();
  }
  if (!live) return;
  bool nan = false;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
      for (int e = 0; e < 4; e += 2) nan |= __builtin_isunordered(acc[c][f][e], acc[c][f][e + 1]);
  if (__ballot(nan)) {
    // This wave's sums once more, from V as it is, over the same chunks: a lane takes its elements row by row.  Slow (8192
    // rows x 4096, rank 16 27 -> 280 us), but only where Z or V hold NaN or infinities: other calls take up to 2 % longer for
    // it, 3 to 5 if this were the loop above again.
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int f = 0; f < FR; ++f) acc[c][f] = f32x4{};
    auto rows_of = [&](int64_t chunk) { return (uint32_t)__ballot(adapter_of(p, chunk * 32 + (lane & 31)) == a); };
#pragma unroll 1
    for (int64_t from = 0; from < chunks; from += kGradList) {
      const int64_t end = from + kGradList < chunks ? from + kGradList : chunks;
      int total = 0, i = 0;
#pragma unroll 1
      for (int64_t chunk = from; chunk < end; ++chunk) total += rows_of(chunk) != 0;
      const int lo = (int)((int64_t)total * part / parts), hi = (int)((int64_t)total * (part + 1) / parts);
#pragma unroll 1
      for (int64_t chunk = from; chunk < end; ++chunk) {
        uint32_t rows = rows_of(chunk);
        if (!rows || i++ < lo || i > hi) continue;
#pragma unroll 1
        for (; rows; rows &= rows - 1) {
          const int64_t t = chunk * 32 + __builtin_ctz(rows);
          const uint16_t* z = p.X + t * p.ldx;
          const float* v = p.V + t * p.ldv;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int64_t n = c0 + 16 * c + (NK ? col : 4 * g + e);
              const float zf = bf16_low(z[n < p.cols ? n : p.cols - 1]);
#pragma unroll
              for (int f = 0; f < FR; ++f) {
                const int r = r0 + 16 * f + (NK ? 4 * g + e : col);
                acc[c][f][e] = __builtin_fmaf(zf, v[r < p.rank ? r : p.rank - 1], acc[c][f][e]);
              }
            }
        }
      }
    }
  }
  // NK: a lane holds column l % 16 and 4 ranks of a fragment, else rank l % 16 and 4 columns
  const int64_t line = NK ? p.rank : p.all_cols;                         // of the sums of a part
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int f = 0; f < FR; ++f) {
      const int64_t n = c0 + 16 * c + (NK ? col : 4 * g);
      const int r = r0 + 16 * f + (NK ? 4 * g : col);
      if (n >= p.cols || r >= p.rank) continue;
      const int64_t inside = NK ? p.rank - r : p.cols - n;               // of the 4
      const f32x4 v = acc[c][f];
      if (parts > 1) {
        float* to = p.sums + (int64_t)(first_part + part) * p.all_cols * p.rank + (NK ? (p.first_col + n) * line + r : r * line + p.first_col + n);
        store4(to, v, inside);
      } else {
        const int64_t at = (int64_t)a * p.stride_y + (NK ? n * p.ldy + r : r * p.ldy + n);
        if constexpr (OB) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < inside) reinterpret_cast<__bf16*>(p.Y)[at + e] = (__bf16)v[e];
        } else {
          store4(reinterpret_cast<float*>(p.Y) + at, v, inside);
        }
      }
    }
}

// G of an adapter from the sums of its parts, in their order; a thread takes an element.
template <bool OB>
__global__ __launch_bounds__(256) void lora_grad_sum(LoraParams p, int64_t lines, int64_t line) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = lines * line;
  const int first = p.parts[2 * blockIdx.y], parts = p.parts[2 * blockIdx.y + 1];
  if (i >= n || parts < 2) return;
  const float* s = p.sums + first * n + i;
  float v = 0.f;
  for (int k = 0; k < parts; k += 8) {
    float part[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) part[u] = s[(k + u < parts ? k + u : parts - 1) * n];
    loads_first();
#pragma unroll
    for (int u = 0; u < 8; ++u) v = k + u < parts ? v + part[u] : v;
  }
  const int64_t row = (uint32_t)i / (uint32_t)line, to = blockIdx.y * p.stride_y + row * p.ldy + (i - row * line);
  if constexpr (OB) reinterpret_cast<__bf16*>(p.Y)[to] = (__bf16)v;
  else reinterpret_cast<float*>(p.Y)[to] = v;
}

hipError_t launch_row_down(const LoraParams& p, bool nk, hipStream_t stream) {
  if (nk) {
    const bool one = lora_row_ranks(p.rows, p.rank) == 1;
    const int64_t jobs = p.rows * (one ? p.rank : (p.rank + 3) / 4);
    return launch_kernel(one ? lora_row_down_nk<1> : lora_row_down_nk<4>, dim3((unsigned)((jobs + 3) / 4)), dim3(256), 0, stream, p);
  }
  const dim3 grid((unsigned)p.rows), block(kRowWaves * 64);
  switch (lora_row_lanes(p.rank, 32)) {
    case 1: return launch_kernel(lora_row_down_kn<1>, grid, block, 0, stream, p);
    case 2: return launch_kernel(lora_row_down_kn<2>, grid, block, 0, stream, p);
    case 4: return launch_kernel(lora_row_down_kn<4>, grid, block, 0, stream, p);
    case 8: return launch_kernel(lora_row_down_kn<8>, grid, block, 0, stream, p);
    case 16: return launch_kernel(lora_row_down_kn<16>, grid, block, 0, stream, p);
    default: return launch_kernel(lora_row_down_kn<32>, grid, block, 0, stream, p);
  }
}

template <bool OB>
hipError_t launch_row_up(const LoraParams& p, bool nk, hipStream_t stream) {
  const dim3 block(256);
  if (!nk) return launch_kernel(lora_row_up_kn<OB>, dim3((unsigned)((p.cols + 2047) / 2048), (unsigned)p.rows), block, 0, stream, p);
  const int lanes = lora_row_lanes(p.rank, 8);
  const dim3 grid((unsigned)((p.cols + 1024 / lanes - 1) / (1024 / lanes)), (unsigned)p.rows);
  switch (lanes) {
    case 1: return launch_kernel(lora_row_up_nk<1, OB>, grid, block, 0, stream, p);
    case 2: return launch_kernel(lora_row_up_nk<2, OB>, grid, block, 0, stream, p);
    case 4: return launch_kernel(lora_row_up_nk<4, OB>, grid, block, 0, stream, p);
    default: return launch_kernel(lora_row_up_nk<8, OB>, grid, block, 0, stream, p);
  }
}

}  // namespace

hipError_t launch_lora_down(const LoraParams& p, bool nk, hipStream_t stream) {
  return lora_by_rows(p.rows, p.cols, p.rank) ? launch_row_down(p, nk, stream) : launch_lora_down_tiles(p, nk, stream);
}

template <int NC, bool NK, bool OB>
static hipError_t up_launch(const LoraParams& p, int num_cus, hipStream_t stream) {
  const unsigned across = (unsigned)((p.cols + lora_up_columns(NC, OB) - 1) / lora_up_columns(NC, OB));
  if (lora_up_tiles(p.rows, p.cols, p.rank, OB, num_cus) == 4)
    return launch_kernel(lora_up_kernel<4, NC, NK, OB>, dim3(across, (unsigned)((p.rows + 255) / 256)), dim3(256), 0, stream, p);
  return launch_kernel(lora_up_kernel<1, NC, NK, OB>, dim3(across, (unsigned)((p.rows + 63) / 64)), dim3(256), 0, stream, p);
}

template <bool NK, bool OB>
static hipError_t up_rank(const LoraParams& p, int num_cus, hipStream_t stream) {
  switch (lora_up_chunks(p.rank)) {
    case 1: return up_launch<1, NK, OB>(p, num_cus, stream);
    case 2: return up_launch<2, NK, OB>(p, num_cus, stream);
    case 4: return up_launch<4, NK, OB>(p, num_cus, stream);
    default: return up_launch<8, NK, OB>(p, num_cus, stream);
  }
}

hipError_t launch_lora_up(const LoraParams& p, bool nk, bool bf16, int num_cus, hipStream_t stream) {
  if (lora_by_rows(p.rows, p.cols, p.rank)) return bf16 ? launch_row_up<true>(p, nk, stream) : launch_row_up<false>(p, nk, stream);
  return nk ? (bf16 ? up_rank<true, true>(p, num_cus, stream) : up_rank<true, false>(p, num_cus, stream))
            : (bf16 ? up_rank<false, true>(p, num_cus, stream) : up_rank<false, false>(p, num_cus, stream));
}

template <bool NK, bool OB>
static hipError_t wgrad_launch(const LoraParams& all, hipStream_t stream) {
  const bool narrow = lora_grad_narrow(all.cols, all.rank);
  const int fr = lora_grad_ranks(all.cols, all.rank);
  const auto kernel = narrow    ? lora_wgrad_kernel<1, true, NK, OB>
                      : fr == 1 ? lora_wgrad_kernel<1, false, NK, OB>
                      : fr == 2 ? lora_wgrad_kernel<2, false, NK, OB>
                      : fr == 3 ? lora_wgrad_kernel<3, false, NK, OB>
                                : lora_wgrad_kernel<4, false, NK, OB>;
  const int64_t across = (all.cols + kGradColumns - 1) / kGradColumns;
  const int64_t ranks = (all.rank + 16 * fr - 1) / (16 * fr), threads = kGradWaves * 64;
  LoraParams p = all;
  p.all_cols = all.cols;
  if (all.splits > 1) {
    // (an adapter has a part at least, and all of them together `splits` more at most)
    const int64_t most = all.adapters == 1 ? all.splits : all.adapters + all.splits;
    hipError_t e = launch_kernel(kernel, dim3((unsigned)across, (unsigned)ranks, (unsigned)most), dim3((unsigned)threads), 0, stream, p);
    if (e != hipSuccess) return e;
    const int64_t lines = NK ? all.cols : all.rank, line = NK ? all.rank : all.cols;
    return launch_kernel(lora_grad_sum<OB>, dim3((unsigned)((lines * line + 255) / 256), (unsigned)all.adapters), dim3(256), 0,
                         stream, p, lines, line);
  }
  // launches of less than 2^31 threads
  const int64_t width = across < (1 << 14) ? across : 1 << 14;
  int64_t deep = ((int64_t)1 << 31) / (width * ranks * threads);
  deep = deep < 1 ? 1 : deep > 32768 ? 32768 : deep;
  for (int64_t first = 0; first < all.adapters; first += deep)
    for (int64_t c = 0; c < across; c += width) {
      p.first_adapter = (int)first;
      p.first_col = c * kGradColumns;
      p.X = all.X + p.first_col;
      p.cols = all.cols - p.first_col < width * kGradColumns ? all.cols - p.first_col : width * kGradColumns;
      p.Y = static_cast<char*>(all.Y) + p.first_col * (NK ? all.ldy : 1) * (OB ? 2 : 4);
      const dim3 grid((unsigned)((p.cols + kGradColumns - 1) / kGradColumns), (unsigned)ranks,
                      (unsigned)(all.adapters - first < deep ? all.adapters - first : deep));
      const hipError_t e = launch_kernel(kernel, grid, dim3((unsigned)threads), 0, stream, p);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

hipError_t launch_lora_wgrad(const LoraParams& p, bool nk, bool bf16, hipStream_t stream) {
  return nk ? (bf16 ? wgrad_launch<true, true>(p, stream) : wgrad_launch<true, false>(p, stream))
            : (bf16 ? wgrad_launch<false, true>(p, stream) : wgrad_launch<false, false>(p, stream));
}

}  // namespace sfc
