// Low-rank adapters of many requests beside a shared projection, for gfx950.
//
//   down      V[t] = s[a] X[t] A[a]^T            a = ids[t], zeros where there is none
//   up        Y[t] = base[t] + V[t] B[a]^T       base[t] where there is none
//   gradient  G[a] = sum over t with ids[t] = a of Z[t]^T V[t]
//
// with ranks of a few to a few hundred: X, base and Y are read and written once, and that
// traffic is what bounds them; the products are small beside it.  V is fp32.  Where it meets bf16 weights in
// MFMAs it is taken apart into bf16 terms of the same sign, each the leading 8 bits of what the ones before
// leave, the last one rounded: two are off by at most 2^-16 of it (bf16 results, which are rounded to 2^-8),
// three hold every bit of it (fp32 results).
//
// A wave takes 16 rows.  They may belong to up to 16 adapters: it computes with one
// adapter after the other and keeps the results of that adapter's rows, so no row sees another
// adapter's weights, infinities and NaN among them.
#include "sfc_gemm_kernel.h"
#include "sfc_launch.h"
#include "sfc_lora_params.h"
#include "sfc_row_io.h"

namespace sfc {

namespace {

__device__ __forceinline__ bf16x8 as_bf16x8(const row_u32x4& v) { return __builtin_bit_cast(bf16x8, v); }

// 8 elements of a bf16 row from column c on; zeros past its end.
__device__ __forceinline__ bf16x8 load_bf16x8(const uint16_t* row, int64_t c, int64_t cols) {
  return as_bf16x8(load8<true>(row, c, cols).w[0]);
}

// The adapter of row t, or -1.
__device__ __forceinline__ int adapter_of(const LoraParams& p, int64_t t) {
  const int a = t < p.rows ? p.ids[t] : -1;
  return a >= 0 && a < p.adapters ? a : -1;
}

// Leading bf16 terms of 8 fp32 values.
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&v)[8], bf16x8 (&out)[TERMS]) {
  uint32_t w[TERMS][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t h[TERMS][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float rest = v[2 * i + e];
      const bool finite = __builtin_fabsf(rest) < __builtin_inff();
#pragma unroll
      for (int k = 0; k < TERMS; ++k) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, rest);
        // (a NaN whose payload lies in the lower half alone has to stay one)
        if (k == 0) h[k][e] = (bits >> 16) | (rest != rest ? 0x40u : 0u);
        else if (k + 1 < TERMS) h[k][e] = bits >> 16;
        else h[k][e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)rest);
        rest = finite ? rest - __builtin_bit_cast(float, bits & 0xFFFF0000u) : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < TERMS; ++k) w[k][i] = h[k][0] | (h[k][1] << 16);
  }
#pragma unroll
  for (int k = 0; k < TERMS; ++k) out[k] = __builtin_bit_cast(bf16x8, u32x4{w[k][0], w[k][1], w[k][2], w[k][3]});
}

// Transposing read of 32 rows x 16 columns: lane l gets column column0(l % 16) of rows 8 (l / 16) .. + 7,
// from LDS rows `pitch` bytes apart; `at` is this lane's address, row 8 (l / 16) + (l % 16) / 4 and the
// first of 4 columns.
__device__ __forceinline__ bf16x8 read_transposed(uint32_t at, int pitch) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)at);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)(at + (uint32_t)(4 * pitch)));
  const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

// ---- down ------------------------------------------------------------------------------------

constexpr int kDownWaves = 8;

// A workgroup takes 16 rows and 16 FR ranks; its waves deal K out in blocks of 64 and add up
// through LDS, in the order of the waves.  Weights that lie along the ranks (KN) pass
// through a wave's own LDS and the transposing read.
template <int FR, bool NK>
__global__ __launch_bounds__(kDownWaves * 64) void lora_down_kernel(LoraParams p) {
  constexpr int PITCH = 16 * FR * 2 + 16;
  __shared__ __attribute__((aligned(16))) float sums[kDownWaves][16][16 * FR + 4];
  __shared__ __attribute__((aligned(16))) unsigned char slab[NK ? 16 : kDownWaves * 32 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int64_t t0 = (int64_t)blockIdx.x * 16;
  const int r0 = blockIdx.y * 16 * FR;
  const int64_t row = t0 + col < p.rows ? t0 + col : p.rows - 1;
  const uint16_t* x = p.X + row * p.ldx;
  const int id = adapter_of(p, t0 + col);
  const uint32_t own = lds_addr(slab) + (uint32_t)(NK ? 0 : wave * 32 * PITCH);

  // rows without an adapter
  for (int i = tid; i < 16 * 16 * FR; i += kDownWaves * 64) {
    const int tr = i / (16 * FR), r = r0 + i % (16 * FR);
    if (t0 + tr < p.rows && r < p.rank && adapter_of(p, t0 + tr) < 0) p.V[(t0 + tr) * p.ldv + r] = 0.f;
  }
  uint32_t pending = (uint32_t)__ballot(id >= 0) & 0xFFFFu;
  while (pending) {
    const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(pending));
    pending &= ~(uint32_t)__ballot(id == a);
    const uint16_t* w = p.W + (int64_t)a * p.stride_w;
    f32x4 acc[FR] = {};
    for (int64_t kb = (int64_t)wave * 64; kb < p.cols; kb += kDownWaves * 64) {
      bf16x8 xf[2], wf[2][FR];
#pragma unroll
      for (int s = 0; s < 2; ++s) xf[s] = load_bf16x8(x, kb + 32 * s + 8 * g, p.cols);
      if constexpr (NK) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int f = 0; f < FR; ++f) {
            const int r = r0 + 16 * f + col;
            wf[s][f] = r < p.rank ? load_bf16x8(w + (int64_t)r * p.ldw, kb + 32 * s + 8 * g, p.cols) : bf16x8{};
          }
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          // 32 rows of 16 FR ranks, 8 of them a lane
#pragma unroll
          for (int i = lane; i < 32 * 2 * FR; i += 64) {
            const int k = i / (2 * FR), c = i % (2 * FR);
            const int64_t kk = kb + 32 * s + k;
            const row_u32x4 v = kk < p.cols ? load8<true>(w + kk * p.ldw, r0 + 8 * c, p.rank).w[0] : row_u32x4{};
            lds_write16(own + (uint32_t)(k * PITCH + 16 * c), v);
          }
          wait_lds_all();
#pragma unroll
          for (int f = 0; f < FR; ++f)
            wf[s][f] = read_transposed(own + (uint32_t)((8 * g + (col >> 2)) * PITCH + 32 * f + 8 * (col & 3)), PITCH);
          wait_lds_all();
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int f = 0; f < FR; ++f) acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[s][f], xf[s], acc[f], 0, 0, 0);
    }
    // lane: row l % 16, ranks 4 (l / 16) .. + 3 of every fragment
#pragma unroll
    for (int f = 0; f < FR; ++f) *reinterpret_cast<f32x4*>(&sums[wave][col][16 * f + 4 * g]) = acc[f];
    __syncthreads();
    const float scale = p.scales ? p.scales[a] : 1.f;
    for (int i = tid; i < 16 * 16 * FR; i += kDownWaves * 64) {
      const int tr = i / (16 * FR), r = i % (16 * FR);
      if (r0 + r < p.rank && adapter_of(p, t0 + tr) == a) {
        float v = sums[0][tr][r];
#pragma unroll
        for (int k = 1; k < kDownWaves; ++k) v += sums[k][tr][r];
        p.V[(t0 + tr) * p.ldv + r0 + r] = scale * v;
      }
    }
    __syncthreads();
  }
}

// ---- up --------------------------------------------------------------------------------------

constexpr int kUpColumns = 64;         // columns of a unit: a lane's part of a row is 16 of them
constexpr int kUpUnits = 4;            // units of a wave

// Column of a unit that lane n of fragment j computes.  bf16: a lane ends with 4 columns of each of 4
// fragments, which make 16 in a row, 32 bytes; fp32: 4 columns of a fragment are 16 bytes.
template <bool OB>
__device__ __forceinline__ int up_column(int j, int n) {
  return OB ? 16 * (n >> 2) + 4 * j + (n & 3) : 16 * j + n;
}

// A workgroup takes 64 rows, 16 a wave, and up to kUpUnits units of columns; ranks in chunks of 32, of
// which a wave keeps its rows' terms in registers.
template <int NC, bool NK, bool OB>
__global__ __launch_bounds__(256) void lora_up_kernel(LoraParams p) {
  constexpr int TERMS = OB ? 2 : 3;
  constexpr int PITCH = kUpColumns * 2 + 16;
  __shared__ __attribute__((aligned(16))) unsigned char slab[NK ? 16 : 4 * 32 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * 16;
  if (t0 >= p.rows) return;
  const bool live = t0 + col < p.rows;
  const int64_t row = live ? t0 + col : p.rows - 1;
  const int id = adapter_of(p, t0 + col);
  const uint32_t own = lds_addr(slab) + (uint32_t)(NK ? 0 : wave * 32 * PITCH);
  bf16x8 vf[NC][TERMS];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = 32 * c + 8 * g + e;
      v[e] = r < p.rank && id >= 0 ? p.V[row * p.ldv + r] : 0.f;
    }
    split_terms<TERMS>(v, vf[c]);
  }
  const uint32_t all = (uint32_t)__ballot(id >= 0) & 0xFFFFu;
  for (int u = 0; u < kUpUnits; ++u) {
    const int64_t n0 = ((int64_t)blockIdx.y * kUpUnits + u) * kUpColumns;
    if (n0 >= p.cols) break;
    float y[16];
    // this lane's columns: OB 16 in a row, else 4 of every fragment
    if (p.base) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (OB) {
          to_float<true>(load8<true>(reinterpret_cast<const uint16_t*>(p.base) + row * p.ld_base, n0 + 16 * g + 8 * h, p.cols), y + 8 * h);
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int64_t n = n0 + 16 * (2 * h + (q >> 2)) + 4 * g + (q & 3);
            y[8 * h + q] = n < p.cols ? reinterpret_cast<const float*>(p.base)[row * p.ld_base + n] : 0.f;
          }
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = 0.f;
    }
    uint32_t pending = all;
    while (pending) {
      const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(pending));
      pending &= ~(uint32_t)__ballot(id == a);
      const uint16_t* w = p.W + (int64_t)a * p.stride_w;
      f32x4 acc[4] = {};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (32 * c >= p.rank) break;
        bf16x8 wf[4];
        if constexpr (NK) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + up_column<OB>(j, col);
            wf[j] = n < p.cols ? load_bf16x8(w + n * p.ldw, 32 * c + 8 * g, p.rank) : bf16x8{};
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3), cc = 8 * (lane & 7);
            const row_u32x4 v = 32 * c + r < p.rank && n0 + cc < p.cols
                                    ? load8<true>(w + (int64_t)(32 * c + r) * p.ldw, n0 + cc, p.cols).w[0] : row_u32x4{};
            lds_write16(own + (uint32_t)(r * PITCH + 2 * cc), v);
          }
          wait_lds_all();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            wf[j] = read_transposed(own + (uint32_t)((8 * g + (col >> 2)) * PITCH + 2 * up_column<OB>(j, 4 * (col & 3))), PITCH);
          wait_lds_all();
        }
#pragma unroll
        for (int k = 0; k < TERMS; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], vf[c][k], acc[j], 0, 0, 0);
      }
      const bool mine = id == a;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[4 * j + e] = mine ? y[4 * j + e] + acc[j][e] : y[4 * j + e];
    }
    if (live) {
      if constexpr (OB) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          store8<true, false>(reinterpret_cast<uint16_t*>(p.Y) + row * p.ldy, n0 + 16 * g + 8 * h, p.cols, from_float<true>(y + 8 * h));
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t n = n0 + 16 * (e >> 2) + 4 * g + (e & 3);
          if (n < p.cols) reinterpret_cast<float*>(p.Y)[row * p.ldy + n] = y[e];
        }
      }
    }
  }
}

// ---- gradient of the weights -------------------------------------------------------------------

constexpr int kGradWaves = 8, kGradColumns = 64;

// A workgroup takes an adapter, 64 columns of Z and 16 FR ranks; its waves deal the rows out in chunks of
// 32, leave out chunks without a row of the adapter, and add up through LDS in the order of the
// waves.  In a chunk, rows of other adapters are zeros in both operands.
template <int FR, bool NK, bool OB>
__global__ __launch_bounds__(kGradWaves * 64) void lora_wgrad_kernel(LoraParams p) {
  constexpr int TERMS = 3, FC = kGradColumns / 16;
  constexpr int ZP = kGradColumns * 2 + 16, VP = 16 * FR * 2 + 16;       // bytes from row to row
  constexpr int WAVE = 32 * ZP + TERMS * 32 * VP;
  constexpr int SUMS = 16 * FC * (16 * FR + 4) * 4;                       // bytes of a wave's sums
  __shared__ __attribute__((aligned(16))) unsigned char smem[kGradWaves * WAVE > SUMS ? kGradWaves * WAVE : SUMS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int64_t c0 = (int64_t)blockIdx.x * kGradColumns;
  const int r0 = blockIdx.y * 16 * FR, a = p.first_adapter + (int)blockIdx.z;
  const uint32_t z_own = lds_addr(smem) + (uint32_t)(wave * WAVE), v_own = z_own + 32 * ZP;
  f32x4 acc[FC][FR] = {};
  for (int64_t t0 = (int64_t)wave * 32; t0 < p.rows; t0 += kGradWaves * 32) {
    const uint32_t mine = (uint32_t)__ballot(lane < 32 && adapter_of(p, t0 + lane) == a);
    if (!mine) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 8 * i + (lane >> 3), c = 8 * (lane & 7);
      const row_u32x4 v = (mine >> t & 1) && c0 + c < p.cols ? load8<true>(p.X + (t0 + t) * p.ldx, c0 + c, p.cols).w[0] : row_u32x4{};
      lds_write16(z_own + (uint32_t)(t * ZP + 2 * c), v);
    }
#pragma unroll
    for (int i = lane; i < 32 * 2 * FR; i += 64) {
      const int t = i / (2 * FR), r = 8 * (i % (2 * FR));
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (mine >> t & 1) && r0 + r + e < p.rank ? p.V[(t0 + t) * p.ldv + r0 + r + e] : 0.f;
      bf16x8 terms[TERMS];
      split_terms<TERMS>(v, terms);
#pragma unroll
      for (int k = 0; k < TERMS; ++k)
        lds_write16(v_own + (uint32_t)(k * 32 * VP + t * VP + 2 * r), __builtin_bit_cast(u32x4, terms[k]));
    }
    wait_lds_all();
    const uint32_t lane_row = (uint32_t)(8 * g + (col >> 2));
    bf16x8 zf[FC];
#pragma unroll
    for (int c = 0; c < FC; ++c) zf[c] = read_transposed(z_own + lane_row * ZP + (uint32_t)(32 * c + 8 * (col & 3)), ZP);
#pragma unroll
    for (int k = 0; k < TERMS; ++k)
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        const bf16x8 vf = read_transposed(v_own + (uint32_t)(k * 32 * VP) + lane_row * VP + (uint32_t)(32 * f + 8 * (col & 3)), VP);
#pragma unroll
        for (int c = 0; c < FC; ++c)
          acc[c][f] = NK ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, zf[c], acc[c][f], 0, 0, 0)
                         : __builtin_amdgcn_mfma_f32_16x16x32_bf16(zf[c], vf, acc[c][f], 0, 0, 0);
      }
    wait_lds_all();
  }
  // Sums of the waves, one after the other.  NK: a lane holds column l % 16 and 4 ranks of a fragment,
  // else rank l % 16 and 4 columns.
  float* sums = reinterpret_cast<float*>(smem);
  constexpr int SP = 16 * FR + 4;
  for (int w = 0; w < kGradWaves; ++w) {
    __syncthreads();
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < FC; ++c)
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float& s = NK ? sums[(16 * c + col) * SP + 16 * f + 4 * g + e] : sums[(16 * c + 4 * g + e) * SP + 16 * f + col];
            s = w == 0 ? acc[c][f][e] : s + acc[c][f][e];
          }
    }
  }
  __syncthreads();
  for (int i = tid; i < kGradColumns * 16 * FR; i += kGradWaves * 64) {
    const int c = NK ? i / (16 * FR) : i % kGradColumns, r = NK ? i % (16 * FR) : i / kGradColumns;
    if (c0 + c >= p.cols || r0 + r >= p.rank) continue;
    const int64_t at = (int64_t)a * p.stride_y + (NK ? (c0 + c) * p.ldy + r0 + r : (int64_t)(r0 + r) * p.ldy + c0 + c);
    if constexpr (OB) reinterpret_cast<__bf16*>(p.Y)[at] = (__bf16)sums[c * SP + r];
    else reinterpret_cast<float*>(p.Y)[at] = sums[c * SP + r];
  }
}

}  // namespace

hipError_t launch_lora_down(const LoraParams& p, bool nk, int num_cus, hipStream_t stream) {
  const int fr = p.rank <= 16 ? 1 : p.rank <= 32 ? 2 : 4;
  const dim3 grid((unsigned)((p.rows + 15) / 16), (unsigned)((p.rank + 16 * fr - 1) / (16 * fr))), block(kDownWaves * 64);
  if (fr == 1) return launch_kernel(nk ? lora_down_kernel<1, true> : lora_down_kernel<1, false>, grid, block, 0, stream, p);
  if (fr == 2) return launch_kernel(nk ? lora_down_kernel<2, true> : lora_down_kernel<2, false>, grid, block, 0, stream, p);
  return launch_kernel(nk ? lora_down_kernel<4, true> : lora_down_kernel<4, false>, grid, block, 0, stream, p);
}

template <bool NK, bool OB>
static hipError_t up_launch(const LoraParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)((p.rows + 63) / 64), (unsigned)((p.cols + kUpUnits * kUpColumns - 1) / (kUpUnits * kUpColumns))), block(256);
  if (p.rank <= 32) return launch_kernel(lora_up_kernel<1, NK, OB>, grid, block, 0, stream, p);
  if (p.rank <= 64) return launch_kernel(lora_up_kernel<2, NK, OB>, grid, block, 0, stream, p);
  if (p.rank <= 128) return launch_kernel(lora_up_kernel<4, NK, OB>, grid, block, 0, stream, p);
  return launch_kernel(lora_up_kernel<8, NK, OB>, grid, block, 0, stream, p);
}

hipError_t launch_lora_up(const LoraParams& p, bool nk, bool bf16, int num_cus, hipStream_t stream) {
  return nk ? (bf16 ? up_launch<true, true>(p, stream) : up_launch<true, false>(p, stream))
            : (bf16 ? up_launch<false, true>(p, stream) : up_launch<false, false>(p, stream));
}

template <bool NK, bool OB>
static hipError_t wgrad_launch(const LoraParams& all, hipStream_t stream) {
  const int fr = all.rank <= 16 ? 1 : all.rank <= 32 ? 2 : 4;
  const int64_t across = (all.cols + kGradColumns - 1) / kGradColumns, ranks = (all.rank + 16 * fr - 1) / (16 * fr);
  // launches of less than 2^31 threads
  LoraParams p = all;
  const int64_t width = across < (1 << 20) ? across : 1 << 20;
  int64_t deep = ((int64_t)1 << 31) / (width * ranks * kGradWaves * 64);
  deep = deep < 1 ? 1 : deep > 32768 ? 32768 : deep;
  for (int64_t first = 0; first < all.adapters; first += deep)
    for (int64_t c = 0; c < across; c += width) {
      p.first_adapter = (int)first;
      p.X = all.X + c * kGradColumns;
      p.cols = all.cols - c * kGradColumns < width * kGradColumns ? all.cols - c * kGradColumns : width * kGradColumns;
      p.Y = static_cast<char*>(all.Y) + c * kGradColumns * (NK ? all.ldy : 1) * (OB ? 2 : 4);
      const dim3 grid((unsigned)((p.cols + kGradColumns - 1) / kGradColumns), (unsigned)ranks,
                      (unsigned)(all.adapters - first < deep ? all.adapters - first : deep));
      const dim3 block(kGradWaves * 64);
      const hipError_t e = launch_kernel(fr == 1   ? lora_wgrad_kernel<1, NK, OB>
                                         : fr == 2 ? lora_wgrad_kernel<2, NK, OB>
                                                   : lora_wgrad_kernel<4, NK, OB>, grid, block, 0, stream, p);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

hipError_t launch_lora_wgrad(const LoraParams& p, bool nk, bool bf16, int num_cus, hipStream_t stream) {
  return nk ? (bf16 ? wgrad_launch<true, true>(p, stream) : wgrad_launch<true, false>(p, stream))
            : (bf16 ? wgrad_launch<false, true>(p, stream) : wgrad_launch<false, false>(p, stream));
}

}  // namespace sfc
