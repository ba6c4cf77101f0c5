// MFMA product of microscaled 4-bit operands for gfx950, C = A B^T with both operands
// contiguous along K.
//
//   C[m][n] = sum_b 2^(sA[m][b] - 127) 2^(sB[n][b] - 127) sum_{k in block b} a[m][k] b[n][k]
//
// over blocks b of 32 values; MFMA 32x32x64 f8f6f4 takes two blocks of 4-bit elements of
// 32 rows with one scale byte per row and block, and accumulates in fp32.
//
// Mapping.  A workgroup of 4 waves (2 x 2) computes a BM x BN block.  K runs in stages of
// 128 values: 64 bytes of codes per row, in a ring of four LDS slots that buffer loads
// fill straight from memory, and 16 bytes of scales per row for four stages, in a ring of
// two.  During stage t the loads of stage t+4 go out; one barrier per stage, between its
// two MFMA steps, where all waves have read stage t and the loads of stage t+1 have
// landed: behind it slot t is free and slot t+1 may be read.
//   * lane l of a fragment holds row l%32 and, in step s, block 2*(l/32) + s of the stage:
//     its two scale bytes lie side by side, and the MFMA selects one by an immediate;
//   * 16-byte chunk c of row r is stored at chunk c ^ ((r >> 2) & 3): 16 consecutive rows
//     read at one logical chunk touch the 16 16-byte bank groups;
//   * rows past M or N and blocks outside the range of K are loaded as zeros (lanes past
//     the descriptor's range); scale bytes outside the range are masked to code 0, because
//     a NaN scale makes even zeros NaN;
//   * the MFMA takes B first, so a lane ends with one row of C and runs of 4 columns; the
//     block leaves through LDS, a wave's 32-row strips at a time, as whole row segments.
#pragma once
#include "sfc_gemm_kernel.h"
#include "sfc_ops_params.h"

namespace sfc {

typedef __attribute__((address_space(3))) const i32x4 lds_ci32x4;
typedef __attribute__((address_space(3))) const uint16_t lds_cu16;

constexpr int kMxStage = 128;                   // values of K in a stage
constexpr int kMxRing = 4;                      // stages in LDS
constexpr int kMxScaleStages = 4;               // stages that one load of scales covers

template <int BM, int BN>
struct MxTile {
  static constexpr int THREADS = 256;
  static constexpr int WTM = BM / 2, WTN = BN / 2;            // a wave's part
  static constexpr int FM = WTM / 32, FN = WTN / 32;          // fragments of 32 rows
  static constexpr int A_BYTES = BM * 64, B_BYTES = BN * 64, SLOT = A_BYTES + B_BYTES;
  static constexpr int AL = A_BYTES / 1024 / 4, BL = B_BYTES / 1024 / 4;   // loads per wave and stage
  static constexpr int SA_OFF = kMxRing * SLOT;               // scale ring
  static constexpr int S_SLOT = (BM + BN) * 16;
  static constexpr int LDS = SA_OFF + 2 * S_SLOT;
  static constexpr int LOADS = AL + BL;
  static constexpr int PER_CU = BM == 256 ? 1 : 2;            // workgroups
  // epilogue: a wave's strip of 32 rows, fp32, rows 16 bytes apart from a multiple of 256
  static constexpr int RS = WTN * 4 + 16;
  static_assert(4 * 32 * RS <= SA_OFF, "strips fit the ring");
  static_assert(PER_CU * (LDS + 4 * (kMaxExperts + 2)) <= 160 * 1024, "LDS of one CU");
};

__device__ __forceinline__ void mx_dma16(const i32x4& rsrc, uint32_t lds, int voffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(voffset), "s"(rsrc) : "memory");
}

// One operand's rows of a block: where its loads start.
struct MxSide {
  uint64_t codes, scales;      // first byte of the stage / of the scale chunk to load next
  uint32_t scale_range;        // bytes from `scales` to the end of the last row's scales
};

__device__ __forceinline__ i32x8 mx_wide(const i32x4& v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}

// What a workgroup computes in one go: a block of C over a range of blocks of K.
struct MxTask {
  int64_t a_row, b_row;        // first row of A and of B
  int64_t c_row;               // first row of C (relative to C)
  int m_valid, n_valid;        // rows of A and of B inside the matrix
  int64_t block0;              // first block of K (a multiple of 4), with `lo` blocks to skip
  int lo, hi;                  // blocks lo .. hi-1 from block0 count
  const uint8_t *B, *Bs;
  char* C;
};

template <int BM, int BN, bool OB, bool FULL>
__device__ __forceinline__ void mx_store(const Mx4GemmParams& p, const MxTask& t, f32x16 (&acc)[BM / 64][BN / 64],
                                         uint32_t lds0, int wave, int lane) {
  using T = MxTile<BM, BN>;
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t strip = lds0 + (uint32_t)(wave * 32 * T::RS);
  const int h = lane >> 5;
  constexpr int CPL = OB ? 8 : 4;                  // columns a lane stores
  constexpr int LPR = T::WTN / CPL;                // lanes per row
  constexpr int RPI = 64 / LPR;                    // rows per store
  const int col = (lane % LPR) * CPL, row = lane / LPR;
  const int n_left = t.n_valid - wn * T::WTN - col;
  const int64_t ldb = p.ldc * (OB ? 2 : 4);
  char* base = t.C + (t.c_row + wm * T::WTM + row) * ldb + (t.b_row + wn * T::WTN + col) * (OB ? 2 : 4);
#pragma unroll
  for (int i = 0; i < T::FM; ++i) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        lds_write16(strip + (uint32_t)((lane & 31) * T::RS + (32 * j + 8 * q + 4 * h) * 4),
                    __builtin_bit_cast(u32x4, f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                                                    acc[i][j][4 * q + 3]}));
#pragma unroll
    for (int r = 0; r < 32; r += RPI) {
      const uint32_t at = strip + (uint32_t)((r + row) * T::RS + col * 4);
      char* dst = base + (int64_t)(32 * i + r) * ldb;
      const bool in = FULL || 32 * i + r + row < t.m_valid - wm * T::WTM;
      u32x4 v = lds_read16(at);
      if constexpr (OB) {
        const u32x4 w = lds_read16(at + 16);
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t a = e < 2 ? v[2 * e] : w[2 * e - 4], b = e < 2 ? v[2 * e + 1] : w[2 * e - 3];
          const bf16x2_t x = {(__bf16)__builtin_bit_cast(float, a), (__bf16)__builtin_bit_cast(float, b)};
          o[e] = __builtin_bit_cast(uint32_t, x);
        }
        v = o;
      }
      struct __attribute__((packed, aligned(OB ? 2 : 4))) Any { u32x4 v; };
      if (FULL || (in && n_left >= CPL)) {
        reinterpret_cast<Any*>(dst)->v = v;
      } else if (in) {
#pragma unroll
        for (int e = 0; e < CPL; ++e) {
          if (e < n_left) {
            if constexpr (OB) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
            else reinterpret_cast<uint32_t*>(dst)[e] = v[e];
          }
        }
      }
    }
  }
}

template <int BM, int BN, bool OB>
__device__ __forceinline__ void mx_block(const Mx4GemmParams& p, const MxTask& t, uint32_t lds0, int wave, int lane) {
  using T = MxTile<BM, BN>;
  const int wm = wave >> 1, wn = wave & 1;
  f32x16 acc[T::FM][T::FN];
#pragma unroll
  for (int i = 0; i < T::FM; ++i)
#pragma unroll
    for (int j = 0; j < T::FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int stages = (t.hi + 3) >> 2;
  // loads: lane i of a load takes row i/4 of 16 rows, and the logical chunk that lies at i%4
  const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
  int av[T::AL], bv[T::BL], sav, sbv;
#pragma unroll
  for (int i = 0; i < T::AL; ++i) {
    const int r = (wave * T::AL + i) * 16 + (lane >> 2);
    av[i] = r < t.m_valid ? (int)(r * p.lda) + 16 * chunk : kOobOffset;
  }
#pragma unroll
  for (int i = 0; i < T::BL; ++i) {
    const int r = (wave * T::BL + i) * 16 + (lane >> 2);
    bv[i] = r < t.n_valid ? (int)(r * p.ldb) + 16 * chunk : kOobOffset;
  }
  // scales: 64 rows a load; blocks of fewer than 256 rows are loaded by two waves, alike
  const int sa_seg = wave & (BM / 64 - 1), sb_seg = wave & (BN / 64 - 1);
  {
    const int ra = sa_seg * 64 + lane, rb = sb_seg * 64 + lane;
    sav = ra < t.m_valid ? (int)(ra * p.ldas) : kOobOffset;
    sbv = rb < t.n_valid ? (int)(rb * p.ldbs) : kOobOffset;
  }
  uint64_t a_at = reinterpret_cast<uint64_t>(p.A) + (uint64_t)(t.a_row * p.lda + t.block0 * 16);
  uint64_t b_at = reinterpret_cast<uint64_t>(t.B) + (uint64_t)(t.b_row * p.ldb + t.block0 * 16);
  uint64_t sa_at = reinterpret_cast<uint64_t>(p.As) + (uint64_t)(t.a_row * p.ldas + t.block0);
  uint64_t sb_at = reinterpret_cast<uint64_t>(t.Bs) + (uint64_t)(t.b_row * p.ldbs + t.block0);
  // bytes to the end of the last row's scales (whole dwords): nothing past it is read
  const int s_row_end = (t.hi + 3) & ~3;
  int sa_range = t.hi > 0 ? (int)((t.m_valid - 1) * p.ldas) + s_row_end : 0;
  int sb_range = t.hi > 0 ? (int)((t.n_valid - 1) * p.ldbs) + s_row_end : 0;
  int load_stage = 0;

  // codes of the next stage into slot `slot`, one of LOADS pieces at a time
  i32x4 ra, rb;
  int lane_in = 0;
  auto stage_begin = [&]() {
    ra = make_rsrc_addr(a_at, (uint32_t)kOobOffset);
    rb = make_rsrc_addr(b_at, (uint32_t)kOobOffset);
    const int blk = 4 * load_stage + chunk;
    lane_in = blk >= t.lo && blk < t.hi;
  };
  auto stage_piece = [&](uint32_t slot_at, int k) {
    const uint32_t at = lds0 + slot_at;
    if (k < T::AL) mx_dma16(ra, at + (uint32_t)((wave * T::AL + k) * 1024), lane_in ? av[k] : kOobOffset);
    else mx_dma16(rb, at + (uint32_t)(T::A_BYTES + (wave * T::BL + k - T::AL) * 1024),
                  lane_in ? bv[k - T::AL] : kOobOffset);
  };
  auto stage_end = [&]() {
    a_at += 64;
    b_at += 64;
    ++load_stage;
  };
  // scales of four stages into scale slot `slot`
  auto scales_load = [&](int slot) {
    const i32x4 qa = make_rsrc_addr(sa_at, sa_range > 0 ? (uint32_t)sa_range : 0u);
    const i32x4 qb = make_rsrc_addr(sb_at, sb_range > 0 ? (uint32_t)sb_range : 0u);
    const uint32_t at = lds0 + (uint32_t)(T::SA_OFF + slot * T::S_SLOT);
    mx_dma16(qa, at + (uint32_t)(sa_seg * 1024), sav);
    mx_dma16(qb, at + (uint32_t)(BM * 16 + sb_seg * 1024), sbv);
    sa_at += 16;
    sb_at += 16;
    sa_range -= 16;
    sb_range -= 16;
  };

  // fragment reads
  const int h = lane >> 5, r32 = lane & 31;
  const uint32_t frag = (uint32_t)(r32 * 64 + (((2 * h) ^ ((r32 >> 2) & 3)) << 4));
  const uint32_t a_frag = lds0 + (uint32_t)(wm * T::WTM * 64) + frag;
  const uint32_t b_frag = lds0 + (uint32_t)(T::A_BYTES + wn * T::WTN * 64) + frag;
  const uint32_t a_sc = lds0 + (uint32_t)(T::SA_OFF + (wm * T::WTM + r32) * 16 + 2 * h);
  const uint32_t b_sc = lds0 + (uint32_t)(T::SA_OFF + BM * 16 + (wn * T::WTN + r32) * 16 + 2 * h);
  i32x4 fa[2][T::FM], fb[2][T::FN];
  int sa[2][T::FM], sb[2][T::FN];
  // (step 1's chunk is step 0's ^ 1)
  auto read_frag = [&](uint32_t slot_at, int step, int k) {
    const uint32_t flip = step ? 16u : 0u;
    if (k < T::FM) fa[step][k] = *(lds_ci32x4*)(uintptr_t)((a_frag ^ flip) + slot_at + (uint32_t)(k * 2048));
    else fb[step][k - T::FM] = *(lds_ci32x4*)(uintptr_t)((b_frag ^ flip) + slot_at + (uint32_t)((k - T::FM) * 2048));
  };
  auto read_scale = [&](uint32_t off, int mask, int k) {
    if (k < T::FM) sa[1][k] = *(lds_cu16*)(uintptr_t)(a_sc + off + (uint32_t)(k * 512)) & mask;
    else sb[1][k - T::FM] = *(lds_cu16*)(uintptr_t)(b_sc + off + (uint32_t)((k - T::FM) * 512)) & mask;
  };
  // which of this lane's two scale bytes of stage st count
  auto scale_mask = [&](int st) {
    const int b0 = 4 * st + 2 * h;
    return (b0 >= t.lo && b0 < t.hi ? 0xFF : 0) | (b0 + 1 >= t.lo && b0 + 1 < t.hi ? 0xFF00 : 0);
  };
  constexpr int NF = T::FM + T::FN, NM = T::FM * T::FN;

  // prologue: stages 0 .. 3
  scales_load(0);
#pragma unroll
  for (int s = 0; s < kMxRing; ++s) {
    stage_begin();
#pragma unroll
    for (int k = 0; k < T::LOADS; ++k) stage_piece((uint32_t)(s * T::SLOT), k);
    stage_end();
  }
  wait_vmem_at_most<3 * T::LOADS>();
  __builtin_amdgcn_s_barrier();
  {
    const int mask = scale_mask(0);
#pragma unroll
    for (int k = 0; k < NF; ++k) {
      read_frag(0, 0, k);
      read_scale(0, mask, k);
    }
  }

  for (int st = 0; st < stages; ++st) {
    const uint32_t slot_at = (uint32_t)((st & 3) * T::SLOT), next_at = (uint32_t)(((st + 1) & 3) * T::SLOT);
    const uint32_t scale_at = (uint32_t)((((st + 1) >> 2) & 1) * T::S_SLOT + 4 * ((st + 1) & 3));
#pragma unroll
    for (int k = 0; k < T::FM; ++k) sa[0][k] = sa[1][k];
#pragma unroll
    for (int k = 0; k < T::FN; ++k) sb[0][k] = sb[1][k];
    // step 0, beside it the fragments of step 1
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      const int i = m / T::FN, j = m % T::FN;
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_wide(fb[0][j]), mx_wide(fa[0][i]), acc[i][j], 4, 4, 0,
                                                                  sb[0][j], 0, sa[0][i]);
      constexpr int RP = (NF + NM - 1) / NM;           // reads beside one MFMA
#pragma unroll
      for (int k = m * RP; k < (m + 1) * RP; ++k)
        if (k < NF) read_frag(slot_at, 1, k);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_lds_all();
    // younger loads: stages st+2 and st+3 (and, at times, the scales that came with one)
    wait_vmem_at_most<2 * T::LOADS>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    const int mask = scale_mask(st + 1);
    if ((st & 3) == 0) scales_load(((st >> 2) & 1) ^ 1);
    stage_begin();
    // step 1, beside it the next stage's first fragments and scales, and the loads of stage st + 4
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      const int i = m / T::FN, j = m % T::FN;
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_wide(fb[1][j]), mx_wide(fa[1][i]), acc[i][j], 4, 4, 1,
                                                                  sb[0][j], 1, sa[0][i]);
      constexpr int RP = (NF + NM - 1) / NM;
#pragma unroll
      for (int k = m * RP; k < (m + 1) * RP; ++k)
        if (k < NF) {
          read_frag(next_at, 0, k);
          read_scale(scale_at, mask, k);
        }
      constexpr int LP = (T::LOADS + NM - 1) / NM;
#pragma unroll
      for (int k = m * LP; k < (m + 1) * LP; ++k)
        if (k < T::LOADS) stage_piece(slot_at, k);
      __builtin_amdgcn_sched_barrier(0);
    }
    stage_end();
  }
  wait_vmem_at_most<0>();
  __syncthreads();                // every wave is done with the ring, and no load is in flight
  const bool full = t.m_valid == BM && t.n_valid == BN;
  if (full) mx_store<BM, BN, OB, true>(p, t, acc, lds0, wave, lane);
  else mx_store<BM, BN, OB, false>(p, t, acc, lds0, wave, lane);
  __syncthreads();                // the ring may be filled again
}

// Blocks of C in this order: curve positions (dense products, and each expert's in turn
// for kMxDepth); for kMxRows supertiles of up to 8 blocks of rows by all blocks of columns.
template <int BM, int BN, bool OB, int MODE>
__global__ __launch_bounds__(256, (MxTile<BM, BN>::PER_CU)) void mx4_gemm_kernel(Mx4GemmParams p) {
  using T = MxTile<BM, BN>;
  __shared__ __attribute__((aligned(16))) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = lds_addr(smem);
  const int P = gridDim.x, rank = xcd_rank(blockIdx.x, P);
  constexpr int ES = OB ? 2 : 4;
  MxTask t;
  t.B = p.B;
  t.Bs = p.Bs;
  t.C = reinterpret_cast<char*>(p.C);

  if constexpr (MODE == kMxRows) {
    // blocks of rows before each expert
    __shared__ int before[kMaxExperts + 1];
    __shared__ int used;             // rows up to the end of the last segment
    if (wave == 0) {
      int carry = 0, end = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const int e = e0 + lane;
        int n = 0;
        if (e < p.experts) {
          int64_t lo = p.offsets[e], hi = p.offsets[e + 1];
          lo = lo < 0 ? 0 : lo > p.M ? p.M : lo;
          hi = hi < lo ? lo : hi > p.M ? p.M : hi;
          n = (int)((hi - lo + BM - 1) / BM);
          end = hi > end ? (int)hi : end;
        }
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int up = __shfl_up(sum, d);
          sum += lane >= d ? up : 0;
        }
        if (e < p.experts) before[e] = carry + sum - n;
        carry += __shfl(sum, 63);
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const int other = __shfl_xor(end, d);
        end = other > end ? other : end;
      }
      if (lane == 0) {
        before[p.experts] = carry;
        used = end;
      }
    }
    __syncthreads();
    const int64_t total = (int64_t)before[p.experts] * p.gn;
    const int blocks = (int)(p.K >> 5);
    for (int64_t task = rank; task < total; task += P) {
      // the expert whose blocks hold this one: the last whose start is not past it
      const int mt = (int)(task / p.gn);
      int e = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const bool le = e0 + lane < p.experts && before[e0 + lane] <= mt;
        const uint64_t m = __ballot(le);
        if (m == 0) break;
        e = e0 + 63 - __clzll((long long)m);
      }
      e = __builtin_amdgcn_readfirstlane(e);
      const int first = __builtin_amdgcn_readfirstlane(before[e]);
      const int gm = __builtin_amdgcn_readfirstlane(before[e + 1]) - first;
      int64_t lo = p.offsets[e], hi = p.offsets[e + 1];
      lo = lo < 0 ? 0 : lo > p.M ? p.M : lo;
      hi = hi < lo ? lo : hi > p.M ? p.M : hi;
      const int64_t local = task - (int64_t)first * p.gn;
      const int super = (int)(local / (8 * (int64_t)p.gn));
      const int height = gm - 8 * super < 8 ? gm - 8 * super : 8;
      const int within = (int)(local - (int64_t)super * 8 * p.gn);
      const int in = within / height, im = 8 * super + within - in * height;
      t.a_row = lo + (int64_t)im * BM;
      t.c_row = t.a_row;
      t.b_row = (int64_t)in * BN;
      t.m_valid = hi - t.a_row < BM ? (int)(hi - t.a_row) : BM;
      t.n_valid = p.N - t.b_row < BN ? (int)(p.N - t.b_row) : BN;
      t.block0 = 0;
      t.lo = 0;
      t.hi = blocks;
      t.B = p.B + (int64_t)e * p.stride_b;
      t.Bs = p.Bs + (int64_t)e * p.stride_bs;
      mx_block<BM, BN, OB>(p, t, lds0, wave, lane);
    }
    // rows of no expert
    for (int64_t r = (int64_t)used + blockIdx.x; r < p.M; r += P)
      for (int64_t c = tid; c < p.N; c += 256) {
        if constexpr (OB) reinterpret_cast<uint16_t*>(p.C)[r * p.ldc + c] = 0;
        else reinterpret_cast<uint32_t*>(p.C)[r * p.ldc + c] = 0;
      }
  } else {
    const int64_t cells = (int64_t)p.gm * p.gn;
    const int groups = MODE == kMxDepth ? p.experts : p.layers;
    const int64_t total = cells * groups;
    const int blocks = (int)((p.K + 31) >> 5);
    for (int64_t task = rank; task < total; task += P) {
      const int g = (int)(task / cells);
      const int cell = load_scalar_i32(p.table + (task - (int64_t)g * cells));
      const int im = cell / p.gn, in = cell - im * p.gn;
      t.a_row = (int64_t)im * BM;
      t.b_row = (int64_t)in * BN;
      t.c_row = t.a_row;
      t.m_valid = p.M - t.a_row < BM ? (int)(p.M - t.a_row) : BM;
      t.n_valid = p.N - t.b_row < BN ? (int)(p.N - t.b_row) : BN;
      t.C = reinterpret_cast<char*>(p.C) + (int64_t)g * p.stride_c * ES;
      int64_t b0, b1;
      if constexpr (MODE == kMxDepth) {
        int64_t lo = p.offsets[g], hi = p.offsets[g + 1];
        lo = lo < 0 ? 0 : lo > p.K ? p.K : lo;
        hi = hi < lo ? lo : hi > p.K ? p.K : hi;
        b0 = lo >> 5;                    // segments start at multiples of 32
        b1 = (hi + 31) >> 5;
        if (hi == lo) b1 = b0;
      } else {
        // whole loads of scales (16 blocks) to each layer
        const int64_t units = (blocks + 15) >> 4;
        b0 = units * g / groups * 16;
        b1 = units * (g + 1) / groups * 16;
        if (b1 > blocks) b1 = blocks;
      }
      t.block0 = b0 & ~(int64_t)3;
      t.lo = (int)(b0 - t.block0);
      t.hi = (int)(b1 - t.block0);
      if (b1 == b0) t.hi = t.lo = 0;
      mx_block<BM, BN, OB>(p, t, lds0, wave, lane);
    }
  }
}

template <int BM, int BN, bool OB>
static hipError_t mx4_launch(const Mx4GemmParams& p, Mx4Mode mode, int grid, hipStream_t stream) {
  const void* k = mode == kMxDense ? reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, kMxDense>)
                  : mode == kMxRows ? reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, kMxRows>)
                                    : reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, kMxDepth>);
  Mx4GemmParams local = p;
  void* args[] = {&local};
  return hipLaunchKernel(k, dim3((unsigned)grid), dim3(256), args, 0, stream);
}

}  // namespace sfc
