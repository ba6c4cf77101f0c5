// MFMA product of microscaled 4-bit operands for gfx950, C = A B^T with both operands
// contiguous along K.
//
//   C[m][n] = sum_b 2^(sA[m][b] - 127) 2^(sB[n][b] - 127) sum_{k in block b} a[m][k] b[n][k]
//
// over blocks b of 32 values; MFMA 32x32x64 f8f6f4 takes two blocks of 4-bit elements of
// 32 rows with one scale byte per row and block, and accumulates in fp32.
//
// Mapping.  A workgroup of 4 waves (2 x 2) computes a BM x BN block.  K runs in stages of
// 256 values: 128 bytes of codes per row, one cache line (a load of half a line brings the
// whole line out of L2: with stages of 128 values the kernel drew twice its bytes and took
// 0.69 us a 128 values and CU against 0.54 with the loads left out).  LDS holds two stages.
// During stage t the rows of stage t+1 go from registers, loaded a stage ago, into the
// slot that stage t-1 left, and the same registers receive stage t+2.  A stage is four MFMA
// steps of 64 values; one barrier per stage, before its last step: by then every wave has
// read stage t and written its part of t+1.
//   * lane l of a fragment holds row l%32 and, in step s, block 4*(l/32) + s of the stage:
//     its four scale bytes are one dword, and the MFMA selects the byte by an immediate;
//   * 16-byte chunk c of row r is stored at chunk c ^ ((r >> 1) & 7): the 16 rows that a part
//     of a wave reads at one logical chunk touch the 16 16-byte bank groups;
//   * scales come straight from memory into LDS, 32 bytes of a row at a time (four stages),
//     into a ring of two slots, four stages ahead;
//   * rows past M or N and blocks outside the range of K are loaded as zeros (lanes past
//     the descriptor's range); scale bytes outside the range are masked to code 0, because
//     a NaN scale makes even zeros NaN;
//   * the MFMA takes B first, so a lane ends with one row of C and runs of 4 columns; the
//     block leaves through LDS, a wave's 32-row strips at a time, as whole row segments.
//
// Bound: the clock that power allows, times the share of it in which MFMAs run.  On random
// operands MFMAs that only read registers reach 6.3-6.5 PFLOP/s (zeros: 9.5) at 1.6 GHz, always
// busy.  Here (normal values to 4 bits, bf16 out) 8192^3 runs at 1.74 GHz with MFMAs busy in 57 % of
// the cycles and the waves waiting in 18 %, 4096x14336x4096 at 2.0 GHz, 41 % and 20 %: 3.5 rounds of
// blocks, whose stores all workgroups begin at once.  LDS conflicts are 13 % of LDS cycles.
// Several hundred calls in a row: 8192^3 261 us (4.2 PFLOP/s), 16384^3 1910 (4.6), 4096x4096x16384 130
// (4.2), 4096x14336x4096 139 (3.45; 11 less without its stores), 8192x4096x4096 80 (3.45; 9 less).  The
// first 20 calls after a rest, before the clock has settled: 309, 1960, 142, 154, 79.
// The next block's first stages loaded before the stores, and waited for past them, gained
// 0-1 %: the stores wait for the memory.  Weight gradients of 8 experts, 2048x4096, 8192 rows: fp32 88 us
// (68 without the stores of 268 MB), five stages to a block; 8672 rows, outputs in rotation, fp32 107,
// bf16 79.
#pragma once
#include "sfc_gemm_kernel.h"
#include "sfc_ops_params.h"

namespace sfc {

typedef __attribute__((address_space(3))) const i32x4 lds_ci32x4;
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;
typedef __attribute__((address_space(3))) const int lds_cint;

template <int BM, int BN>
struct MxTile {
  static constexpr int THREADS = 256;
  static constexpr int WTM = BM / 2, WTN = BN / 2;            // a wave's part
  static constexpr int FM = WTM / 32, FN = WTN / 32;          // fragments of 32 rows
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, SLOT = A_BYTES + B_BYTES;
  static constexpr int L = BM / 32;                           // loads of 8 rows per wave, operand and stage
  // scales: two slots of four stages, for every 32 rows [two stages][row][16 bytes]
  static constexpr int SA_OFF = 2 * SLOT;
  static constexpr int S_SLOT = (BM + BN) * 32;
  static constexpr int SC = (BM + BN) / 128;                  // loads of scales per wave (32 rows each)
  static constexpr int LDS = SA_OFF + 2 * S_SLOT;
  static constexpr int PER_CU = BM == 256 ? 1 : 2;            // workgroups
  // epilogue: a wave's strip of 32 rows, fp32, rows 16 bytes apart from a multiple of 256
  static constexpr int RS = WTN * 4 + 16;
  static_assert(BM == BN, "square blocks");
  static_assert(4 * 32 * RS <= SA_OFF, "strips fit the ring");
  static_assert(PER_CU * LDS <= 160 * 1024, "LDS of one CU");
};

// 16 bytes per lane from descriptor base + voffset to LDS lds + 16 * lane, zeros past the
// descriptor's range, behind the compiler's back: whoever reads them waits for them (it counts
// the other loads, which return in order).
__device__ __forceinline__ void mx_dma16(const i32x4& rsrc, uint32_t lds, uint32_t voffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(voffset), "s"(rsrc) : "memory");
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_rsrc(const uint8_t* base, uint32_t range) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)range, 0x00020000);
}
// 16 bytes at base + voffset + koffset; zeros past the descriptor's range.
__device__ __forceinline__ i32x4 mx_load16(__amdgpu_buffer_rsrc_t rsrc, int voffset, int koffset) {
  return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, voffset, koffset, 0));
}

__device__ __forceinline__ i32x8 mx_wide(const i32x4& v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}

// What a workgroup computes in one go: a block of C over a range of blocks of K.
struct MxTask {
  int64_t a_row, b_row;        // first row of A and of B
  int64_t c_row;               // first row of C (relative to C)
  int m_valid, n_valid;        // rows of A and of B inside the matrix
  int64_t block0;              // first block of K (a multiple of 8), with `lo` blocks to skip
  int lo, hi;                  // blocks lo .. hi-1 from block0 count
  const uint8_t *B, *Bs;
  char* C;
};

// PAST: past the caches (a template argument: the compiler joins a branch's stores into one).
template <int BM, int BN, bool OB, bool FULL, bool PAST>
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
      typedef u32x4 any_u32x4 __attribute__((aligned(2)));
      if (FULL || (in && n_left >= CPL)) {
        if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<any_u32x4*>(dst));
        else *reinterpret_cast<any_u32x4*>(dst) = v;
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

template <int BM, int BN, bool OB, bool PAST>
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

  constexpr int L = T::L, NF = T::FM + T::FN, NM = T::FM * T::FN;
  const int stages = (t.hi + 7) >> 3;
  // Loads: lane i of a load takes row i/8 of 8 rows, chunk i%8; wave w the rows w*BM/4 ..
  const int chunk = lane & 7;
  int av[L], bv[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int r = (wave * L + i) * 8 + (lane >> 3);
    av[i] = r < t.m_valid ? (int)(r * p.lda) + 16 * chunk : kOobOffset;
    bv[i] = r < t.n_valid ? (int)(r * p.ldb) + 16 * chunk : kOobOffset;
  }
  const __amdgpu_buffer_rsrc_t qa = mx_rsrc(p.A + t.a_row * p.lda + t.block0 * 16, kOobOffset);
  const __amdgpu_buffer_rsrc_t qb = mx_rsrc(t.B + t.b_row * p.ldb + t.block0 * 16, kOobOffset);
  // stages from here on hold blocks past the range: the lanes that would load them turn into
  // lanes that read zeros, for good
  const int full_stages = t.hi >> 3;
  auto cut_lanes = [&](int stage) {
    const bool out = 8 * stage + chunk >= t.hi;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      av[i] = out ? kOobOffset : av[i];
      bv[i] = out ? kOobOffset : bv[i];
    }
  };
  // Scales: a load takes 32 bytes of 32 rows (of A's, then B's).  They end with the last
  // row's (whole dwords): nothing past it is read, whatever comes of the last loads, which run
  // ahead of the range (so all of their offset is in the lane's, which the range is checked against).
  const int s_row_end = (t.hi + 3) & ~3;
  const i32x4 qas = make_rsrc_addr(reinterpret_cast<uint64_t>(p.As) + (uint64_t)(t.a_row * p.ldas + t.block0),
                                   t.hi > 0 ? (uint32_t)((t.m_valid - 1) * p.ldas + s_row_end) : 0u);
  const i32x4 qbs = make_rsrc_addr(reinterpret_cast<uint64_t>(t.Bs) + (uint64_t)(t.b_row * p.ldbs + t.block0),
                                   t.hi > 0 ? (uint32_t)((t.n_valid - 1) * p.ldbs + s_row_end) : 0u);
  uint32_t sv[T::SC];                          // of the next group of four stages
#pragma unroll
  for (int k = 0; k < T::SC; ++k) {
    const bool of_a = (wave * T::SC + k) * 32 < BM;
    const int r = (wave * T::SC + k) * 32 - (of_a ? 0 : BM) + (lane & 31);
    sv[k] = r < (of_a ? t.m_valid : t.n_valid) ? (uint32_t)(r * (of_a ? p.ldas : p.ldbs)) + 16 * (lane >> 5) : (uint32_t)kOobOffset;
  }
  auto load_scales = [&](int group) {        // four stages of scales, number `group` (one after another), into their slot
    const uint32_t at = lds0 + (uint32_t)(T::SA_OFF + (group & 1) * T::S_SLOT + wave * T::SC * 1024);
#pragma unroll
    for (int k = 0; k < T::SC; ++k) {
      const bool of_a = (wave * T::SC + k) * 32 < BM;
      mx_dma16(of_a ? qas : qbs, at + (uint32_t)(k * 1024), sv[k]);
      sv[k] += 32;
    }
  };

  // LDS addresses: writes of even loads (odd ones: ^ 64) and fragment reads of step 0 (step s: ^ 16 s)
  const uint32_t w0 = lds0 + (uint32_t)(wave * L * 1024 + (lane >> 3) * 128 + ((chunk ^ (lane >> 4)) << 4));
  const int h = lane >> 5, r32 = lane & 31;
  const uint32_t frag = (uint32_t)(r32 * 128 + (((4 * h) ^ ((r32 >> 1) & 7)) << 4));
  const uint32_t a_frag = lds0 + (uint32_t)(wm * T::WTM * 128) + frag, b_frag = lds0 + (uint32_t)(wn * T::WTN * 128) + frag;
  const uint32_t a_sc = lds0 + (uint32_t)(T::SA_OFF + wm * T::WTM * 32 + r32 * 16 + 4 * h);
  const uint32_t b_sc = lds0 + (uint32_t)(T::SA_OFF + (BM + wn * T::WTN) * 32 + r32 * 16 + 4 * h);
  i32x4 ga[L], gb[L];
  i32x4 fa[2][T::FM], fb[2][T::FN];
  int sa[2][T::FM], sb[2][T::FN];              // the stage's scales, and the next one's
  auto write_rows = [&](uint32_t slot, int k) {      // load k of 2 L: A's, then B's
    const uint32_t at = ((k & 1) ? w0 ^ 64u : w0) + slot + (uint32_t)((k < L ? k : k - L) * 1024);
    if (k < L) *(lds_i32x4*)(uintptr_t)at = ga[k];
    else *(lds_i32x4*)(uintptr_t)(at + T::A_BYTES) = gb[k - L];
  };
  auto load_rows = [&](int koff, int k) {
    if (k < L) ga[k] = mx_load16(qa, av[k], koff);
    else gb[k - L] = mx_load16(qb, bv[k - L], koff);
  };
  auto read_frag = [&](uint32_t slot, int step, int set, int k) {
    if (k < T::FM) fa[set][k] = *(lds_ci32x4*)(uintptr_t)((a_frag ^ (uint32_t)(16 * step)) + slot + (uint32_t)(k * 4096));
    else fb[set][k - T::FM] = *(lds_ci32x4*)(uintptr_t)((b_frag ^ (uint32_t)(16 * step)) + slot +
                                                        (uint32_t)(T::A_BYTES + (k - T::FM) * 4096));
  };
  auto read_scale = [&](uint32_t off, int k) {
    if (k < T::FM) sa[1][k] = *(lds_cint*)(uintptr_t)(a_sc + off + (uint32_t)(k * 1024));
    else sb[1][k - T::FM] = *(lds_cint*)(uintptr_t)(b_sc + off + (uint32_t)((k - T::FM) * 1024));
  };
  // stages that hold blocks outside the range: their scale bytes there become 0
  const int first_cut = t.lo > 0 ? 0 : -1, last_cut = (t.hi & 7) ? stages - 1 : -1;
  auto cut_scales = [&](int st) {
    int mask = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int b = 8 * st + 4 * h + k;
      mask |= b >= t.lo && b < t.hi ? 0xFF << (8 * k) : 0;
    }
#pragma unroll
    for (int k = 0; k < T::FM; ++k) sa[1][k] &= mask;
#pragma unroll
    for (int k = 0; k < T::FN; ++k) sb[1][k] &= mask;
  };

  // prologue: stage 0 and its scales into LDS, stage 1 into registers
  load_scales(0);
  if (0 >= full_stages) cut_lanes(0);
  {
    const bool in = chunk >= t.lo;
#pragma unroll
    for (int k = 0; k < L; ++k) ga[k] = mx_load16(qa, in ? av[k] : kOobOffset, 0);
#pragma unroll
    for (int k = 0; k < L; ++k) gb[k] = mx_load16(qb, in ? bv[k] : kOobOffset, 0);
  }
  if (1 >= full_stages) cut_lanes(1);
#pragma unroll
  for (int k = 0; k < 2 * L; ++k) {
    write_rows(0, k);
    load_rows(128, k);
  }
  wait_vmem_at_most<2 * L>();                  // the scales
  wait_lds_all();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int k = 0; k < NF; ++k) {
    read_frag(0, 0, 0, k);
    read_scale(0, k);
  }

  // What goes beside which MFMA: fragment reads on the first MFMAs of a step, the 2 L moves of rows
  // (into LDS, and the next load into the same registers) evenly over steps 0 .. 2.
  constexpr auto read_at = [](int k) { return NM >= 16 ? k + k / 2 : k * NM / NF; };
  constexpr auto move_at = [](int k) { return (k * 3 * NM) / (2 * L) + (NM >= 16 ? 2 : 0); };
  uint32_t slot = 0;                           // LDS offset of the stage's slot
  for (int st = 0; st < stages; ++st) {
    uint32_t next = (uint32_t)T::SLOT - slot;
    pin_scalar(next);                          // (one value: the LDS offsets stay in the instructions)
    const int koff = 128 * (st + 2);
    const uint32_t scale_at = (uint32_t)((((st + 1) >> 2) & 1) * T::S_SLOT + (((st + 1) >> 1) & 1) * 512 + 8 * ((st + 1) & 1));
    // (no branch between the steps: the compiler would move MFMAs down past it)
    if (st == first_cut || st == last_cut) cut_scales(st);
    if (st + 2 >= full_stages) cut_lanes(st + 2);
    // (their slot's last reader was stage st - 2)
    if ((st & 3) == 0) load_scales((st >> 2) + 1);
    sb[0][0] = sb[1][0];
    sa[0][0] = sa[1][0];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        // (back and forth over j, so that one operand at least stays from MFMA to MFMA: 0.5-1 % less
        // time, which is power here)
        const int i = m / T::FN, j = (i & 1) ? T::FN - 1 - m % T::FN : m % T::FN;
        const i32x8 xb = mx_wide(fb[s & 1][j]), xa = mx_wide(fa[s & 1][i]);
        if (s == 0) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xb, xa, acc[i][j], 4, 4, 0, sb[0][j], 0, sa[0][i]);
        if (s == 1) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xb, xa, acc[i][j], 4, 4, 1, sb[0][j], 1, sa[0][i]);
        if (s == 2) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xb, xa, acc[i][j], 4, 4, 2, sb[0][j], 2, sa[0][i]);
        if (s == 3) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xb, xa, acc[i][j], 4, 4, 3, sb[0][j], 3, sa[0][i]);
        if (s == 0) {
          if (m + 1 < T::FN) sb[0][m + 1] = sb[1][m + 1];
          if ((m + 1) % T::FN == 0 && m + 1 < NM) sa[0][(m + 1) / T::FN] = sa[1][(m + 1) / T::FN];
        }
#pragma unroll
        for (int k = 0; k < NF; ++k)
          if (read_at(k) == m) {
            if (s < 3) {
              read_frag(slot, s + 1, (s + 1) & 1, k);
            } else {
              read_frag(next, 0, 0, k);
              read_scale(scale_at, k);
            }
          }
#pragma unroll
        for (int k = 0; k < 2 * L; ++k)
          if (move_at(k) == s * NM + m) {
            write_rows(next, k);
            load_rows(koff, k);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (s == 2) {
        // this stage's 2 L loads are younger than all scales
        wait_vmem_at_most<2 * L>();
        wait_lds_all();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    slot = next;
  }
  __syncthreads();                // every wave is done with the ring
  const bool full = t.m_valid == BM && t.n_valid == BN;
  if (full) mx_store<BM, BN, OB, true, PAST>(p, t, acc, lds0, wave, lane);
  else mx_store<BM, BN, OB, false, PAST>(p, t, acc, lds0, wave, lane);
  __syncthreads();                // the ring may be filled again
}

// Blocks of C in this order: curve positions (dense products, and each expert's in turn
// for kMxDepth); for kMxRows supertiles of up to 8 blocks of rows by all blocks of columns.
template <int BM, int BN, bool OB, bool PAST, int MODE>
__global__ __launch_bounds__(256, (MxTile<BM, BN>::PER_CU)) void mx4_gemm_kernel(Mx4GemmParams p) {
  using T = MxTile<BM, BN>;
  __shared__ __attribute__((aligned(16))) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = lds_addr(smem);
  const int P = gridDim.x, rank = xcd_rank(blockIdx.x, P);
  // Tasks of this workgroup: its rank of every full round, and in the last, partial one its
  // rank among as many workgroups as there are tasks left.  Those are the first, which spreads them
  // over all chiplets, and one to a CU where two fit (by full ranks they would fill some
  // chiplets and leave the others idle).
  auto next_task = [&](int64_t task, int64_t total) {
    const int64_t from = task < 0 ? 0 : (task / P + 1) * P;       // the round's first task
    if (from + P <= total) return from + rank;
    const int left = (int)(total - from);
    return (int)blockIdx.x < left ? from + xcd_rank(blockIdx.x, left) : (int64_t)-1;
  };
  constexpr int ES = OB ? 2 : 4;
  MxTask t;
  t.B = p.B;
  t.Bs = p.Bs;
  t.C = reinterpret_cast<char*>(p.C);

  if constexpr (MODE == kMxRows) {
    // rows lo .. hi-1 of expert e
    auto segment = [&](int e, int64_t& lo, int64_t& hi) {
      lo = p.offsets[e];
      hi = p.offsets[e + 1];
      lo = lo < 0 ? 0 : lo > p.M ? p.M : lo;
      hi = hi < lo ? lo : hi > p.M ? p.M : hi;
    };
    // the expert that holds block of rows `mt` (counted over all experts; there is one), the
    // blocks before it and its own
    auto find = [&](int mt, int& first, int& gm) {
      int carry = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 64) {
        int n = 0;
        if (e0 + lane < p.experts) {
          int64_t lo, hi;
          segment(e0 + lane, lo, hi);
          n = (int)((hi - lo + BM - 1) / BM);
        }
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int up = __shfl_up(sum, d);
          sum += lane >= d ? up : 0;
        }
        const uint64_t past = __ballot(carry + sum > mt);
        if (past) {
          const int l = __ffsll((unsigned long long)past) - 1;
          gm = __builtin_amdgcn_readfirstlane(__shfl(n, l));
          first = __builtin_amdgcn_readfirstlane(carry + __shfl(sum, l)) - gm;
          return e0 + l;
        }
        carry += __builtin_amdgcn_readfirstlane(__shfl(sum, 63));
      }
      return -1;
    };
    const int blocks = (int)(p.K >> 5);
    int blocks_of_rows = 0, used = 0;        // of all experts; rows up to the end of the last segment
    for (int e = lane; e < p.experts; e += 64) {
      int64_t lo, hi;
      segment(e, lo, hi);
      blocks_of_rows += (int)((hi - lo + BM - 1) / BM);
      used = hi > used ? (int)hi : used;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const int other = __shfl_xor(used, d);
      used = other > used ? other : used;
      blocks_of_rows += __shfl_xor(blocks_of_rows, d);
    }
    const int64_t total = (int64_t)__builtin_amdgcn_readfirstlane(blocks_of_rows) * p.gn;
    for (int64_t task = next_task(-1, total); task >= 0; task = next_task(task, total)) {
      int first = 0, gm = 0;
      const int e = __builtin_amdgcn_readfirstlane(find((int)(task / p.gn), first, gm));
      int64_t lo, hi;
      segment(e, lo, hi);
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
      mx_block<BM, BN, OB, PAST>(p, t, lds0, wave, lane);
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
    for (int64_t task = next_task(-1, total); task >= 0; task = next_task(task, total)) {
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
      t.block0 = b0 & ~(int64_t)7;     // whole 128-byte lines of codes
      t.lo = (int)(b0 - t.block0);
      t.hi = (int)(b1 - t.block0);
      if (b1 == b0) t.hi = t.lo = 0;
      mx_block<BM, BN, OB, PAST>(p, t, lds0, wave, lane);
    }
  }
}

template <int BM, int BN, bool OB, bool PAST>
static const void* mx4_kernel(Mx4Mode mode) {
  return mode == kMxDense  ? reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, PAST, kMxDense>)
         : mode == kMxRows ? reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, PAST, kMxRows>)
                           : reinterpret_cast<const void*>(&mx4_gemm_kernel<BM, BN, OB, PAST, kMxDepth>);
}

template <int BM, int BN>
static hipError_t mx4_launch(const Mx4GemmParams& p, Mx4Mode mode, bool out_bf16, int grid, hipStream_t stream) {
  const void* k = out_bf16 ? (p.past ? mx4_kernel<BM, BN, true, true>(mode) : mx4_kernel<BM, BN, true, false>(mode))
                           : (p.past ? mx4_kernel<BM, BN, false, true>(mode) : mx4_kernel<BM, BN, false, false>(mode));
  Mx4GemmParams local = p;
  void* args[] = {&local};
  return hipLaunchKernel(k, dim3((unsigned)grid), dim3(256), args, 0, stream);
}

}  // namespace sfc
