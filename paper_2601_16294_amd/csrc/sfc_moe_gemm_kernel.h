// MFMA products of bf16 rows that are grouped by expert, for gfx950:
//
//   kMoeNK   C[p] = A[r(p)] B[e]^T       B[e] is N x K, as a linear layer holds its weights
//   kMoeKN   C[p] = A[r(p)] B[e]         B[e] is K x N: the gradient of A, with the same weights
//   kMoeTN   C[e] = A[seg]^T B[seg]      the gradient of the weights, over the expert's rows
//
// for the rows p of every expert e, fp32 sums, fp32 or bf16 out; r(p) is p, or the row that a sort
// order names (rows of no slot are zeros).
//
// Mapping.  A workgroup of 4 waves (2 x 2) computes a BM x BN block.  K runs in stages of 64;
// an operand's part of a stage, 128 bytes for each of its rows or columns, is a unit of a ring of
// five units in LDS (A and B of a stage in turn), filled straight from memory: the whole of one
// stage, and of the next stage but one A's half, are on their way while a stage is
// computed.  A stage is two MFMA steps of 32; one barrier per stage, between its steps: by then every
// wave has read the stage, and its two units take the loads that come next.
//   * an operand along K is kept [row][64], 16-byte chunk c of row r at chunk c ^ ((r >> 1) & 7), and
//     read 16 bytes a lane; one along M or N is kept [64][columns], chunk c of row k at chunk
//     c ^ moe_swz(k), and read by the transposing LDS load.  Both swizzles keep the banks apart;
//   * rows past the segment and K past its end are loaded as zeros (lanes past the
//     descriptor's range).  A chunk that the end of a row cuts is left out of the loads of the last
//     stage and written to LDS element by element, so nothing outside the matrices is used, nor read
//     where no row follows;
//   * the MFMA takes B first, so a lane ends with one row of C and runs of 4 columns; the block
//     leaves through LDS, a wave's 16-row strips at a time, as whole row segments.
//
// Bound: the MFMAs' rate, for segments long enough to fill blocks.  One segment of 8192^3, normal values: 1390 to 1425
// TFLOP/s for kMoeNK and kMoeKN, 1330 for kMoeTN, with the MFMAs busy in 63, 60 and 58 % of the cycles at 2.16 GHz, no
// bank conflicts, waves waiting in a fifth of the cycles (other places of the barrier and of the loads: within 1.5 %).
// Stores take 5 to 6 % of a product, up to a fifth of a weight gradient in fp32.  4096 tokens, 2 of 8 experts
// 14336x4096: 845 us = 1139 TFLOP/s, 12 % more with the empty rows of last blocks.  256x256 blocks of kMoeNK and kMoeKN spill 2
// to 9 registers, outside of the stages' loop, where one reload waits for the loads in flight, once a block.  256x256 blocks read each
// operand least often; 128x128 and 64x64, two and four workgroups to a CU, fill the chip where there are few rows or
// columns: moe_tile_us() of the host layer estimates which takes least.
#pragma once
#include "sfc_gemm_kernel.h"
#include "sfc_moe_params.h"
#include "sfc_segments.h"

namespace sfc {

constexpr uint32_t kMoeRange = 0xFFFFFF00u;       // descriptors' range: byte offsets below it are loaded
constexpr uint32_t kMoeOut = 0xFFFFFFF0u;         // a lane that loads zeros

// Chunk c of row k of an operand along M or N lies at chunk c ^ moe_swz(k) (rows of 8 chunks at least).
template <int BX>
__device__ __forceinline__ int moe_swz(int k) { return b_swz(k) & (BX / 8 - 1); }

template <int BM, int BN>
struct MoeTile {
  static constexpr int WTM = BM / 2, WTN = BN / 2;           // a wave's part
  static constexpr int FM = WTM / 16, FN = WTN / 16;         // 16x16 fragments
  static constexpr int UNIT = BM * 128;                      // bytes of an operand's stage
  static constexpr int L = BM / 32;                          // loads of 1 KiB per wave and unit
  static constexpr int LDS = 5 * UNIT;
  static constexpr int PER_CU = BM == 256 ? 1 : BM == 128 ? 2 : 4;
  // epilogue: a wave's strip of 16 rows, fp32, rows 16 bytes apart from a multiple of 256
  static constexpr int RS = WTN * 4 + 16;
  static_assert(BM == BN, "square blocks");
  static_assert(4 * 16 * RS <= LDS, "strips fit the ring");
  static_assert(PER_CU * LDS <= 160 * 1024, "LDS of one CU");
};

// f(0), .., f(N - 1) with constant arguments.
template <int N, class F>
__device__ __forceinline__ void each(F f) {
  [&]<int... I>(std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
  }(std::make_integer_sequence<int, N>{});
}
// Items 0 .. n-1 of a step stand beside MFMAs at(0) <= at(1) <= ..: how many stand before MFMA m.
template <class F>
constexpr int items_before(int m, int n, F at) {
  int k = 0;
  while (k < n && at(k) < m) ++k;
  return k;
}

// One operand of a block.  ALONG_K: rows along K; else rows are K and their columns the block's.
struct MoeOperand {
  uint64_t base;             // address of the block's first element in stage 0
  int64_t ld;                // elements
  int valid;                 // rows (ALONG_K) or columns of the block inside the matrix
  // rows taken through a sort order: of the block's first row (null: as they lie)
  const int32_t* order;
  int64_t rows;
  int topk;
};
struct MoeTask {
  MoeOperand a, b;
  int64_t depth;             // K
  char* C;                   // the block's first element
};

// Row of A behind a sorted row, or -1.
__device__ __forceinline__ int64_t moe_source(const MoeOperand& o, int r) {
  const int s = o.order[r];
  const int64_t row = s < 0 ? -1 : s / o.topk;
  return row < o.rows ? row : -1;
}

template <int BX, bool ALONG_K, bool GATHER>
struct MoeLoads {
  static constexpr int L = BX / 32;
  static constexpr int UNIT = BX * 128;
  uint32_t at[L];            // byte offsets of this lane's chunks
  uint64_t base;
  uint64_t step;             // bytes from one stage to the next

  // index (in 16-byte chunks) of load j along K (ALONG_K) or along the columns, and its row
  static __device__ __forceinline__ void place(int wave, int lane, int j, int& row, int& chunk) {
    if constexpr (ALONG_K) {
      row = (wave * L + j) * 8 + (lane >> 3);
      chunk = (lane & 7) ^ ((row >> 1) & 7);
    } else {
      const int e = (wave * L + j) * 512 + lane * 8;
      row = e / BX;
      chunk = ((e % BX) >> 3) ^ moe_swz<BX>(row);
    }
  }

  __device__ __forceinline__ void init(const MoeOperand& o, int wave, int lane) {
    base = o.base;
    step = ALONG_K ? 128 : (uint64_t)o.ld * 128;
#pragma unroll
    for (int j = 0; j < L; ++j) {
      int row, chunk;
      place(wave, lane, j, row, chunk);
      if constexpr (ALONG_K && GATHER) {
        const int64_t source = row < o.valid ? moe_source(o, row) : -1;
        at[j] = source >= 0 ? (uint32_t)((uint64_t)source * (uint64_t)o.ld * 2 + 16 * chunk) : kMoeOut;
      } else if constexpr (ALONG_K) {
        at[j] = row < o.valid ? (uint32_t)(row * (int)o.ld * 2 + 16 * chunk) : kMoeOut;
      } else {
        at[j] = 8 * chunk < o.valid ? (uint32_t)(row * (int)o.ld * 2 + 16 * chunk) : kMoeOut;
      }
    }
  }

  // From the stage on that has `left` of K left: lanes outside of it, and lanes whose chunk the end of
  // a row cuts, load zeros.
  __device__ __forceinline__ void cut(const MoeOperand& o, int left, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < L; ++j) {
      int row, chunk;
      place(wave, lane, j, row, chunk);
      const bool in = ALONG_K ? 8 * chunk + 8 <= left : row < left && 8 * chunk + 8 <= o.valid;
      at[j] = in ? at[j] : kMoeOut;
    }
  }

  __device__ __forceinline__ void load(uint32_t unit, int wave, int j) const {
    const i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
                        __builtin_amdgcn_readfirstlane((int)((uint32_t)(base >> 32) & 0xFFFFu)), (int)kMoeRange, 0x00020000};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(unit + (uint32_t)((wave * L + j) * 1024)), "v"(at[j]), "s"(rsrc) : "memory");
  }

  // Chunks of the stage that the end of a row cuts: their elements inside, zeros behind.  `left` of K
  // are left; `stage_base` is the stage's base.
  static __device__ __forceinline__ void patch(const MoeOperand& o, uint64_t stage_base, int left, uint32_t unit, int tid) {
    const int c = ALONG_K ? left >> 3 : o.valid >> 3, n = (ALONG_K ? left : o.valid) & 7;
    if (n == 0 || tid >= (ALONG_K ? o.valid : left)) return;
    int64_t row = tid;
    if constexpr (ALONG_K && GATHER) row = moe_source(o, tid);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (row >= 0) {
      typedef const __attribute__((address_space(1))) uint16_t global_u16;
      global_u16* p = (global_u16*)(stage_base + (uint64_t)(row * o.ld + 8 * c) * 2);
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    }
    const uint32_t at = ALONG_K ? (uint32_t)(tid * 128 + ((c ^ ((tid >> 1) & 7)) << 4))
                                : (uint32_t)(tid * BX * 2 + ((c ^ moe_swz<BX>(tid)) << 4));
    lds_write16(unit + at, u32x4{w[0], w[1], w[2], w[3]});
  }
};

// Fragment reads of an operand: 16 rows (columns) x 32 of K.
template <int BX, bool ALONG_K>
struct MoeReads {
  static constexpr int PARTS = ALONG_K ? 1 : 2;              // LDS loads of a fragment
  uint32_t at;                                               // of fragment 0, step 0 (byte offset in the unit)
  __device__ __forceinline__ void init(int first, int lane) {
    if constexpr (ALONG_K) {
      at = (uint32_t)(2 * a_frag_off(first, lane, 0));
    } else {
      // lane (g = l / 16, j = l % 16) points at row 8 g + j / 4 and 4 columns; it gets column j of 4 rows
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2), n = first + 4 * (lane & 3);
      at = (uint32_t)(2 * (k * BX + (((n >> 3) ^ moe_swz<BX>(k)) << 3) + (n & 7)));
    }
  }
  __device__ __forceinline__ void read(uint32_t unit, int step, int i, int part, bf16x8& f) const {
    if constexpr (ALONG_K) {
      f = *(lds_bf16x8*)(uintptr_t)(unit + (at ^ (uint32_t)(64 * step)) + (uint32_t)(i * 2048));
    } else {
      const uint32_t p = unit + (at ^ (uint32_t)(32 * i)) + (uint32_t)(step * 64 * BX + part * 8 * BX);
      const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)p);
      i16x8 w = __builtin_bit_cast(i16x8, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * part + e] = v[e];
      f = __builtin_bit_cast(bf16x8, w);
    }
  }
};

// PAST: past the caches (a template argument: the compiler joins a branch's stores into one).
template <int BM, int BN, bool OB, bool FULL, bool PAST>
__device__ __forceinline__ void moe_store(const MoeGemmParams& p, const MoeTask& t, int m_valid, int n_valid,
                                          f32x4 (&acc)[BM / 32][BN / 32], uint32_t lds0, int wave, int lane) {
  using T = MoeTile<BM, BN>;
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t strip = lds0 + (uint32_t)(wave * 16 * T::RS);
  constexpr int CPL = OB ? 8 : 4;                  // columns a lane stores
  constexpr int LPR = T::WTN / CPL;                // lanes per row
  constexpr int RPI = 64 / LPR;                    // rows per store
  const int col = (lane % LPR) * CPL, row = lane / LPR;
  const int n_left = n_valid - wn * T::WTN - col;
  const int64_t ldb = p.ldc * (OB ? 2 : 4);
  char* base = t.C + (int64_t)(wm * T::WTM + row) * ldb + (wn * T::WTN + col) * (OB ? 2 : 4);
#pragma unroll
  for (int i = 0; i < T::FM; ++i) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j)
      lds_write16(strip + (uint32_t)((lane & 15) * T::RS + (16 * j + 4 * (lane >> 4)) * 4),
                  __builtin_bit_cast(u32x4, acc[i][j]));
#pragma unroll
    for (int r = 0; r < 16; r += RPI) {
      const uint32_t at = strip + (uint32_t)((r + row) * T::RS + col * 4);
      char* dst = base + (int64_t)(16 * i + r) * ldb;
      const bool in = FULL || 16 * i + r + row < m_valid - wm * T::WTM;
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

// acc = the block's sums; every wave is done with the ring when it returns.
template <int BM, int BN, MoeLayout LAYOUT, bool GATHER>
__device__ __forceinline__ void moe_accumulate(const MoeTask& t, uint32_t lds0, int wave, int lane, f32x4 (&acc)[BM / 32][BN / 32]) {
  using T = MoeTile<BM, BN>;
  constexpr bool AK = LAYOUT != kMoeTN, BK = LAYOUT == kMoeNK;
  constexpr int L = T::L, FM = T::FM, FN = T::FN, NM = FM * FN;
  using LA = MoeLoads<BM, AK, GATHER>;
  using LB = MoeLoads<BN, BK, false>;
  const int wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;

  const int stages = (int)((t.depth + 63) >> 6);
  const int tail = (int)(t.depth - 64 * (int64_t)(stages - 1));       // of K in the last stage
  // the last stage of A or B has lanes to cut, or chunks to write by elements
  const bool patch = (AK || BK ? (tail & 7) != 0 : false) || (!AK && (t.a.valid & 7)) || (!BK && (t.b.valid & 7));
  // (rows of fewer than 8 elements: a chunk reaches past the next row too, so every stage is patched)
  const bool every = (!AK && t.a.ld < 8) || (!BK && t.b.ld < 8);
  const int whole = every ? 0 : patch || tail < 64 ? stages - 1 : stages;    // stages before the first to cut
  LA la;
  LB lb;
  la.init(t.a, wave, lane);
  lb.init(t.b, wave, lane);
  MoeReads<BM, AK> ra;
  MoeReads<BN, BK> rb;
  ra.init(wm * T::WTM, lane);
  rb.init(wn * T::WTN, lane);
  bf16x8 fa[2][FM], fb[2][FN];
  const int tid = wave * 64 + lane;

  // the loads of A's and of B's next stage begin
  int a_stage = 0, b_stage = 0;
  uint32_t a_unit = lds0, b_unit = lds0 + (uint32_t)T::UNIT;          // where they go
  const uint32_t ring_end = lds0 + (uint32_t)T::LDS;
  auto two_on = [&](uint32_t unit) {
    const uint32_t next = unit + (uint32_t)(2 * T::UNIT);
    return next >= ring_end ? next - (uint32_t)T::LDS : next;
  };
  auto left_at = [&](int stage) {              // of K, from a stage on, up to 64
    const int64_t left = t.depth - 64 * (int64_t)stage;
    return left < 0 ? 0 : left > 64 ? 64 : (int)left;
  };
  auto a_begin = [&]() {
    if (a_stage >= whole) la.cut(t.a, left_at(a_stage), wave, lane);
  };
  auto a_end = [&]() {
    la.base += la.step;
    ++a_stage;
    a_unit = two_on(a_unit);
  };
  auto b_begin = [&]() {
    if (b_stage >= whole) lb.cut(t.b, left_at(b_stage), wave, lane);
  };
  auto b_end = [&]() {
    lb.base += lb.step;
    ++b_stage;
    b_unit = two_on(b_unit);
  };
  // chunks of a stage in LDS that the end of a row cuts (every wave has its loads)
  auto patch_stage = [&](int stage, uint32_t una, uint32_t unb) {
    if (!patch || stage >= stages || (stage + 1 < stages && !every)) return;
    LA::patch(t.a, t.a.base + (uint64_t)stage * la.step, left_at(stage), una, tid);
    LB::patch(t.b, t.b.base + (uint64_t)stage * lb.step, left_at(stage), unb, tid);
    wait_lds_all();
    __builtin_amdgcn_s_barrier();
  };

  // prologue: A and B of stages 0 and 1, A of stage 2
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    a_begin();
#pragma unroll
    for (int j = 0; j < L; ++j) la.load(a_unit, wave, j);
    a_end();
    if (s < 2) {
      b_begin();
#pragma unroll
      for (int j = 0; j < L; ++j) lb.load(b_unit, wave, j);
      b_end();
    }
  }
  uint32_t ua = lds0, ub = lds0 + (uint32_t)T::UNIT;                  // the stage's units
  wait_vmem_at_most<3 * L>();
  __builtin_amdgcn_s_barrier();
  patch_stage(0, ua, ub);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int q = 0; q < MoeReads<BM, AK>::PARTS; ++q) ra.read(ua, 0, i, q, fa[0][i]);
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int q = 0; q < MoeReads<BN, BK>::PARTS; ++q) rb.read(ub, 0, j, q, fb[0][j]);

  // What goes beside which MFMA of a step.  Fragment reads of the next step, in the order its MFMAs
  // take them (A0, all of B, the rest of A), over its first MFMAs; B's loads at the start of step 1,
  // A's over the rest of it and the next step 0.
  constexpr int PA = MoeReads<BM, AK>::PARTS, PB = MoeReads<BN, BK>::PARTS, NR = FM * PA + FN * PB;
  constexpr auto read_at = [](int k) { return k * (NM - NM / 8) / NR; };
  constexpr auto b_load_at = [](int k) { return 1 + k * (NM / 2) / L; };
  constexpr auto a_load_at = [](int k) { return NM / 2 + 2 + k * (NM - 4) / L; };    // NM and on: in the next step 0
  auto step = [&](auto second, uint32_t una, uint32_t unb, bool load) {
    constexpr int set = second, next = 1 - set;          // fragments used; step (and set) that is read
    each<NM>([&](auto mc) {
      constexpr int m = mc, i = m / FN, j = (i & 1) ? FN - 1 - m % FN : m % FN;
      // (back and forth over j, so that one operand at least stays from MFMA to MFMA)
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][j], fa[set][i], acc[i][j], 0, 0, 0);
      constexpr int r0 = items_before(m, NR, read_at), r1 = items_before(m + 1, NR, read_at);
      each<r1 - r0>([&](auto kc) {
        constexpr int k = r0 + kc;
        if constexpr (k < PA) ra.read(una, next, 0, k, fa[next][0]);
        else if constexpr (k < PA + FN * PB) rb.read(unb, next, (k - PA) / PB, (k - PA) % PB, fb[next][(k - PA) / PB]);
        else ra.read(una, next, 1 + (k - PA - FN * PB) / PA, (k - PA - FN * PB) % PA, fa[next][1 + (k - PA - FN * PB) / PA]);
      });
      if constexpr (set == 1) {
        constexpr int b0 = items_before(m, L, b_load_at), b1 = items_before(m + 1, L, b_load_at);
        each<b1 - b0>([&](auto kc) { lb.load(b_unit, wave, b0 + kc); });
      }
      constexpr int at = set == 1 ? m : NM + m;
      constexpr int a0 = items_before(at, L, a_load_at), a1 = items_before(at + 1, L, a_load_at);
      if constexpr (a1 > a0) {
        if (load) each<a1 - a0>([&](auto kc) { la.load(a_unit, wave, a0 + kc); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  for (int st = 0; st < stages; ++st) {
    const uint32_t na = two_on(ua), nb = two_on(ub);
    step(std::integral_constant<int, 0>{}, ua, ub, st > 0);
    if (st > 0) a_end();
    // A of stage st + 2 may still be under way
    wait_vmem_at_most<L>();
    wait_lds_all();
    __builtin_amdgcn_s_barrier();
    patch_stage(st + 1, na, nb);
    __builtin_amdgcn_sched_barrier(0);
    a_begin();
    b_begin();
    step(std::integral_constant<int, 1>{}, na, nb, true);
    b_end();
    ua = na;
    ub = nb;
  }
  // (loads of stages past the end write zeros to the ring)
  wait_vmem_at_most<0>();
  __syncthreads();                // every wave is done with the ring
}

template <int BM, int BN, MoeLayout LAYOUT, bool GATHER, bool OB, bool PAST>
__device__ __forceinline__ void moe_block(const MoeGemmParams& p, const MoeTask& t, uint32_t lds0, int wave, int lane) {
  f32x4 acc[BM / 32][BN / 32];
  moe_accumulate<BM, BN, LAYOUT, GATHER>(t, lds0, wave, lane, acc);
  const int mv = t.a.valid, nv = t.b.valid;
  if (mv == BM && nv == BN) moe_store<BM, BN, OB, true, PAST>(p, t, mv, nv, acc, lds0, wave, lane);
  else moe_store<BM, BN, OB, false, PAST>(p, t, mv, nv, acc, lds0, wave, lane);
  // the ring may be filled again (the stores need not have arrived for that)
  wait_lds_all();
  __builtin_amdgcn_s_barrier();
}

// Blocks of rows of all experts in turn, in supertiles of up to 8 of them by all blocks of columns
// (kMoeTN: every expert's blocks along the curve).
template <int BM, int BN, MoeLayout LAYOUT, bool GATHER, bool OB, bool PAST>
__global__ __launch_bounds__(256, (MoeTile<BM, BN>::PER_CU)) void moe_gemm_kernel(MoeGemmParams p) {
  using T = MoeTile<BM, BN>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = lds_addr(smem);
  const int P = gridDim.x, rank = xcd_rank(blockIdx.x, P);
  constexpr int ES = OB ? 2 : 4;
  // Calls block(task) for this workgroup's tasks: its rank of every full round, and in the last, partial one its
  // rank among as many workgroups as there are tasks left (the first ones: spread over all chiplets).  A last round
  // that is at most half full is taken in quarters of blocks, quarter(task, q): 1088 blocks of 256x256 and 64 stages on
  // 256 CUs take 473 us instead of 495.
  constexpr bool QUARTERS = BM > 64;
  auto each_task = [&](int64_t total, auto block, auto quarter) {
    const int64_t full = total / P * P;
    const int left = (int)(total - full);
    const bool quarters = QUARTERS && 2 * left <= P;
    const int64_t last = !quarters && (int)blockIdx.x < left ? full + xcd_rank(blockIdx.x, left) : -1;
    for (int64_t task = full > 0 ? rank : last; task >= 0; task = task + P < full ? task + P : task < full ? last : -1) block(task);
    if (!quarters) return;
    for (int i = blockIdx.x; i < 4 * left; i += P) {
      // (quarters of a task run on one chiplet: its ranks are consecutive)
      const int r = 4 * left <= P ? xcd_rank(i, 4 * left) : i < P ? xcd_rank(i, P) : P + xcd_rank(i - P, 4 * left - P);
      quarter(full + r / 4, r % 4);
    }
  };
  // the quarter q of a block: rows and columns it starts at, in the block
  auto cut = [&](MoeTask& t, int q) {
    const int m = (q >> 1) * (BM / 2), n = (q & 1) * (BN / 2);
    t.a.valid = t.a.valid - m < BM / 2 ? t.a.valid - m : BM / 2;
    t.b.valid = t.b.valid - n < BN / 2 ? t.b.valid - n : BN / 2;
    if constexpr (GATHER) t.a.order += m;
    else t.a.base += (uint64_t)(LAYOUT == kMoeTN ? m : m * p.lda) * 2;
    t.b.base += (uint64_t)(LAYOUT == kMoeNK ? n * p.ldb : n) * 2;
    t.C += (m * p.ldc + n) * ES;
    return t.a.valid > 0 && t.b.valid > 0;
  };
  MoeTask t = {};
  t.a.ld = p.lda;
  t.b.ld = p.ldb;
  auto run = [&](int64_t total, auto place) {
    each_task(total,
              [&](int64_t task) {
                place(task);
                moe_block<BM, BN, LAYOUT, GATHER, OB, PAST>(p, t, lds0, wave, lane);
              },
              [&](int64_t task, int q) {
                place(task);
                if constexpr (QUARTERS)
                  if (cut(t, q)) moe_block<BM / 2, BN / 2, LAYOUT, GATHER, OB, PAST>(p, t, lds0, wave, lane);
              });
  };
  if constexpr (LAYOUT == kMoeTN) {
    const Segments seg = {p.offsets, p.experts, p.K};
    const int64_t cells = (int64_t)p.gm * p.gn, total = cells * p.experts;
    auto place = [&](int64_t task) {
      const int e = (int)(task / cells);
      const int cell = load_scalar_i32(p.table + (task - (int64_t)e * cells));
      const int64_t m0 = (int64_t)(cell / p.gn) * BM, n0 = (int64_t)(cell % p.gn) * BN;
      int64_t lo, hi;
      seg.bounds(e, lo, hi);
      t.a.base = reinterpret_cast<uint64_t>(p.A) + (uint64_t)(lo * p.lda + m0) * 2;
      t.b.base = reinterpret_cast<uint64_t>(p.B) + (uint64_t)(lo * p.ldb + n0) * 2;
      t.a.valid = p.M - m0 < BM ? (int)(p.M - m0) : BM;
      t.b.valid = p.N - n0 < BN ? (int)(p.N - n0) : BN;
      t.depth = hi - lo;
      t.C = reinterpret_cast<char*>(p.C) + ((int64_t)e * p.stride_c + m0 * p.ldc + n0) * ES;
    };
    run(total, place);
  } else {
    const Segments seg = {p.offsets, p.experts, p.M};
    int used;
    const int64_t total = (int64_t)seg.blocks<BM>(lane, used) * p.gn;
    t.a.rows = p.a_rows;
    t.a.topk = p.topk;
    t.depth = p.K;
    auto place = [&](int64_t task) {
      int first = 0, gm = 0;
      const int e = __builtin_amdgcn_readfirstlane(seg.find<BM>((int)(task / p.gn), lane, first, gm));
      int64_t lo, hi;
      seg.bounds(e, lo, hi);
      const int64_t local = task - (int64_t)first * p.gn;
      const int super = (int)(local / (8 * (int64_t)p.gn));
      const int height = gm - 8 * super < 8 ? gm - 8 * super : 8;
      const int within = (int)(local - (int64_t)super * 8 * p.gn);
      const int in = within / height, im = 8 * super + within - in * height;
      const int64_t m0 = lo + (int64_t)im * BM, n0 = (int64_t)in * BN;
      t.a.base = reinterpret_cast<uint64_t>(p.A) + (GATHER ? 0 : (uint64_t)(m0 * p.lda) * 2);
      t.a.order = GATHER ? p.order + m0 : nullptr;
      t.b.base = reinterpret_cast<uint64_t>(p.B) + (uint64_t)(e * p.stride_b + (LAYOUT == kMoeNK ? n0 * p.ldb : n0)) * 2;
      t.a.valid = hi - m0 < BM ? (int)(hi - m0) : BM;
      t.b.valid = p.N - n0 < BN ? (int)(p.N - n0) : BN;
      t.C = reinterpret_cast<char*>(p.C) + (m0 * p.ldc + n0) * ES;
    };
    run(total, place);
    // rows of no expert
    for (int64_t r = (int64_t)used + blockIdx.x; r < p.M; r += P)
      for (int64_t c = tid; c < p.N; c += 256) {
        if constexpr (OB) reinterpret_cast<uint16_t*>(p.C)[r * p.ldc + c] = 0;
        else reinterpret_cast<uint32_t*>(p.C)[r * p.ldc + c] = 0;
      }
  }
}

template <int BM, int BN, MoeLayout LAYOUT, bool GATHER>
static const void* moe_kernel(bool ob, bool past) {
  return ob ? (past ? reinterpret_cast<const void*>(&moe_gemm_kernel<BM, BN, LAYOUT, GATHER, true, true>)
                    : reinterpret_cast<const void*>(&moe_gemm_kernel<BM, BN, LAYOUT, GATHER, true, false>))
            : (past ? reinterpret_cast<const void*>(&moe_gemm_kernel<BM, BN, LAYOUT, GATHER, false, true>)
                    : reinterpret_cast<const void*>(&moe_gemm_kernel<BM, BN, LAYOUT, GATHER, false, false>));
}

template <int BM, int BN>
static hipError_t moe_launch(const MoeGemmParams& p, MoeLayout layout, bool out_bf16, int grid, hipStream_t stream) {
  const void* k = layout == kMoeTN   ? moe_kernel<BM, BN, kMoeTN, false>(out_bf16, p.past)
                  : layout == kMoeKN ? (p.order ? moe_kernel<BM, BN, kMoeKN, true>(out_bf16, p.past)
                                                : moe_kernel<BM, BN, kMoeKN, false>(out_bf16, p.past))
                                     : (p.order ? moe_kernel<BM, BN, kMoeNK, true>(out_bf16, p.past)
                                                : moe_kernel<BM, BN, kMoeNK, false>(out_bf16, p.past));
  MoeGemmParams local = p;
  void* args[] = {&local};
  return hipLaunchKernel(k, dim3((unsigned)grid), dim3(256), args, 0, stream);
}

}  // namespace sfc
