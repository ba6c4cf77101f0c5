// Adapters, down in tiles: V[t] = s[a] X[t] A[a]^T for batches whose rows come in runs, on the K loop of the
// experts' products with 64x64 blocks (rows x ranks).
//
// A workgroup takes 64 rows, 64 ranks, a range of K and every kSlots-th of the rows' adapters; it computes with
// one adapter after the other, from its weights and all 64 rows, and keeps the sums of that adapter's
// rows.  A rank of 16 or 64 is one block of columns, so without a split of K there would be 64
// workgroups for 4096 rows: the sums of the ranges of K go to memory, and a second kernel adds them up in
// order, scales them and clears rows of no adapter.  (Rows of one adapter leave the other slots
// nothing to do; a tile where two meet takes no longer, for they run beside each other.)  Bound: one read of X for every 64
// ranks: 6.5 us for 4096 rows x 4096, where rank 64 takes 20: 16 stages, the sums' way through memory and a second launch, 4.
#include "sfc_launch.h"
#include "sfc_lora_params.h"
#include "sfc_moe_gemm_kernel.h"

namespace sfc {

namespace {

constexpr int kTile = kDownTile, kSlots = 4;

template <bool NK>
__global__ __launch_bounds__(256, 4) void lora_down_kernel(LoraParams p) {
  using T = MoeTile<kTile, kTile>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[T::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t t0 = (int64_t)blockIdx.x * kTile;
  const int slot = blockIdx.z % kSlots, r0 = (int)(blockIdx.z / kSlots) * kTile;
  // this workgroup's range of K, in stages
  const int64_t stages = (p.cols + 63) >> 6;
  const int64_t k0 = stages * blockIdx.y / p.splits * 64, k1 = stages * (blockIdx.y + 1) / p.splits * 64;
  const int64_t t = t0 + lane < p.rows ? t0 + lane : p.rows - 1;
  const int a0 = p.ids[t], id = t0 + lane < p.rows && a0 >= 0 && a0 < p.adapters ? a0 : -1;
  float* sums = p.sums + (int64_t)blockIdx.y * p.rows * p.rank;
  MoeTask task = {};
  task.a.base = reinterpret_cast<uint64_t>(p.X) + (uint64_t)(t0 * p.ldx + k0) * 2;
  task.a.ld = p.ldx;
  task.a.valid = p.rows - t0 < kTile ? (int)(p.rows - t0) : kTile;
  task.b.ld = p.ldw;
  task.b.valid = p.rank - r0 < kTile ? p.rank - r0 : kTile;
  task.depth = (k1 < p.cols ? k1 : p.cols) - k0;
  uint64_t pending = __ballot(id >= 0);
  for (int turn = 0; pending; ++turn) {
    const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(pending));
    const uint64_t rows = __ballot(id == a);
    pending &= ~rows;
    if (turn % kSlots != slot) continue;
    task.b.base = reinterpret_cast<uint64_t>(p.W) + (uint64_t)(a * p.stride_w + (NK ? r0 * p.ldw + k0 : k0 * p.ldw + r0)) * 2;
    f32x4 acc[2][2];
    moe_accumulate<kTile, kTile, NK ? kMoeNK : kMoeKN, false>(task, lds_addr(smem), wave, lane, acc);
    // wave: 32 rows x 32 ranks; lane: row l % 16 and 4 ranks of a fragment
    const float scale = p.splits == 1 && p.scales ? p.scales[a] : 1.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 32 * (wave >> 1) + 16 * i + (lane & 15);
      if (!(rows >> row & 1)) continue;
      float* out = p.splits == 1 ? p.V + (t0 + row) * p.ldv : sums + (t0 + row) * p.rank;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = r0 + 32 * (wave & 1) + 16 * j + 4 * (lane >> 4) + e;
          if (r < p.rank) out[r] = scale * acc[i][j][e];
        }
    }
  }
  if (p.splits > 1 || slot != 0) return;
  // rows of no adapter
  for (uint64_t none = __ballot(id < 0 && t0 + lane < p.rows); none; none &= none - 1) {
    const int64_t row = t0 + __builtin_ctzll(none);
    if (tid < kTile && r0 + tid < p.rank) p.V[row * p.ldv + r0 + tid] = 0.f;
  }
}

// V from the sums of the ranges of K, in their order: a workgroup takes 256 / LANES rows, LANES threads a row.
template <int LANES>
__global__ __launch_bounds__(256) void lora_down_sum(LoraParams p) {
  const int64_t t = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (t >= p.rows) return;
  const int a = p.ids[t];
  const bool live = a >= 0 && a < p.adapters;
  const float scale = live && p.scales ? p.scales[a] : 1.f;
  const int64_t n = p.rows * p.rank;
  for (int r = threadIdx.x % LANES; r < p.rank; r += LANES) {
    const float* s = p.sums + t * p.rank + r;
    float v = 0.f;
    for (int k = 0; k < p.splits; k += 8) {
      float part[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) part[u] = s[(k + u < p.splits ? k + u : p.splits - 1) * n];
      __builtin_amdgcn_sched_barrier(0);       // (all loads are on their way first)
#pragma unroll
      for (int u = 0; u < 8; ++u) v = k + u < p.splits ? v + part[u] : v;
    }
    p.V[t * p.ldv + r] = live ? scale * v : 0.f;
  }
}

}  // namespace

hipError_t launch_lora_down_tiles(const LoraParams& p, bool nk, hipStream_t stream) {
  const dim3 grid((unsigned)((p.rows + kTile - 1) / kTile), (unsigned)p.splits, (unsigned)(kSlots * ((p.rank + kTile - 1) / kTile)));
  hipError_t e = launch_kernel(nk ? lora_down_kernel<true> : lora_down_kernel<false>, grid, dim3(256), 0, stream, p);
  if (e != hipSuccess || p.splits == 1) return e;
  if (p.rank <= 16) return launch_kernel(lora_down_sum<16>, dim3((unsigned)((p.rows + 15) / 16)), dim3(256), 0, stream, p);
  return launch_kernel(lora_down_sum<64>, dim3((unsigned)((p.rows + 3) / 4)), dim3(256), 0, stream, p);
}

}  // namespace sfc
