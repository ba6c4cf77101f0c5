// Tokens sorted by expert and back.
//
// A slot is one (token, choice) pair, slot = token * topk + choice, with an expert id; ids
// outside 0 .. experts-1 are dropped slots.  Sorting is stable: the rows of an expert
// follow one another in slot order, from a start that is a multiple of `align`.
//
//   dispatch   Xs[p] = w[order[p]] * X[order[p] / topk]          (0 where order[p] < 0)
//   combine    Y[t] = sum_j w[t, j] * Ys[pos[t, j]]              (pos < 0: no term)
//   gradient   dYs[pos[t, j]] = w[t, j] * dY[t],  dw[t, j] = <dY[t], Ys[pos[t, j]]>
//
// The gradient of dispatch without weights is combine without weights.  Sums run in fp32
// over j ascending, dot products in fp32 over a fixed split of the columns: no result
// depends on the order in which workgroups run.
//
// Bound: memory, every row read and written once (a token's row once per choice).  8192
// tokens x 4096 bf16, 2 of 8 experts: dispatch 40.8 us (4.9 TB/s), combine 36.7 (5.5), its
// gradient 66 (5.1); a copy of as much runs at 5.2.
#include "sfc_launch.h"
#include "sfc_ops_params.h"
#include "sfc_row_io.h"

namespace sfc {

// ---- sort ----------------------------------------------------------------------------------
// A workgroup of 16 waves ranks a chunk of kSortChunk slots, a wave 64 at a time in slot
// order.  The lanes of a wave that hold the same expert find each other by one ballot per
// bit of the id; a running count per wave and expert lies in LDS.  With several chunks a
// first launch counts every chunk's slots per expert, which every workgroup of the sort adds
// up; past kSortScan chunks a launch between them does (us, added up by all / by that launch,
// 64 experts: 2^17 slots 9.5 / 11.0, 2^18 10.7 / 11.7, 2^20 20.8 / 15.8; 2^23 slots of 256
// experts 350 / 70, where reading the ids twice and writing both orders once is 27 at copy rate).
constexpr int kSortWaves = 16;

__global__ __launch_bounds__(1024) void moe_count_kernel(MoeSortParams p) {
  extern __shared__ int32_t hist[];
  for (int e = threadIdx.x; e < p.experts; e += 1024) hist[e] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortChunk;
  for (int i = threadIdx.x; i < kSortChunk; i += 1024) {
    if (first + i < p.slots) {
      const uint32_t e = (uint32_t)p.ids[first + i];
      if (e < (uint32_t)p.experts) atomicAdd(&hist[e], 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += 1024) p.counts[(int64_t)blockIdx.x * p.experts + e] = hist[e];
}

// The chunks' counts replaced by the counts of the chunks before, their sums in a last row; a
// workgroup takes 16 experts, thread (g, e) every chunk of the g-th of 64 ranges.
__global__ __launch_bounds__(1024) void moe_scan_kernel(int32_t* counts, int experts, int chunks) {
  __shared__ int32_t sums[64][16];
  const int e16 = threadIdx.x & 15, g = threadIdx.x >> 4, e = blockIdx.x * 16 + e16;
  const int each = (chunks + 63) >> 6, first = g * each < chunks ? g * each : chunks;
  const int last = first + each < chunks ? first + each : chunks;
  int sum = 0;
  if (e < experts) {
#pragma unroll 8
    for (int ch = first; ch < last; ++ch) sum += counts[(int64_t)ch * experts + e];
  }
  sums[g][e16] = sum;
  __syncthreads();
  int run = 0;
  for (int i = 0; i < g; ++i) run += sums[i][e16];
  if (e < experts) {
    if (g == 63) counts[(int64_t)chunks * experts + e] = run + sum;
    for (int ch = first; ch < last; ch += 8) {
      int32_t n[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = ch + i < last ? counts[(int64_t)(ch + i) * experts + e] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (ch + i < last) counts[(int64_t)(ch + i) * experts + e] = run;
        run += n[i];
      }
    }
  }
}

// LDS: [kSortWaves][experts] running positions, then 16 + 1 scan words.
__global__ __launch_bounds__(1024) void moe_sort_kernel(MoeSortParams p, int chunks, int bits) {
  extern __shared__ int32_t hist[];
  int32_t* wave_sum = hist + kSortWaves * p.experts;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kSortWaves * p.experts; i += 1024) hist[i] = 0;
  __syncthreads();

  constexpr int kRounds = kSortChunk / 1024;
  const int64_t first = (int64_t)blockIdx.x * kSortChunk + wave * (64 * kRounds) + lane;
  int32_t* mine = hist + wave * p.experts;
  uint32_t id[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t slot = first + 64 * r;
    id[r] = slot < p.slots ? (uint32_t)p.ids[slot] : 0xFFFFFFFFu;
    if (id[r] < (uint32_t)p.experts) atomicAdd(&mine[id[r]], 1);
  }
  __syncthreads();

  // thread e: expert e's count in all chunks and in those before this one
  int total = 0, before = 0;
  if (tid < p.experts) {
    if (chunks == 1) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) total += hist[w * p.experts + tid];
    } else if (chunks > kSortScan) {
      total = p.counts[(int64_t)chunks * p.experts + tid];
      before = p.counts[(int64_t)blockIdx.x * p.experts + tid];
    } else {
#pragma unroll 8
      for (int ch = 0; ch < chunks; ++ch) {
        const int n = p.counts[(int64_t)ch * p.experts + tid];
        total += n;
        before += ch < (int)blockIdx.x ? n : 0;
      }
    }
  }
  const int padded = (total + p.align - 1) / p.align * p.align;
  // inclusive sum of the padded counts
  int sum = padded;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(sum, d);
    sum += lane >= d ? up : 0;
  }
  if (lane == 63) wave_sum[wave] = sum;
  __syncthreads();
  if (wave == 0) {
    int s = lane < kSortWaves ? wave_sum[lane] : 0;
#pragma unroll
    for (int d = 1; d < kSortWaves; d <<= 1) {
      const int up = __shfl_up(s, d);
      s += lane >= d ? up : 0;
    }
    if (lane < kSortWaves) wave_sum[lane] = s;
  }
  __syncthreads();
  if (wave > 0) sum += wave_sum[wave - 1];
  const int start = sum - padded;
  const int end = wave_sum[kSortWaves - 1];
  if (tid < p.experts) {
    int run = start + before;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int n = hist[w * p.experts + tid];
      hist[w * p.experts + tid] = run;
      run += n;
    }
    if (blockIdx.x == 0) {
      p.offsets[tid] = start;
      if (tid == p.experts - 1) p.offsets[p.experts] = sum;
      for (int i = start + total; i < sum; ++i) p.order[i] = -1;
    }
  }
  for (int64_t i = end + (int64_t)blockIdx.x * 1024 + tid; i < p.rows; i += (int64_t)gridDim.x * 1024) p.order[i] = -1;
  __syncthreads();

#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t slot = first + 64 * r;
    const bool valid = id[r] < (uint32_t)p.experts;
    uint64_t same = __ballot(valid);
    for (int b = 0; b < bits; ++b) {
      const uint64_t ones = __ballot((id[r] >> b) & 1);
      same &= ((id[r] >> b) & 1) ? ones : ~ones;
    }
    int at = -1;
    if (valid) at = mine[id[r]] + __popcll(same & ((1ull << lane) - 1));
    // (the other lanes' stores are seen: LDS serves a wave's accesses in order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // the last lane of each expert carries the count on
    if (valid && (same >> lane) == 1) mine[id[r]] = at + 1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (slot < p.slots) p.pos[slot] = at;
    if (valid) p.order[at] = (int32_t)slot;
  }
}

hipError_t launch_moe_sort(const MoeSortParams& p, hipStream_t stream) {
  const int chunks = p.slots > 0 ? (int)((p.slots + kSortChunk - 1) / kSortChunk) : 1;
  if (chunks > 1) {
    const hipError_t e = launch_kernel(moe_count_kernel, dim3(chunks), dim3(1024), p.experts * 4u, stream, p);
    if (e != hipSuccess) return e;
  }
  if (chunks > kSortScan) {
    const hipError_t e = launch_kernel(moe_scan_kernel, dim3((p.experts + 15) / 16), dim3(1024), 0, stream, p.counts, p.experts,
                                       chunks);
    if (e != hipSuccess) return e;
  }
  int bits = 0;
  while ((1 << bits) < p.experts) ++bits;
  const unsigned lds = (unsigned)(kSortWaves * p.experts + kSortWaves) * 4u;
  return launch_kernel(moe_sort_kernel, dim3(chunks), dim3(1024), lds, stream, p, chunks, bits);
}

// ---- dispatch ------------------------------------------------------------------------------
template <bool BF16, bool PAST>
__global__ __launch_bounds__(256) void moe_dispatch_kernel(MoeRowsParams p, RowShape sh) {
  const RowPlace at = row_place(sh, (p.cols + 7) >> 3);
  if (at.row >= p.rows) return;
  const int32_t slot = p.order[at.row];
  const int64_t token = slot < 0 ? -1 : (int64_t)((uint32_t)slot / (uint32_t)p.topk);
  const bool valid = token >= 0 && token < p.tokens;
  const float w = valid && p.weights ? p.weights[slot] : 1.0f;
  const char* x = reinterpret_cast<const char*>(p.X) + (valid ? token : 0) * p.ldx * (BF16 ? 2 : 4);
  char* y = reinterpret_cast<char*>(p.Y) + at.row * p.ldy * (BF16 ? 2 : 4);
  constexpr int U = 4;
  Raw8<BF16> r[U];
  row_loop<U>(
      at, [&](int u, int64_t c) { r[u] = valid ? load8<BF16>(x, c * 8, p.cols) : zero8<BF16>(); },
      [&](int u, int64_t c) {
        if (p.weights) {
          float f[8];
          to_float<BF16>(r[u], f);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= w;
          r[u] = from_float<BF16>(f);
        }
        store8<BF16, PAST>(y, c * 8, p.cols, r[u]);
      });
}

// ---- combine -------------------------------------------------------------------------------
// Two choices at a time, two chunks of each: four loads in flight.
template <bool BF16, bool PAST>
__global__ __launch_bounds__(256) void moe_combine_kernel(MoeRowsParams p, RowShape sh) {
  const RowPlace at = row_place(sh, (p.cols + 7) >> 3);
  if (at.row >= p.tokens) return;
  const char* ys = reinterpret_cast<const char*>(p.X);
  char* y = reinterpret_cast<char*>(p.Y) + at.row * p.ldy * (BF16 ? 2 : 4);
  const int32_t* pos = p.pos + at.row * p.topk;
  const float* weights = p.weights ? p.weights + at.row * p.topk : nullptr;
  for (int64_t c = at.first + at.lane_tx; c < at.last; c += 2 * at.tx) {
    const bool two = c + at.tx < at.last;
    float sum[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[0][i] = sum[1][i] = 0.f;
    for (int j = 0; j < p.topk; j += 2) {
      Raw8<BF16> r[2][2];
      float w[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t row = j + u < p.topk ? pos[j + u] : -1;
        const bool valid = row >= 0 && row < p.rows;
        const char* src = ys + row * p.ldx * (BF16 ? 2 : 4);
        r[u][0] = valid ? load8<BF16>(src, c * 8, p.cols) : zero8<BF16>();
        r[u][1] = valid && two ? load8<BF16>(src, (c + at.tx) * 8, p.cols) : zero8<BF16>();
        w[u] = valid ? (weights ? weights[j + u] : 1.0f) : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float f[8];
          to_float<BF16>(r[u][k], f);
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[k][i] += f[i] * w[u];
        }
    }
    store8<BF16, PAST>(y, c * 8, p.cols, from_float<BF16>(sum[0]));
    if (two) store8<BF16, PAST>(y, (c + at.tx) * 8, p.cols, from_float<BF16>(sum[1]));
  }
}

// ---- gradient of combine -------------------------------------------------------------------
// L lanes per token, two choices at a time (dy is read once for both); before the tokens'
// workgroups, others clear the rows that no slot has, 16 rows to each (they lie together: 256
// rows to a workgroup took 28 us longer for 8191 tokens in segments of 32).
template <bool BF16, bool PAST, int L>
__global__ __launch_bounds__(256) void moe_combine_grad_kernel(MoeRowsParams p, int64_t clear_groups) {
  __shared__ float part[2][4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t chunks = (p.cols + 7) >> 3;
  constexpr int ES = BF16 ? 2 : 4;
  if ((int64_t)blockIdx.x < clear_groups) {
    for (int i = 0; i < 4; ++i) {
      const int64_t r = p.first_row + (int64_t)blockIdx.x * 16 + 4 * wave + i;
      if (r >= p.end_row) break;
      const int32_t slot = p.order[r];
      if (slot >= 0 && (int64_t)slot < p.tokens * p.topk) continue;
      char* y = reinterpret_cast<char*>(p.Y) + r * p.ldy * ES;
      for (int64_t c = lane; c < chunks; c += 64) store8<BF16, PAST>(y, c * 8, p.cols, zero8<BF16>());
    }
    return;
  }
  const int64_t t = p.first_token + ((int64_t)blockIdx.x - clear_groups) * (256 / L) + threadIdx.x / L;
  const int lane_t = threadIdx.x & (L - 1);
  const bool in = t < p.end_token;
  const char* dy = reinterpret_cast<const char*>(p.X) + (in ? t : 0) * p.ldx * ES;
  for (int j = 0; j < p.topk; j += 2) {
    bool valid[2];
    float w[2], dot[2] = {0.f, 0.f};
    const char* ys[2];
    char* y[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = in && j + u < p.topk ? p.pos[t * p.topk + j + u] : -1;
      valid[u] = at >= 0 && at < p.rows;
      w[u] = valid[u] && p.weights ? p.weights[t * p.topk + j + u] : 1.0f;
      ys[u] = reinterpret_cast<const char*>(p.Ys) + (valid[u] ? at : 0) * p.ldys * ES;
      y[u] = reinterpret_cast<char*>(p.Y) + (valid[u] ? at : 0) * p.ldy * ES;
    }
    if (valid[0] || valid[1]) {
      constexpr int U = 2;
      for (int64_t c = lane_t; c < chunks; c += U * L) {
        Raw8<BF16> a[U], b[U][2];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t ck = c + k * L;
          if (ck < chunks) {
            a[k] = load8<BF16>(dy, ck * 8, p.cols);
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (valid[u]) b[k][u] = load8<BF16>(ys[u], ck * 8, p.cols);
          }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t ck = c + k * L;
          if (ck < chunks) {
            float f[8];
            to_float<BF16>(a[k], f);
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (valid[u]) {
                float g[8], o[8];
                to_float<BF16>(b[k][u], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  dot[u] += f[i] * g[i];
                  o[i] = f[i] * w[u];
                }
                store8<BF16, PAST>(y[u], ck * 8, p.cols, from_float<BF16>(o));
              }
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int d = L < 64 ? L / 2 : 32; d >= 1; d >>= 1) dot[u] += __shfl_xor(dot[u], d);
    if constexpr (L == 256) {
      if (lane == 0) {
        part[0][wave] = dot[0];
        part[1][wave] = dot[1];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < 2; ++u) dot[u] = (part[u][0] + part[u][1]) + (part[u][2] + part[u][3]);
      __syncthreads();
    }
    if (in && lane_t == 0) {
      p.dW[t * p.topk + j] = dot[0];
      if (j + 1 < p.topk) p.dW[t * p.topk + j + 1] = dot[1];
    }
  }
}

hipError_t launch_moe_dispatch(const MoeRowsParams& in, bool bf16, int num_cus, hipStream_t stream) {
  MoeRowsParams p = in;
  if (!bf16 && !p.weights) {
    // a copy of bits: as rows of twice as many 2-byte values, a lane's stores are the wave's whole lines
    // (8192 tokens x 4096 fp32, 2 of 8: 104 -> 77 us)
    p.cols *= 2;
    p.ldx *= 2;
    p.ldy *= 2;
    bf16 = true;
  }
  // (fp32: a lane's two stores leave holes in a line, which only the caches fill: 104 -> 81 us)
  const bool past = bf16 && streams_past_caches(p.rows * p.cols * 2);
  const RowShape sh = row_shape(p.rows, (p.cols + 7) / 8, num_cus);
  const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
  if (past) return launch_kernel(moe_dispatch_kernel<true, true>, g, b, 0, stream, p, sh);
  if (bf16) return launch_kernel(moe_dispatch_kernel<true, false>, g, b, 0, stream, p, sh);
  return launch_kernel(moe_dispatch_kernel<false, false>, g, b, 0, stream, p, sh);
}

hipError_t launch_moe_combine(const MoeRowsParams& p, bool bf16, int num_cus, hipStream_t stream) {
  // (us, through / past, 2 choices: fp32 8192x1024 22.3 / 19.0, 131072x64 22.8 / 19.7, 16384x1024 42.4 / 40.5,
  // 8192x4096 77.7 / 77.3, 16384x4096 155 / 153, 1 choice 8192x8192 104 / 106; bf16 16384x1024 21.5 / 17.1,
  // 65536x256 22.3 / 16.8, 16384x4096 79.8 / 74.5)
  const bool past = streams_past_caches(p.tokens * p.cols * (bf16 ? 2 : 4));
  const RowShape sh = row_shape(p.tokens, (p.cols + 7) / 8, num_cus);
  const dim3 g((unsigned)(sh.row_blocks * sh.splits)), b(256);
  if (bf16 && past) return launch_kernel(moe_combine_kernel<true, true>, g, b, 0, stream, p, sh);
  if (bf16) return launch_kernel(moe_combine_kernel<true, false>, g, b, 0, stream, p, sh);
  if (past) return launch_kernel(moe_combine_kernel<false, true>, g, b, 0, stream, p, sh);
  return launch_kernel(moe_combine_kernel<false, false>, g, b, 0, stream, p, sh);
}

template <bool BF16, bool PAST>
static const void* grad_kernel(int lanes) {
  return lanes == 256  ? reinterpret_cast<const void*>(&moe_combine_grad_kernel<BF16, PAST, 256>)
         : lanes == 64 ? reinterpret_cast<const void*>(&moe_combine_grad_kernel<BF16, PAST, 64>)
                       : reinterpret_cast<const void*>(&moe_combine_grad_kernel<BF16, PAST, 16>);
}

hipError_t launch_moe_combine_grad(const MoeRowsParams& p, bool bf16, int num_cus, hipStream_t stream) {
  // as many lanes to a token as have about two loads of its row (us, 4 waves / one / 16 lanes: 8192 tokens
  // x 4096 bf16 67 / 81 / -, 16384 x 1024 - / 35 / -, 16384 x 200 - / 12.5 / 8.1,
  // 16384 x 64 - / 10.5 / 5.2)
  const int lanes = p.cols >= 2048 ? 256 : p.cols > 256 ? 64 : 16;
  // fp32 rows of 128 MB or more stay in the caches, which join a line's halves (us, through / past, 2 choices:
  // fp32 8192x1024, 64 MB, 39.3 / 33.9, 131072x64 66 / 61, 16384x1024, 128 MB, 73.3 / 75.7, 4096x4096 71.8 / 76.2,
  // 65536x256 79 / 82, 8192x4096, 256 MB, 137 / 150, 16384x4096 268 / 295; bf16 16384x1024, 64 MB, 38.5 / 32.2,
  // 131072x64 40 / 35, 8192x4096, 128 MB, 70.0 / 69.0, 16384x4096 137 / 136)
  const int64_t bytes = p.rows * p.cols * (bf16 ? 2 : 4);
  const bool past = streams_past_caches(bytes) && (bf16 || bytes < (int64_t)128 << 20);
  const int64_t groups = ((p.end_token - p.first_token) * lanes + 255) / 256;
  const int64_t clear = (p.end_row - p.first_row + 15) / 16;
  const dim3 g((unsigned)(groups + clear)), b(256);
  const void* k = bf16 ? (past ? grad_kernel<true, true>(lanes) : grad_kernel<true, false>(lanes))
                       : (past ? grad_kernel<false, true>(lanes) : grad_kernel<false, false>(lanes));
  MoeRowsParams local = p;
  int64_t clear_groups = clear;
  void* args[] = {&local, &clear_groups};
  return hipLaunchKernel(k, g, b, args, 0, stream);
}

}  // namespace sfc
