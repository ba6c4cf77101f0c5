// Rows sorted by expert, seen by a workgroup: segment bounds, and which expert holds the n-th
// block of rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sfc {

// Rows offsets[e] .. offsets[e+1]-1 belong to expert e; bounds outside 0 .. rows are moved there.
struct Segments {
  const int32_t* offsets;
  int experts;
  int64_t rows;

  __device__ __forceinline__ void bounds(int e, int64_t& lo, int64_t& hi) const {
    lo = offsets[e];
    hi = offsets[e + 1];
    lo = lo < 0 ? 0 : lo > rows ? rows : lo;
    hi = hi < lo ? lo : hi > rows ? rows : hi;
  }

  // Blocks of BM rows of all experts (a part-filled last one for each), and the end of the last
  // segment.  Whole waves call it.
  template <int BM>
  __device__ __forceinline__ int blocks(int lane, int& used) const {
    int n = 0;
    used = 0;
    for (int e = lane; e < experts; e += 64) {
      int64_t lo, hi;
      bounds(e, lo, hi);
      n += (int)((hi - lo + BM - 1) / BM);
      used = hi > used ? (int)hi : used;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const int other = __shfl_xor(used, d);
      used = other > used ? other : used;
      n += __shfl_xor(n, d);
    }
    return __builtin_amdgcn_readfirstlane(n);
  }

  // The expert that holds block of rows `mt` (there is one), the blocks of rows before its own,
  // and its own.
  template <int BM>
  __device__ __forceinline__ int find(int mt, int lane, int& first, int& own) const {
    int carry = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
      int n = 0;
      if (e0 + lane < experts) {
        int64_t lo, hi;
        bounds(e0 + lane, lo, hi);
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
        own = __builtin_amdgcn_readfirstlane(__shfl(n, l));
        first = __builtin_amdgcn_readfirstlane(carry + __shfl(sum, l)) - own;
        return e0 + l;
      }
      carry += __builtin_amdgcn_readfirstlane(__shfl(sum, 63));
    }
    return -1;
  }
};

}  // namespace sfc
