// Device helpers shared by the kernels of the paged cache.
#pragma once

#include "gemm_device.h"
#include "paged.h"
#include "sq_device.h"

namespace sq {

// A softmax state is sums of 2^(s - m), m at or near the running maximum of s.  With m = -inf it has no
// token: the output is zero where all states are such.  One with tokens whose scores are all -inf or
// NaN has m = kNoScore instead, which weighs as little beside a finite m and keeps its sums (0 or NaN:
// 0 / 0 or NaN in the end, as the definition has it).
constexpr float kNoScore = -3.402823466e38f;

// value of the lane whose quad index is this lane's xor M (M = 1 or 2)
template <int M>
__device__ __forceinline__ float quad_swap(float v) {
  constexpr int ctrl = (M == 1) ? 0xB1 : 0x4E;  // quad_perm [1,0,3,2] / [2,3,0,1]
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xF, 0xF, false));
}
template <int M>
__device__ __forceinline__ double quad_swap(double v) {
  constexpr int ctrl = (M == 1) ? 0xB1 : 0x4E;
  const int lo = __builtin_amdgcn_mov_dpp(__double2loint(v), ctrl, 0xF, 0xF, false);
  const int hi = __builtin_amdgcn_mov_dpp(__double2hiint(v), ctrl, 0xF, 0xF, false);
  return __hiloint2double(hi, lo);
}

// Unscaled 128-point Sylvester transform of the 128 values of a quad of lanes: register r and
// lane bits j are the index bits in any order (the transform is the same under a permutation of
// the bits that input and output share).
template <typename F>
__device__ __forceinline__ void quad_fwht(F (&e)[32], int j) {
#pragma unroll
  for (int h = 1; h < 32; h <<= 1)
#pragma unroll
    for (int r = 0; r < 32; ++r)
      if ((r & h) == 0) {
        const F u = e[r], w = e[r + h];
        e[r] = u + w;
        e[r + h] = u - w;
      }
  const F s1 = (j & 1) ? F(-1) : F(1), s2 = (j & 2) ? F(-1) : F(1);
#pragma unroll
  for (int r = 0; r < 32; ++r) e[r] = fma(s1, e[r], quad_swap<1>(e[r]));
#pragma unroll
  for (int r = 0; r < 32; ++r) e[r] = fma(s2, e[r], quad_swap<2>(e[r]));
}

// Sequence of row t of a packed call (cu [B + 1], ascending): its index, the rows it begins at and
// ends before, and its length; -1 for a row of none.  The whole wave searches, 64 sequences a step,
// and their lengths come along (a second trip to memory would follow the first).
struct RowSeq {
  int seq;
  int end;
  int len;
};
__device__ __forceinline__ RowSeq find_sequence(const int32_t* cu, const int32_t* lens, int64_t B, int64_t t) {
  const int lane = threadIdx.x & 63;
  for (int64_t b0 = 0; b0 < B; b0 += 64) {
    const int64_t b = b0 + lane;
    int begin = 0, end = 0, len = 0;
    if (b < B) {
      begin = cu[b];
      end = cu[b + 1];
      len = lens[b];
    }
    const uint64_t past = __ballot(b < B && end > t);
    if (past) {
      const int first = __builtin_ctzll(past);
      const int seq = t < __builtin_amdgcn_readlane(begin, first) ? -1 : static_cast<int>(b0) + first;
      return {seq, __builtin_amdgcn_readlane(end, first), __builtin_amdgcn_readlane(len, first)};
    }
  }
  return {-1, 0, 0};
}

// op over the lane's value and those of the lanes 16, 32 and 48 further (mod 64)
template <typename Op>
__device__ __forceinline__ float rows_all(float v, Op op) {
  const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
  const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
}

// Exchanges a in the upper (odd) halves / rows of 16 lanes with b in the lower (even) ones: what was
// a lane bit of the pair becomes the choice of a or b.
__device__ __forceinline__ void swap_halves(double& a, double& b) {
  const auto lo = __builtin_amdgcn_permlane32_swap(__double2loint(a), __double2loint(b), false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap(__double2hiint(a), __double2hiint(b), false, false);
  a = __hiloint2double(hi[0], lo[0]);
  b = __hiloint2double(hi[1], lo[1]);
}
__device__ __forceinline__ void swap_rows(double& a, double& b) {
  const auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(a), __double2loint(b), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(a), __double2hiint(b), false, false);
  a = __hiloint2double(hi[0], lo[0]);
  b = __hiloint2double(hi[1], lo[1]);
}

}  // namespace sq
