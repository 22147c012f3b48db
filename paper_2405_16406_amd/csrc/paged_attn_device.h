// What the attentions over the paged cache share: how a wave takes 64 tokens' codes as matrix operands,
// and its softmax states (paged_attn.hip has the mathematics).
#pragma once

#include "paged_device.h"
#include "paged_plan.h"
#include "sq_internal.h"

namespace sq {

constexpr int kBlock = kPagedBlock;  // tokens of a wave's step
constexpr float kSlack = 3.0f;      // log2: weights stay below 2^(kWeightBits + kSlack) < 65504
constexpr float kWeightBits = 12.0f;
// Exponents of this size have steps of 1/2: from there on m is the maximum itself, since kWeightBits
// below it might be rounded to more than fp16 holds (the differences s - m themselves are exact).
constexpr float kLargeScore = 4194304.0f;  // 2^22

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 2^(a - b), 0 when a is -inf (an empty state)
__device__ __forceinline__ float rescale(float a, float b) { return a == -INFINITY ? 0.0f : exp2_fast(__fsub_rn(a, b)); }

__device__ __forceinline__ v8h operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(v8h, v4u{a, b, c, d});
}

// LDS of a wave: value codes of a block, then four rows of 64 token coefficients (a, b, 1 / va,
// vb / va with s_t + log2 va_t = a_t (q . c_t) + b_t sum(q) + lv_t, five rows with lv).
template <int BITS>
struct WaveLds {
  static constexpr int ROW = BITS * 16;          // bytes of a token's value codes
  static constexpr int CODES = kBlock * ROW;
  static constexpr int BYTES = CODES + 5 * kBlock * 4;
};

// Two value codes n, each times 2^shift in a half's low bits, as the normal numbers n 2^-9.
// Beside a much larger weight, sums of subnormal codes lose the low bits of the smaller ones, always
// downwards: as if products were lined up by their operands' exponents, which for a subnormal is the
// smallest normal one whatever its leading zeros.  Over 131071 tokens of 4 bits that is 2e-6 of
// sum w e, whose bulk cancels against b: the output was off by 7.3e-4 of its size, 6.6e-4 of it
// one-sided, and with normal codes by 2.7e-4, less than 1e-5 one-sided (8 bits: 2.7e-4 and 6.6e-5,
// now 2.6e-4).  It costs 0.2 us of 10.5 for one short sequence, 0.4 of 39.8 for that long one, 1.1 of
// 57.6 for 64 sequences.
// Key codes stay subnormal: with normal ones no output came nearer, with queries 4 and 16 times as
// large neither, and the products cost up to 1.6 us more.
__device__ __forceinline__ uint32_t normal(uint32_t two, int shift) {
  const _Float16 up = static_cast<_Float16>(static_cast<float>(1 << (15 - shift)));
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, two) * v2h{up, up});
}

// Floats of a row of the merge of a workgroup's states.
constexpr int kDimRow = 132;

}  // namespace sq
