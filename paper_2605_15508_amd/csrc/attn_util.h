// Device helpers that the attention kernels share.
#pragma once

#include "common.h"

// position of the n-th set bit (n < popcount)
__device__ __forceinline__ int nth_member(uint32_t mask, int n) {
  const int first = __builtin_ctz(mask);
  const uint32_t run = mask >> first;
  if ((run & (run + 1)) == 0) return first + n;      // (mask is the same for all lanes; nearly always one run of bits)
  int pos = 0;
#pragma unroll
  for (int i = 0; i < STS_MAX_GROUP; ++i) {
    const bool set = (mask >> i) & 1u;
    if (set && n == 0) pos = i;
    n -= set ? 1 : 0;
  }
  return pos;
}

// The larger of two numbers, one instruction: the median with +infinity (fmaxf first turns signalling NaNs into quiet ones, an
// instruction per operand that the compiler cannot vouch for).
__device__ __forceinline__ float larger(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, INFINITY); }

// the larger of two, or a NaN where one of them is one
__device__ __forceinline__ float top(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// maximum over the four lanes 16 apart (the row-of-16 swaps of this chip: no LDS round trip)
__device__ __forceinline__ float max_over_groups(float x) {
  const uint32_t w = __builtin_bit_cast(uint32_t, x);
  const auto p = __builtin_amdgcn_permlane16_swap(w, w, false, false);       // rows 0, 0, 2, 2 and 1, 1, 3, 3
  const float y = larger(__builtin_bit_cast(float, (uint32_t)p[0]), __builtin_bit_cast(float, (uint32_t)p[1]));
  const uint32_t v = __builtin_bit_cast(uint32_t, y);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);       // the lower and the upper half
  return larger(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}

// The sum over a row's 16 lanes, in every one of them: pairs, quads, halves, all.
__device__ __forceinline__ float row_sum16(float x) {
  auto add = [&](auto ctrl) {
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  add(std::integral_constant<int, 0xb1>());     // quad_perm: lane ^ 1
  add(std::integral_constant<int, 0x4e>());     // quad_perm: lane ^ 2
  add(std::integral_constant<int, 0x141>());    // row_half_mirror: the other quad of the eight
  add(std::integral_constant<int, 0x140>());    // row_mirror: the other eight
  return x;
}

// One more part of a row, of maximum ms (in powers of two), sum ls and weighted sums x relative to it, joined to the row's m, l and
// o. What has no maximum, an empty part or a token whose score is -infinity, has no weight and is left out: -inf - -inf is no
// number.
template <int N>
__device__ __forceinline__ void merge_part(float &m, float &l, float (&o)[N], float ms, float ls, const float *x) {
  if (ms == -INFINITY) return;
  const float m_new = fmaxf(m, ms);
  const float fo = __builtin_amdgcn_exp2f(m - m_new);   // 0 while nothing is accumulated
  const float fn = __builtin_amdgcn_exp2f(ms - m_new);
  l = l * fo + ls * fn;
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = o[e] * fo + x[e] * fn;
  m = m_new;
}
