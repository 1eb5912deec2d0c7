// The 4-bit cache's attention: its arguments and the widening of codes that its kernels share.
#pragma once

#include "fl_paged4.h"
#include "fl_paged_attn.h"

namespace fl {

struct Paged4Args : PagedAttnArgs {
  const uint8_t *km, *vm;
};

// Two codes of 4 bits as fp16, from a word whose halves hold one each at the same place: at the low four bits of a byte they stand
// under the exponent of 1024, at the high four under that of 64.  Exact.  (One constant in a vector register: both as literals take
// two instructions.)
struct Magic {
  uint32_t low, high;
  __device__ __forceinline__ Magic() : low(0x64006400u), high(0x54005400u) { asm volatile("" : "+v"(low), "+v"(high)); }
};
__device__ __forceinline__ f16x2 low_pair(uint32_t w, const Magic& m) {
  const f16x2 off = {(_Float16)-1024.0f, (_Float16)-1024.0f};
  return __builtin_bit_cast(f16x2, (w & 0x000F000Fu) | m.low) + off;
}
__device__ __forceinline__ f16x2 high_pair(uint32_t w, const Magic& m) {
  const f16x2 off = {(_Float16)-64.0f, (_Float16)-64.0f};
  return __builtin_bit_cast(f16x2, (w & 0x00F000F0u) | m.high) + off;
}
__device__ __forceinline__ uint32_t apply(f16x2 c, f16x2 s, f16x2 z) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, s, z));
}
__device__ __forceinline__ f16x2 both_low(uint32_t a, uint32_t b) { return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(b, a, 0x05040100u)); }
__device__ __forceinline__ f16x2 both_high(uint32_t a, uint32_t b) { return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(b, a, 0x07060302u)); }

// What a pair's rounding to fp16 leaves, in fp16.
__device__ __forceinline__ uint32_t pack_rest(float x, float y, uint32_t rounded) {
  const f16x2 r = __builtin_bit_cast(f16x2, rounded);
  return pack_f16x2(fmaf((float)r[0], -1.0f, x), fmaf((float)r[1], -1.0f, y));
}

// Eight codes of one group in fp16: int4 one rounding of z + s c, in the order 0 4 1 5 2 6 3 7; e2m1 exactly, in their order.
template <bool INT>
__device__ __forceinline__ u32x4 widen8(uint32_t w, uint32_t meta, const Magic& g) {
  if constexpr (INT) {
    const f16x2 s = both_low(meta, meta), z = both_high(meta, meta);
    const uint32_t v = w >> 8;
    return u32x4{apply(low_pair(w, g), s, z), apply(high_pair(w, g), s, z), apply(low_pair(v, g), s, z), apply(high_pair(v, g), s, z)};
  } else {
    const float s = __uint_as_float(meta << 23);
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3))};
  }
}
// Eight int4 codes as two parts each whose sum is z + s c to 22 bits: the value's rounding, and that of what it leaves.
__device__ __forceinline__ void widen8_two(uint32_t w, uint32_t meta, const Magic& g, u32x4& hi, u32x4& lo) {
  const f16x2 sz = __builtin_bit_cast(f16x2, meta);
  const float s = (float)sz[0], z = (float)sz[1];
  const uint32_t v = w >> 8;
  const f16x2 c[4] = {low_pair(w, g), high_pair(w, g), low_pair(v, g), high_pair(v, g)};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = fmaf((float)c[e][0], s, z), y = fmaf((float)c[e][1], s, z);
    hi[e] = pack_f16x2(x, y);
    lo[e] = pack_rest(x, y, hi[e]);
  }
}
// byte `i` of a word of e2m1 codes as a pair
template <int I>
__device__ __forceinline__ uint32_t widen_byte(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, I));
}
// A query that is not finite: NaN in its place, and the factor 1, so that what it does not see stays out of its sums.  A factor below
// 2^-126 (a query near 0 and a small sm_scale) counts as that: masked scores, -inf, are multiplied by it, and -inf times 0 would be NaN.
// (The products with it are below 2^24, so their exponents are 0 to 2^-102 either way.)
template <int N>
__device__ __forceinline__ float finite_factor(float m, f16x8* q) {
  if (m == m) return fmaxf(m, 0x1p-126f);
#pragma unroll
  for (int k = 0; k < N; ++k) q[k] = __builtin_bit_cast(f16x8, u32x4{0x7E007E00u, 0x7E007E00u, 0x7E007E00u, 0x7E007E00u});
  return 1.0f;
}
// eight channels of a query in widen8's order
template <bool INT>
__device__ __forceinline__ f16x8 in_order(const f16x8& q) {
  if constexpr (INT) return __builtin_shufflevector(q, q, 0, 4, 1, 5, 2, 6, 3, 7);
  else return q;
}

// many rows
struct PromptShape;
size_t paged4_prompt_ws(const PromptShape& s, int d);
int launch_paged4_prompt(const Paged4Args& a, int d, int format, bool f16, const PromptShape& shape, hipStream_t st);

}  // namespace fl
