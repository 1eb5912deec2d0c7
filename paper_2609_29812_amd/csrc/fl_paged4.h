// The paged 4-bit cache: its groups' numbers and codes, as all its kernels read them.
#pragma once

#include "fl_paged.h"

namespace fl {

constexpr int kGroup = 32;                 // channels of a group
constexpr uint32_t kNaN4 = 0x7E007E00u;    // numbers of a group that is not there: fp16 NaN, NaN
constexpr uint32_t kMaxScale4 = 0x6C45u, kMaxZero4 = 0x7800u;      // fp16 bits of 4372 and 2^15
constexpr int kMinExp4 = -23, kMaxExp4 = 13;

// whether a group's numbers are such as an append writes: int4 scale | zero << 16, e2m1 the exponent's byte
template <bool INT>
__device__ __forceinline__ bool group_ok(uint32_t m) {
  if constexpr (INT) {
    // (pages are never cleared: two numbers within their bounds may still stand for values beyond fp16's)
    const _Float16 s = __builtin_bit_cast(_Float16, (uint16_t)m), z = __builtin_bit_cast(_Float16, (uint16_t)(m >> 16));
    const bool finite = __builtin_elementwise_fma(s, (_Float16)15.0f, z) <= (_Float16)65504.0f;
    return ((m & 0xFFFFu) <= kMaxScale4) & (((m >> 16) & 0x7FFFu) <= kMaxZero4) & finite;
  }
  return m - (uint32_t)(kMinExp4 + 127) <= (uint32_t)(kMaxExp4 - kMinExp4);
}

// Bytes of a group's numbers.
template <bool INT>
constexpr int meta_bytes() { return INT ? 4 : 1; }

template <bool INT>
__device__ __forceinline__ uint32_t load_meta(const uint8_t* at) {
  if constexpr (INT) return *reinterpret_cast<const uint32_t*>(at);
  else return *at;
}

// The eight values of a word of codes in fp32: one rounding of z + s c; c 2^e exactly.  NaN where the group's numbers are none.
template <bool INT>
__device__ __forceinline__ void values8(uint32_t w, uint32_t meta, float* x) {
  const bool ok = group_ok<INT>(meta);
  if constexpr (INT) {
    const float s = ok ? f16_bits_to_f32(meta & 0xFFFFu) : NAN, z = f16_bits_to_f32(meta >> 16);
    const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(s, (float)(((e & 1 ? odd : even) >> (8 * (e / 2))) & 0xFFu), z);
  } else {
    const float s = ok ? __uint_as_float(meta << 23) : NAN;
    typedef float pair __attribute__((ext_vector_type(2)));
    const pair y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s * y[e / 2][e & 1];
  }
}

// host: the checks that the calls of the 4-bit cache have in common
int check_paged4(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                 const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                 int num_pages, int page, int format, const void* kc, const void* vc, const void* km, const void* vm);

}  // namespace fl
