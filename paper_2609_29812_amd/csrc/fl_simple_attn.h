// Softmax attention of one row by one wave, over keys and values that a source hands out in fp32.
#pragma once

#include "fl_paged4.h"

namespace fl {

struct RowOut {
  uint16_t* o;
  float* lse;
};

// The lane's channels of q (lane + 64 x) stand in `q`; keys j in [0, last] with j >= low or j < n_sink that the source has.
template <int D, bool F16, class Src>
__device__ __forceinline__ void attend_row(const Src& src, const float* q, float scale, int last, int low, int n_sink, uint16_t* o,
                                           float* lse) {
  const int lane = threadIdx.x & 63;
  float ref = -INFINITY, sum = 0.0f, acc[D / 64];
#pragma unroll
  for (int x = 0; x < D / 64; ++x) acc[x] = 0.0f;
  for (int j = 0; j <= last; ++j) {
    if (j >= n_sink && j < low) j = low;
    if (!src.there(j)) continue;
    float s = 0.0f;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) s = fmaf(q[x], src.key(j, lane + 64 * x), s);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off, 64);
    s *= scale;
    const float bad = src.spoilt(j);
    const float m = fmaxf(ref, s), f = ref == -INFINITY ? 0.0f : expf(ref - m), p = expf(s - (m == -INFINITY ? 0.0f : m)) + bad;
    sum = fmaf(sum, f, p + s * 0.0f);
#pragma unroll
    for (int x = 0; x < D / 64; ++x) acc[x] = fmaf(acc[x], f, p * src.value(j, lane + 64 * x));
    ref = m;
  }
  const bool none = ref == -INFINITY && sum == 0.0f;
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    const float y = none ? 0.0f : acc[x] / sum;
    o[lane + 64 * x] = (uint16_t)(F16 ? pack_f16x2(y, 0.0f) : pack_bf16x2(y, 0.0f));
  }
  if (lse && lane == 0) *lse = none ? -INFINITY : ref + logf(sum);
}

// q of one row, channel lane + 64 x, turned by row `pos` of the table.
template <int D, bool F16>
__device__ __forceinline__ void turned_query(const uint16_t* row, const Rotary& rt, int pos, float* q) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    const int c = lane + 64 * x;
    q[x] = to_f32<F16>(row[c]);
    if (rt.table && c < rt.rot) {
      const bool apart = rt.layout == FL_ROPE_HALF;
      const int i = apart ? c % (rt.rot / 2) : c / 2;
      const bool first = apart ? c < rt.rot / 2 : (c & 1) == 0;
      const int mate = apart ? (first ? c + rt.rot / 2 : c - rt.rot / 2) : c ^ 1;
      const float y = to_f32<F16>(row[mate]), co = rt.table[(int64_t)pos * rt.rot + 2 * i], si = rt.table[(int64_t)pos * rt.rot + 2 * i + 1];
      q[x] = first ? q[x] * co - y * si : fmaf(q[x], co, y * si);
    }
  }
}

}  // namespace fl
