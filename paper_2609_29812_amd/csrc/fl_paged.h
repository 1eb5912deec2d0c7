// What the paged cache's kernels share: the description of a ragged batch and of a cache, argument checks, and the
// exact conversions between 16-bit values and codes.
#pragma once

#include "fl_attn_util.h"

namespace fl {

struct Batch {                   // rows cu[b] .. cu[b+1]-1 are the last positions of sequence b
  const int32_t *cu, *lens, *table;
  int B, T, max_pages;
};

struct Rotary {                  // cosines and sines fp32 [n_pos, rot / 2, 2]; table == nullptr: no rotation
  const float* table;
  int rot, layout;
};

struct Pages {
  int num, size, log2, heads;    // pages, positions per page, key/value heads
};

// cu[b] as a row number in [0, T], whatever it holds
__device__ __forceinline__ int row_of(const Batch& bt, int b) { return min(max(bt.cu[b], 0), bt.T); }

// The last sequence b whose first slot, f(cu[b]) + extra * b, is at most `slot` (b = -1: there is none), its rows and its
// length.  f ascends, so with extra >= 1 a sequence's slots are slot numbers of its own.  The wave looks at 64 places at a time
// until 64 sequences are left; their rows and lengths are one round of loads, which stands before everything else that a workgroup
// reads.
struct Seq {
  int b, r0, r1, len;
};
template <class F>
__device__ __forceinline__ Seq find_seq(const Batch& bt, int slot, int extra, F f) {
  const int lane = threadIdx.x & 63;
  int lo = 0, left = bt.B;                                   // the sequence is one of lo .. lo + left - 1, if there is one
  while (left > 64) {
    const int step = (left + 63) / 64;
    const int b = lo + lane * step;
    const uint64_t m = __builtin_amdgcn_ballot_w64(lane * step < left && f(row_of(bt, min(b, bt.B - 1))) + extra * b <= slot);
    const int n = max((int)__popcll(m), 1);
    left = min(step, left - (n - 1) * step);
    lo += (n - 1) * step;
  }
  const int b = lo + lane, bc = min(b, bt.B - 1);
  const int r0 = row_of(bt, bc), r1 = row_of(bt, bc + 1), len = bt.lens[bc];
  const int n = __popcll(__builtin_amdgcn_ballot_w64(lane < left && f(r0) + extra * b <= slot));
  if (n == 0) return {-1, 0, 0, 0};
  return {lo + n - 1, __builtin_amdgcn_readlane(r0, n - 1), __builtin_amdgcn_readlane(r1, n - 1), __builtin_amdgcn_readlane(len, n - 1)};
}

// 16-bit value to fp32 (exact)
template <bool F16>
__device__ __forceinline__ float to_f32(uint32_t bits16) {
  if constexpr (F16) return f16_bits_to_f32(bits16);
  else return bf16_to_f32(bits16);
}
// eight values of 16 bytes
template <bool F16>
__device__ __forceinline__ void unpack8(const uint4& w, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = to_f32<F16>(u[e] & 0xFFFFu);
    x[2 * e + 1] = to_f32<F16>(u[e] >> 16);
  }
}
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float* x) {
  uint32_t u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = F16 ? pack_f16x2(x[2 * e], x[2 * e + 1]) : pack_bf16x2(x[2 * e], x[2 * e + 1]);
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// host: the checks that the calls of a paged cache have in common
int check_paged(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                int num_pages, int page, int format, const void* kc, const void* vc, const float* ks, const float* vs);
int check_rows(const char* fn, const char* name, const void* x, int64_t stride, int H, int d);
// T rows of `width` 16-bit elements each: no element in common
int check_apart(const char* fn, const char* xn, const void* x, int64_t xs, const char* yn, const void* y, int64_t ys, int T,
                int width);
int check_rotary(const char* fn, const float* table, int rot, int layout, int d);
// with the index checks on: cu, lens and block_table on the host (`append`: the pages of the new positions too)
int check_batch(const char* fn, const Batch& bt, const Pages& pg, bool append, hipStream_t st);

inline int log2_of(int x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }

}  // namespace fl
