// Appending to the paged key/value cache: rotation of the keys, 8-bit codes with one scale per page and head, and the
// requantization of a page whose scale grows.
#include "fl_paged.h"

#include <algorithm>
#include <vector>

namespace fl {

int check_ragged(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                 const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                 int num_pages, int page) {
  FL_REQUIRE(dtype == FL_BF16 || dtype == FL_F16, FL_E_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  FL_REQUIRE(d == 64 || d == 128, FL_E_SHAPE, "%s: d=%d must be 64 or 128", fn, d);
  FL_REQUIRE(page == 16 || page == 32 || page == 64 || page == 128, FL_E_SHAPE, "%s: page=%d must be 16, 32, 64 or 128", fn,
             page);
  FL_REQUIRE(B >= 1 && B <= 65536 && T >= 0, FL_E_SHAPE, "%s: B=%d must be in [1, 65536] and T=%d >= 0", fn, B, T);
  FL_REQUIRE(Hkv >= 1 && Hkv <= 65535, FL_E_SHAPE, "%s: Hkv=%d must be in [1, 65535]", fn, Hkv);
  FL_REQUIRE(max_pages >= 1 && (int64_t)max_pages * page <= INT_MAX - 4096, FL_E_SHAPE,
             "%s: max_pages=%d pages of %d positions: between 1 page and 2^31 - 4097 positions", fn, max_pages, page);
  FL_REQUIRE(num_pages >= 1, FL_E_SHAPE, "%s: num_pages=%d must be positive", fn, num_pages);
  FL_REQUIRE(cu && lens && block_table, FL_E_NULL, "%s: cu, lens and block_table are required", fn);
  if (table) {
    const int rc = check_rotary(fn, table, rot, layout, d);
    if (rc != FL_OK) return rc;
    FL_REQUIRE((int64_t)n_pos >= (int64_t)max_pages * page, FL_E_RANGE,
               "%s: a table of %d positions for sequences of up to %d pages of %d", fn, n_pos, max_pages, page);
  }
  return FL_OK;
}

int check_paged(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                int num_pages, int page, int format, const void* kc, const void* vc, const float* ks, const float* vs) {
  FL_REQUIRE(format == FL_KV_I8 || format == FL_KV_E4M3, FL_E_UNSUPPORTED, "%s: unknown cache format %d", fn, format);
  const int rc = check_ragged(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(kc && vc && ks && vs, FL_E_NULL, "%s: k_cache, v_cache, k_scale and v_scale are required", fn);
  FL_REQUIRE(kc != vc && ks != vs, FL_E_SHAPE, "%s: keys and values need a cache and scales each", fn);
  FL_REQUIRE(((reinterpret_cast<uintptr_t>(kc) | reinterpret_cast<uintptr_t>(vc)) & 15) == 0, FL_E_SHAPE,
             "%s: the caches must be 16-byte aligned", fn);
  return FL_OK;
}

int check_batch(const char* fn, const Batch& bt, const Pages& pg, bool append, hipStream_t st) {
  if (!index_checks_on()) return FL_OK;
  std::vector<int32_t> cu((size_t)bt.B + 1), lens((size_t)bt.B), table((size_t)bt.B * bt.max_pages);
  hipError_t e = hipStreamSynchronize(st);
  if (e == hipSuccess) e = hipMemcpy(cu.data(), bt.cu, cu.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess) e = hipMemcpy(lens.data(), bt.lens, lens.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && append) e = hipMemcpy(table.data(), bt.table, table.size() * 4, hipMemcpyDeviceToHost);
  FL_REQUIRE(e == hipSuccess, FL_E_HIP, "%s: index check: copy to the host failed: %s", fn, hipGetErrorString(e));
  FL_REQUIRE(cu[0] == 0, FL_E_RANGE, "%s: cu[0] = %d must be 0", fn, cu[0]);
  std::vector<char> used(append ? (size_t)pg.num : 0, 0);
  for (int b = 0; b < bt.B; ++b) {
    const int n = cu[b + 1] - cu[b];
    FL_REQUIRE(cu[b + 1] >= cu[b] && cu[b + 1] <= bt.T, FL_E_RANGE, "%s: cu[%d] = %d after %d, of %d rows", fn, b + 1, cu[b + 1],
               cu[b], bt.T);
    FL_REQUIRE(lens[b] >= n && (int64_t)lens[b] <= (int64_t)bt.max_pages * pg.size, FL_E_RANGE,
               "%s: lens[%d] = %d outside [%d, %lld]", fn, b, lens[b], n, (long long)bt.max_pages * pg.size);
    if (!append || n == 0) continue;
    for (int p = (lens[b] - n) / pg.size; p <= (lens[b] - 1) / pg.size; ++p) {
      const int id = table[(size_t)b * bt.max_pages + p];
      FL_REQUIRE(id >= 0 && id < pg.num, FL_E_RANGE, "%s: block_table[%d][%d] = %d outside [0, %d)", fn, b, p, id, pg.num);
      FL_REQUIRE(!used[id], FL_E_RANGE, "%s: page %d is appended to twice (block_table[%d][%d])", fn, id, b, p);
      used[id] = 1;
    }
  }
  return FL_OK;
}

struct AppendArgs {
  const uint16_t *k, *v;
  int64_t ks, vs;                  // row strides
  Batch bt;
  Rotary rt;
  Pages pg;
  uint8_t *kc, *vc;
  float *ksc, *vsc;
  int hp;                          // heads of a workgroup
};

constexpr uint32_t kInfBits = 0x7F800000u;

// need of (10) for the largest magnitude (its fp32 bits)
template <bool I8>
__device__ __forceinline__ float scale_for(uint32_t amax_bits) {
  if (amax_bits >= kInfBits) return NAN;
  const float a = __uint_as_float(amax_bits);
  if (a < 0x1p-100f) return 0.0f;
  if constexpr (I8) return a * (1.0f / 127.0f);
  // 448 = 1.75 * 2^8: a = m 2^e needs 2^(e - 8), or twice that when m > 1.75
  const int e = (int)(amax_bits >> 23) - 127;
  return ldexpf(1.0f, e - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// the least k >= 0 with s 2^k >= need (both finite and positive); ldexp of a normal fp32 is exact
__device__ __forceinline__ int doublings(float s, float need) {
  if (!(need > s)) return 0;
  const int k = max(0, ilogbf(need) - ilogbf(s));
  return ldexpf(s, k) >= need ? k : k + 1;
}

// round(x / s) to nearest, ties to even, of the exact quotient: the product with the rounded reciprocal is within one step;
// its remainder x - q s is exact in one fma and decides.
__device__ __forceinline__ int code_i8(float x, float s, float inv) {
  const float q = rintf(x * inv);
  const float r = fmaf(-q, s, x);
  const float over = 2.0f * fabsf(r) - s;
  const bool step = (over > 0.0f) | ((over == 0.0f) & (((int)q & 1) != 0));
  return (int)(q + (step ? copysignf(1.0f, r) : 0.0f));   // (|x| <= 127 s (1 + 2^-23): at most 127)
}

// Eight codes.  Int8: x * inv rounded to an integer by the addition of 1.5 * 2^23 (its low byte is the code); inv is off by at
// most 2^-24 of itself, which decides only where the product lies within 2^-16 of a half: there the remainder does.
template <bool I8>
__device__ __forceinline__ uint2 encode8(const float* x, float s, float inv) {
  uint32_t w[2];
  if constexpr (I8) {
    constexpr float kRound = 12582912.0f;
    float t[8], off = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] = fmaf(x[e], inv, kRound);
      off = fmaxf(off, fabsf(fmaf(x[e], inv, kRound - t[e])));
    }
    if (off > 0.49998f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = kRound + (float)code_i8(x[e], s, inv);
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * g + 1]), __float_as_uint(t[4 * g]), 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * g + 3]), __float_as_uint(t[4 * g + 2]), 0x04000c0cu);
      w[g] = lo | hi;
    }
  } else {
#pragma unroll
    for (int g = 0; g < 2; ++g) {               // the scale is a power of two: the products are exact
      int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * g] * inv, x[4 * g + 1] * inv, 0, false);
      w[g] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * g + 2] * inv, x[4 * g + 3] * inv, u, true);
    }
  }
  return make_uint2(w[0], w[1]);
}

// codes / 2^k, rounded to nearest even (f = 2^-k)
template <bool I8>
__device__ __forceinline__ uint2 shrink8(uint2 c, float f) {
  uint32_t in[2] = {c.x, c.y}, w[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if constexpr (I8) {
      uint32_t u = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) u |= (uint32_t)((int)rintf((float)(int8_t)(in[g] >> (8 * e)) * f) & 0xFF) << (8 * e);
      w[g] = u;
    } else {
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[g], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[g], true);
      int u = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
      w[g] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, u, true);
    }
  }
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ uint32_t low16(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high16(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// The page of a slot: slots cu[b] / page + 2 b .. belong to sequence b, which touches at most n / page + 2 pages with n new
// positions (the grid covers T / page + 2 B slots).  Rows lo .. hi - 1 of the page are new, row i being row `first` + i of the
// batch; pid < 0: nothing to do.
struct Place {
  int pid, p0, lo, hi;
  int64_t first;
};
__device__ __forceinline__ Place place_of(const AppendArgs& a, int slot, int log2) {
  Place w{-1, 0, 0, 0, 0};
  const Seq s = find_seq(a.bt, slot, 2, [log2](int c) { return c >> log2; });
  const int n = s.r1 - s.r0;
  if (s.b < 0 || n <= 0 || s.len <= 0) return w;
  const int start = max(s.len - n, 0);                       // first stored position; (len - n < 0: the first are dropped)
  const int64_t pi = (int64_t)(start >> log2) + (slot - ((s.r0 >> log2) + 2 * s.b));
  if (pi >= a.bt.max_pages) return w;
  w.p0 = (int)pi << log2;
  w.lo = max(start, w.p0) - w.p0;
  w.hi = min(s.len - w.p0, 1 << log2);
  if (w.lo >= w.hi) return w;
  w.first = (int64_t)s.r0 + w.p0 - (s.len - n);
  const int pid = a.bt.table[(int64_t)s.b * a.bt.max_pages + pi];
  w.pid = (uint32_t)pid < (uint32_t)a.pg.num ? pid : -1;
  return w;
}

// What a thread does with its 16 channels of a position: chunks c0 and c1 of eight, the two values of every pair that it turns.
// Pairs that lie side by side are drawn apart while the thread holds them (mixed).
struct Unit {
  int c0, c1, u;
  bool turn, mixed;
};
__device__ __forceinline__ Unit unit_of(const AppendArgs& a, bool is_k, int u) {
  const int turned = is_k && a.rt.table ? a.rt.rot / 16 : 0;
  const bool half = a.rt.layout == FL_ROPE_HALF, turn = u < turned;
  return {half && turn ? u : 2 * u, half && turn ? u + turned : 2 * u + 1, u, turn, !half && turned > 0};
}
__device__ __forceinline__ void load_cs(const AppendArgs& a, const Unit& un, int pos, float* cs) {
  const float4* row = reinterpret_cast<const float4*>(a.rt.table + (int64_t)pos * a.rt.rot + un.u * 16);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 w = row[e];
    cs[4 * e] = w.x; cs[4 * e + 1] = w.y; cs[4 * e + 2] = w.z; cs[4 * e + 3] = w.w;
  }
}
template <bool F16>
__device__ __forceinline__ void values_of(const Unit& un, uint4 w0, uint4 w1, const float* cs, float* x) {
  if (un.mixed) {
    const uint4 a0 = w0, a1 = w1;
    w0 = make_uint4(low16(a0.x, a0.y), low16(a0.z, a0.w), low16(a1.x, a1.y), low16(a1.z, a1.w));
    w1 = make_uint4(high16(a0.x, a0.y), high16(a0.z, a0.w), high16(a1.x, a1.y), high16(a1.z, a1.w));
  }
  unpack8<F16>(w0, x);
  unpack8<F16>(w1, x + 8);
  if (un.turn) {
    // the products of 8- or 11-bit values with fp32 ones are exact in fp64: one rounding, by the sum, then fp32
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double p = x[e], q = x[e + 8], c = cs[2 * e], sn = cs[2 * e + 1];
      x[e] = (float)fma(p, c, -(q * sn));
      x[e + 8] = (float)fma(p, sn, q * c);
    }
  }
}
__device__ __forceinline__ uint32_t largest(const float* x, uint32_t most) {          // (NaN above inf above finite)
#pragma unroll
  for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  return most;
}
// The page's scale, and the halvings of what it holds.
template <bool I8>
__device__ __forceinline__ float grow(float held, uint32_t most, bool went_on, int& k) {
  const float need = scale_for<I8>(most);
  k = 0;
  if (!went_on || held == 0.0f) return need;
  if (isnan(need) || !isfinite(held)) return NAN;
  k = doublings(held, need);
  return ldexpf(held, k);
}
// The factor of the codes; 0, for codes of 0, where the scale is NaN or below that of 2^-100: then every value counts as 0 (a held
// scale that a caller formed may be so small that its reciprocal, or a value over it, leaves its range).
template <bool I8>
__device__ __forceinline__ float inverse(float sc) {
  constexpr float kLeast = I8 ? 0x1p-100f * (1.0f / 127.0f) : 0x1p-108f;
  return sc >= kLeast ? 1.0f / sc : 0.0f;
}
template <bool I8>
__device__ __forceinline__ void put(const Unit& un, uint8_t* row, const float* x, float sc, float inv) {
  uint2 y0 = make_uint2(0, 0), y1 = y0;
  if (inv > 0.0f) {
    y0 = encode8<I8>(x, sc, inv);
    y1 = encode8<I8>(x + 8, sc, inv);
  }
  if (un.mixed) {
    const uint2 p = y0, q = y1;
    y0 = make_uint2(__builtin_amdgcn_perm(q.x, p.x, 0x05010400u), __builtin_amdgcn_perm(q.x, p.x, 0x07030602u));
    y1 = make_uint2(__builtin_amdgcn_perm(q.y, p.y, 0x05010400u), __builtin_amdgcn_perm(q.y, p.y, 0x07030602u));
  }
  uint2* at = reinterpret_cast<uint2*>(row);
  at[un.c0] = y0;
  at[un.c1] = y1;
}
template <bool I8>
__device__ __forceinline__ void halve(const Unit& un, uint8_t* row, float f) {
  uint2* at = reinterpret_cast<uint2*>(row);
  at[un.c0] = shrink8<I8>(at[un.c0], f);
  at[un.c1] = shrink8<I8>(at[un.c1], f);
}

// Many positions: a workgroup has one page, keys or values, and hp heads one after the other.  The cosines and sines stay in
// registers for all heads and the next head's values are asked for before this one's are reduced; the largest magnitude meets
// through LDS, then the codes go out.  32768 positions of 8 heads x 128 (210 MB): 57 us as int8, 55 as e4m3, 48 without a
// rotation, 3.7 TB/s; vector instructions are issued in half of the time (18 per value of a wave, fp64 sums and rounding the
// most), the rest waits for a page's chain of load, maximum and store.  8 channels a thread and one head a workgroup took 89 us.
template <int D, int PAGE, bool I8, bool F16>
__global__ __launch_bounds__(PAGE * D / 16 < 256 ? PAGE * D / 16 : 256) void paged_append_kernel(AppendArgs a) {
  constexpr int TPP = D / 16;                                 // threads of a position
  constexpr int NT = PAGE * TPP < 256 ? PAGE * TPP : 256, PER = NT / TPP, NP = PAGE / PER, NW = NT / 64;
  constexpr int LOG2 = PAGE == 16 ? 4 : PAGE == 32 ? 5 : PAGE == 64 ? 6 : 7;
  __shared__ uint32_t s_max[2][NW];
  // the heads of a page, keys and values, by neighbouring workgroups: together they read whole rows
  const int hg = (a.pg.heads + a.hp - 1) / a.hp;
  const int slot = blockIdx.x / (2 * hg), part = blockIdx.x % (2 * hg);
  const bool is_k = part < hg;
  const Place w = place_of(a, slot, LOG2);
  if (w.pid < 0) return;
  const uint16_t* src = is_k ? a.k : a.v;
  const int64_t stride = is_k ? a.ks : a.vs;
  const int i0 = threadIdx.x / TPP;
  const Unit un = unit_of(a, is_k, threadIdx.x % TPP);
  float cs[NP][16];
#pragma unroll
  for (int s = 0; s < NP; ++s) {
    const int i = s * PER + i0;
#pragma unroll
    for (int e = 0; e < 16; ++e) cs[s][e] = 0.0f;
    if (un.turn && i >= w.lo && i < w.hi) load_cs(a, un, w.p0 + i, cs[s]);
  }
  const int h0 = part % hg * a.hp, h1 = min(h0 + a.hp, a.pg.heads);
  uint4 raw[NP][2];                                           // the next head's values
  auto load = [&](int h) {
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      const int i = s * PER + i0;
      raw[s][0] = raw[s][1] = make_uint4(0, 0, 0, 0);
      if (i >= w.lo && i < w.hi) {
        const uint4* at = reinterpret_cast<const uint4*>(src + (w.first + i) * stride + (int64_t)h * D);
        raw[s][0] = at[un.c0];
        raw[s][1] = at[un.c1];
      }
    }
  };
  load(h0);
  for (int h = h0; h < h1; ++h) {
    const int64_t head = (int64_t)w.pid * a.pg.heads + h;
    uint8_t* codes = (is_k ? a.kc : a.vc) + head * (PAGE * D);
    float* scale = (is_k ? a.ksc : a.vsc) + head;
    const float held = *scale;
    float x[NP][16];
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      values_of<F16>(un, raw[s][0], raw[s][1], cs[s], x[s]);
      most = largest(x[s], most);
    }
    if (h + 1 < h1) load(h + 1);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, 64));
    uint32_t* room = s_max[h & 1];                            // (the last head's may still be read)
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < NW; ++v) most = max(most, room[v]);
    int k;
    const float sc = grow<I8>(held, most, w.lo > 0, k);
    if (k > 0) {
      const float f = ldexpf(1.0f, -k);
#pragma unroll
      for (int s = 0; s < NP; ++s) {
        const int i = s * PER + i0;
        if (i < w.lo || i >= w.hi) halve<I8>(un, codes + i * D, f);
      }
    }
    const float inv = inverse<I8>(sc);
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      const int i = s * PER + i0;
      if (i >= w.lo && i < w.hi) put<I8>(un, codes + i * D, x[s], sc, inv);
    }
    if (threadIdx.x == 0) *scale = sc;
  }
}

// Few positions per sequence (single ones, above all): a wave has a page, a head, keys or values, and takes the new rows alone,
// 1024 / D at a time; more than that are read once for the largest magnitude and again for the codes.  Bound by latency: one
// position for each of 32 sequences, 8 heads x 128, 3.7 us.
template <int D, bool I8, bool F16>
__global__ __launch_bounds__(256) void paged_append_few_kernel(AppendArgs a, int waves) {
  constexpr int TPP = D / 16, PER = 64 / TPP;
  const int lane = threadIdx.x & 63;
  const int idx = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (idx >= waves) return;
  const int slot = idx / (2 * a.pg.heads), part = idx % (2 * a.pg.heads);
  const bool is_k = part < a.pg.heads;
  const int h = is_k ? part : part - a.pg.heads;
  const Place w = place_of(a, slot, a.pg.log2);
  if (w.pid < 0) return;
  const uint16_t* src = is_k ? a.k : a.v;
  const int64_t stride = is_k ? a.ks : a.vs;
  const int64_t head = (int64_t)w.pid * a.pg.heads + h;
  uint8_t* codes = (is_k ? a.kc : a.vc) + head * (a.pg.size * D);
  float* scale = (is_k ? a.ksc : a.vsc) + head;
  const float held = *scale;
  const int i0 = lane / TPP;
  const Unit un = unit_of(a, is_k, lane % TPP);
  float x[16];
  auto read = [&](int i) {                                    // row i of the page, when it is new
    float cs[16];
    uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
#pragma unroll
    for (int e = 0; e < 16; ++e) cs[e] = 0.0f;
    if (i < w.hi) {
      const uint4* at = reinterpret_cast<const uint4*>(src + (w.first + i) * stride + (int64_t)h * D);
      w0 = at[un.c0];
      w1 = at[un.c1];
      if (un.turn) load_cs(a, un, w.p0 + i, cs);
    }
    values_of<F16>(un, w0, w1, cs, x);
  };
  uint32_t most = 0;
  const int last = w.lo + (w.hi - w.lo - 1) / PER * PER;      // the last chunk stays in registers
  for (int i = w.lo; i <= last; i += PER) {
    read(i + i0);
    most = largest(x, most);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, 64));
  int k;
  const float sc = grow<I8>(held, most, w.lo > 0, k);
  if (k > 0) {
    const float f = ldexpf(1.0f, -k);
    for (int i = i0; i < a.pg.size; i += PER)
      if (i < w.lo || i >= w.hi) halve<I8>(un, codes + i * D, f);
  }
  const float inv = inverse<I8>(sc);
  for (int i = last; i >= w.lo; i -= PER) {
    if (i < last) read(i + i0);
    if (i + i0 < w.hi) put<I8>(un, codes + (i + i0) * D, x, sc, inv);
  }
  if (lane == 0) *scale = sc;
}

template <int D, int PAGE>
static void launch_append(const AppendArgs& a, unsigned grid, int format, int dtype, hipStream_t st) {
  constexpr int NT = PAGE * D / 16 < 256 ? PAGE * D / 16 : 256;
  if (format == FL_KV_I8) {
    if (dtype == FL_F16) paged_append_kernel<D, PAGE, true, true><<<grid, NT, 0, st>>>(a);
    else paged_append_kernel<D, PAGE, true, false><<<grid, NT, 0, st>>>(a);
  } else {
    if (dtype == FL_F16) paged_append_kernel<D, PAGE, false, true><<<grid, NT, 0, st>>>(a);
    else paged_append_kernel<D, PAGE, false, false><<<grid, NT, 0, st>>>(a);
  }
}

}  // namespace fl

using namespace fl;

extern "C" int fl_paged_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype, const int32_t* cu,
                               const int32_t* lens, int B, int T, int Hkv, int d, const float* table, int n_pos, int rot,
                               int layout, const int32_t* block_table, int max_pages, int num_pages, int page, int format,
                               void* k_cache, void* v_cache, float* k_scale, float* v_scale, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_paged_append";
  int rc = check_paged(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page,
                       format, k_cache, v_cache, k_scale, v_scale);
  if (rc != FL_OK) return rc;
  if (T == 0) return FL_OK;
  rc = check_rows(fn, "k", k, k_stride, Hkv, d);
  if (rc != FL_OK) return rc;
  rc = check_rows(fn, "v", v, v_stride, Hkv, d);
  if (rc != FL_OK) return rc;
  hipStream_t st = as_stream(stream);
  AppendArgs a{};
  a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v); a.ks = k_stride; a.vs = v_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<uint8_t*>(k_cache); a.vc = static_cast<uint8_t*>(v_cache); a.ksc = k_scale; a.vsc = v_scale;
  rc = check_batch(fn, a.bt, a.pg, true, st);
  if (rc != FL_OK) return rc;
  // up to eight new positions per sequence on average: a wave per page and head, without a workgroup's barrier (32 sequences of
  // one position: 4 us against 7)
  if (T <= 8 * (int64_t)B) {
    const int64_t waves = ((int64_t)T / page + 2 * (int64_t)B) * Hkv * 2;
    FL_REQUIRE(waves < (1ll << 31), FL_E_SHAPE, "%s: T * Hkv too large", fn);
    const unsigned few = (unsigned)((waves + 3) / 4);
    const int w = (int)waves;
#define FL_FEW(DD)                                                                                     \
  do {                                                                                                 \
    if (format == FL_KV_I8) {                                                                          \
      if (dtype == FL_F16) paged_append_few_kernel<DD, true, true><<<few, 256, 0, st>>>(a, w);         \
      else paged_append_few_kernel<DD, true, false><<<few, 256, 0, st>>>(a, w);                        \
    } else {                                                                                           \
      if (dtype == FL_F16) paged_append_few_kernel<DD, false, true><<<few, 256, 0, st>>>(a, w);        \
      else paged_append_few_kernel<DD, false, false><<<few, 256, 0, st>>>(a, w);                       \
    }                                                                                                  \
  } while (0)
    if (d == 128) FL_FEW(128);
    else FL_FEW(64);
#undef FL_FEW
    return check_launch("paged_append_few_kernel");
  }
  // one head per workgroup until the chip is full; then more, which share a page's cosines and load one head ahead
  const int64_t pages = T / page + 2 * (int64_t)B;
  a.hp = (int)std::max<int64_t>(1, std::min<int64_t>(Hkv, pages * Hkv * 2 / 2048));
  const int64_t wgs = pages * ((Hkv + a.hp - 1) / a.hp) * 2;
  FL_REQUIRE(wgs < (1ll << 31), FL_E_SHAPE, "%s: T * Hkv too large", fn);
  const unsigned grid = (unsigned)wgs;
#define FL_APPEND(DD)                                                   \
  do {                                                                  \
    if (page == 16) launch_append<DD, 16>(a, grid, format, dtype, st);  \
    else if (page == 32) launch_append<DD, 32>(a, grid, format, dtype, st); \
    else if (page == 64) launch_append<DD, 64>(a, grid, format, dtype, st); \
    else launch_append<DD, 128>(a, grid, format, dtype, st);            \
  } while (0)
  if (d == 128) FL_APPEND(128);
  else FL_APPEND(64);
#undef FL_APPEND
  return check_launch("paged_append_kernel");
  FL_API_END
}
