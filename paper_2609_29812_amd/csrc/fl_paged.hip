// Appending to the paged key/value cache: rotation of the keys, 8-bit codes with one scale per page and head, and the
// requantization of a page whose scale grows.
#include "fl_paged.h"

#include <algorithm>
#include <vector>

namespace fl {

int check_paged(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                int num_pages, int page, int format, const void* kc, const void* vc, const float* ks, const float* vs) {
  FL_REQUIRE(dtype == FL_BF16 || dtype == FL_F16, FL_E_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  FL_REQUIRE(format == FL_KV_I8 || format == FL_KV_E4M3, FL_E_UNSUPPORTED, "%s: unknown cache format %d", fn, format);
  FL_REQUIRE(d == 64 || d == 128, FL_E_SHAPE, "%s: d=%d must be 64 or 128", fn, d);
  FL_REQUIRE(page == 16 || page == 32 || page == 64 || page == 128, FL_E_SHAPE, "%s: page=%d must be 16, 32, 64 or 128", fn,
             page);
  FL_REQUIRE(B >= 1 && B <= 65536 && T >= 0, FL_E_SHAPE, "%s: B=%d must be in [1, 65536] and T=%d >= 0", fn, B, T);
  FL_REQUIRE(Hkv >= 1 && Hkv <= 65535, FL_E_SHAPE, "%s: Hkv=%d must be in [1, 65535]", fn, Hkv);
  FL_REQUIRE(max_pages >= 1 && (int64_t)max_pages * page <= INT_MAX - 4096, FL_E_SHAPE,
             "%s: max_pages=%d pages of %d positions: between 1 page and 2^31 - 4097 positions", fn, max_pages, page);
  FL_REQUIRE(num_pages >= 1, FL_E_SHAPE, "%s: num_pages=%d must be positive", fn, num_pages);
  FL_REQUIRE(cu && lens && block_table, FL_E_NULL, "%s: cu, lens and block_table are required", fn);
  FL_REQUIRE(kc && vc && ks && vs, FL_E_NULL, "%s: k_cache, v_cache, k_scale and v_scale are required", fn);
  FL_REQUIRE(kc != vc && ks != vs, FL_E_SHAPE, "%s: keys and values need a cache and scales each", fn);
  FL_REQUIRE(((reinterpret_cast<uintptr_t>(kc) | reinterpret_cast<uintptr_t>(vc)) & 15) == 0, FL_E_SHAPE,
             "%s: the caches must be 16-byte aligned", fn);
  if (table) {
    const int rc = check_rotary(fn, table, rot, layout, d);
    if (rc != FL_OK) return rc;
    FL_REQUIRE((int64_t)n_pos >= (int64_t)max_pages * page, FL_E_RANGE,
               "%s: a table of %d positions for sequences of up to %d pages of %d", fn, n_pos, max_pages, page);
  }
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

// A workgroup has one page that receives positions, keys or values, and hp heads one after the other.  A sequence with n new
// positions touches at most n / page + 2 pages, so slots cu[b] / page + 2 b .. belong to sequence b (the grid covers
// T / page + 2 B).  A thread holds 16 channels of a position per pass, both values of every pair that it rotates, with the
// cosines and sines in registers for all heads; the largest magnitude meets through LDS, then the codes go out.
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
  const Seq sq = find_seq(a.bt, slot, 2, [](int c) { return c >> LOG2; });
  const int b = sq.b, r0 = sq.r0, n = sq.r1 - sq.r0, len = sq.len;
  if (b < 0) return;
  if (n <= 0 || len <= 0) return;
  const int start = max(len - n, 0);                         // first stored position; (len - n < 0: the first are dropped)
  const int64_t pi = (int64_t)(start >> LOG2) + (slot - ((r0 >> LOG2) + 2 * b));
  if (pi >= a.bt.max_pages) return;
  const int p0 = (int)pi << LOG2;
  const int lo = max(start, p0) - p0, hi = min(len - p0, PAGE);
  if (lo >= hi) return;
  const int pid = a.bt.table[(int64_t)b * a.bt.max_pages + pi];
  if ((uint32_t)pid >= (uint32_t)a.pg.num) return;
  const uint16_t* src = is_k ? a.k : a.v;
  const int64_t stride = is_k ? a.ks : a.vs;
  const int u = threadIdx.x % TPP, i0 = threadIdx.x / TPP;
  const int turned = is_k && a.rt.table ? a.rt.rot / 16 : 0;  // units that rotate, as in the rotation of dense rows
  const bool half = a.rt.layout == FL_ROPE_HALF;
  const bool turn = u < turned;
  const int c0 = half && turn ? u : 2 * u, c1 = half && turn ? u + turned : 2 * u + 1;
  const bool mixed = !half && turned > 0;                    // pairs lie side by side: drawn apart while a thread holds them
  float cs[NP][16];
#pragma unroll
  for (int s = 0; s < NP; ++s) {
    const int i = s * PER + i0;
    if (turn && i >= lo && i < hi) {
      const float4* row = reinterpret_cast<const float4*>(a.rt.table + (int64_t)(p0 + i) * a.rt.rot + u * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 w = row[e];
        cs[s][4 * e] = w.x; cs[s][4 * e + 1] = w.y; cs[s][4 * e + 2] = w.z; cs[s][4 * e + 3] = w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) cs[s][e] = 0.0f;
    }
  }
  const int h0 = part % hg * a.hp, h1 = min(h0 + a.hp, a.pg.heads);
  uint4 raw[NP][2];                                           // the next head's values
  auto load = [&](int h) {
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      const int i = s * PER + i0;
      raw[s][0] = raw[s][1] = make_uint4(0, 0, 0, 0);
      if (i >= lo && i < hi) {
        const uint16_t* at = src + ((int64_t)r0 + (p0 + i) - (len - n)) * stride + (int64_t)h * D;
        raw[s][0] = *reinterpret_cast<const uint4*>(at + c0 * 8);
        raw[s][1] = *reinterpret_cast<const uint4*>(at + c1 * 8);
      }
    }
  };
  load(h0);
  for (int h = h0; h < h1; ++h) {
    const int64_t head = (int64_t)pid * a.pg.heads + h;
    uint8_t* codes = (is_k ? a.kc : a.vc) + head * (PAGE * D);
    float* scale = (is_k ? a.ksc : a.vsc) + head;
    const float held = *scale;
    float x[NP][16];
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      uint4 w0 = raw[s][0], w1 = raw[s][1];
      if (mixed) {
        const uint4 a0 = w0, a1 = w1;
        w0 = make_uint4(low16(a0.x, a0.y), low16(a0.z, a0.w), low16(a1.x, a1.y), low16(a1.z, a1.w));
        w1 = make_uint4(high16(a0.x, a0.y), high16(a0.z, a0.w), high16(a1.x, a1.y), high16(a1.z, a1.w));
      }
      unpack8<F16>(w0, x[s]);
      unpack8<F16>(w1, x[s] + 8);
      if (turn) {
        // the products of 8- or 11-bit values with fp32 ones are exact in fp64: one rounding, by the sum, then fp32
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double p = x[s][e], q = x[s][e + 8], c = cs[s][2 * e], sn = cs[s][2 * e + 1];
          x[s][e] = (float)fma(p, c, -(q * sn));
          x[s][e + 8] = (float)fma(p, sn, q * c);
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(x[s][e]) & 0x7FFFFFFFu);   // (NaN above inf above finite)
    }
    if (h + 1 < h1) load(h + 1);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, 64));
    uint32_t* room = s_max[h & 1];                            // (the last head's may still be read)
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) most = max(most, room[w]);
    const float need = scale_for<I8>(most);
    float sc = need;
    int k = 0;
    if (lo > 0 && held != 0.0f) {                             // earlier positions of the sequence are in the page
      if (isnan(need) || !isfinite(held)) {
        sc = NAN;
      } else {
        k = doublings(held, need);
        sc = ldexpf(held, k);
      }
    }
    if (k > 0) {
      const float f = ldexpf(1.0f, -k);
#pragma unroll
      for (int s = 0; s < NP; ++s) {
        const int i = s * PER + i0;
        if (i >= lo && i < hi) continue;
        uint2* at = reinterpret_cast<uint2*>(codes + i * D);
        at[c0] = shrink8<I8>(at[c0], f);
        at[c1] = shrink8<I8>(at[c1], f);
      }
    }
    const bool zero = !(sc > 0.0f);                           // (NaN too)
    const float inv = zero ? 0.0f : 1.0f / sc;
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      const int i = s * PER + i0;
      if (i < lo || i >= hi) continue;
      uint2* at = reinterpret_cast<uint2*>(codes + i * D);
      uint2 y0 = make_uint2(0, 0), y1 = y0;
      if (!zero) {
        y0 = encode8<I8>(x[s], sc, inv);
        y1 = encode8<I8>(x[s] + 8, sc, inv);
      }
      if (mixed) {
        const uint2 p = y0, q = y1;
        y0 = make_uint2(__builtin_amdgcn_perm(q.x, p.x, 0x05010400u), __builtin_amdgcn_perm(q.x, p.x, 0x07030602u));
        y1 = make_uint2(__builtin_amdgcn_perm(q.y, p.y, 0x05010400u), __builtin_amdgcn_perm(q.y, p.y, 0x07030602u));
      }
      at[c0] = y0;
      at[c1] = y1;
    }
    if (threadIdx.x == 0) *scale = sc;
  }
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
