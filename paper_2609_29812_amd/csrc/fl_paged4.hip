// The paged 4-bit cache: appending (rotation of the keys, groups of 32 channels with numbers of their own) and reading back.
#include "fl_paged4.h"

#include <algorithm>

namespace fl {

int check_paged4(const char* fn, int dtype, const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d,
                 const float* table, int n_pos, int rot, int layout, const int32_t* block_table, int max_pages,
                 int num_pages, int page, int format, const void* kc, const void* vc, const void* km, const void* vm) {
  FL_REQUIRE(format == FL_KV4_INT || format == FL_KV4_E2M1, FL_E_UNSUPPORTED, "%s: unknown cache format %d", fn, format);
  const int rc = check_ragged(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(kc && vc && km && vm, FL_E_NULL, "%s: k_cache, v_cache, k_meta and v_meta are required", fn);
  FL_REQUIRE(kc != vc && km != vm, FL_E_SHAPE, "%s: keys and values need a cache and groups' numbers each", fn);
  FL_REQUIRE(((reinterpret_cast<uintptr_t>(kc) | reinterpret_cast<uintptr_t>(vc) | reinterpret_cast<uintptr_t>(km) |
               reinterpret_cast<uintptr_t>(vm)) & 15) == 0, FL_E_SHAPE, "%s: the caches and the groups' numbers must be 16-byte aligned",
             fn);
  return FL_OK;
}

struct Rows4Args {
  const uint16_t *k, *v;           // append: the new rows
  int64_t ks, vs;
  Batch bt;
  Rotary rt;
  Pages pg;
  uint8_t *kc, *vc, *km, *vm;
  uint16_t *kr, *vr;               // the rows that the codes stand for, or nullptr
  int64_t krs, vrs;
};

// A wave has a row of the batch; a lane has a chunk of eight channels of a head, so that the four lanes of a quad have a group.
// The heads of the keys and then those of the values are taken 512 / d at a time.  Each position stands by itself, so nothing is read
// but the new rows, and rows need no order.
// What bounds it: appending int4, the vector units (32768 rows of 8 heads x 128 with rotation and rows out: busy for 99 % of the
// cycles, 71 us at 4.5 TB/s; a copy has 4.9); reading back, memory (32768 rows 35 us, 5.0 TB/s); one row a sequence, the launch (5.5 and
// 3.3 us).
struct RowPlace {
  int pos;                         // position, or -1: the row belongs to no sequence
  int64_t at;                      // row of [num_pages, Hkv, page] of its head 0; -1: its page is not there
};
__device__ __forceinline__ RowPlace place_of_row(const Rows4Args& a, int t) {
  const Seq s = find_seq(a.bt, t, 0, [](int c) { return c; });
  if (s.b < 0 || t >= s.r1) return {-1, -1};
  const int64_t pos = (int64_t)s.len - (s.r1 - t);
  RowPlace w{(int)max(pos, (int64_t)0), -1};
  const int64_t pi = pos >> a.pg.log2;
  if (pos < 0 || pi >= a.bt.max_pages) return w;
  const int pid = a.bt.table[(int64_t)s.b * a.bt.max_pages + pi];
  if ((uint32_t)pid < (uint32_t)a.pg.num) w.at = (int64_t)pid * a.pg.heads * a.pg.size + (pos & (a.pg.size - 1));
  return w;
}

template <int CTRL>
__device__ __forceinline__ float quad(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, quad<0xB1>(x));                     // lanes 1 0 3 2
  return fmaxf(x, quad<0x4E>(x));                  // lanes 2 3 0 1
}

// x rounded to fp16 towards zero
__device__ __forceinline__ uint32_t f16_rtz(float x) {
  return (uint32_t)__builtin_bit_cast(uint16_t, __builtin_amdgcn_cvt_pkrtz(x, 0.0f)[0]);
}

// The codes of a lane's eight values x (a word) and the group's numbers (every lane of the quad has them); x becomes what the codes
// stand for.
template <bool INT>
__device__ __forceinline__ uint32_t encode_group(float* x, uint32_t& meta) {
  float lo = x[0], hi = x[0], bad = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (INT) lo = fminf(lo, x[e]);
    hi = INT ? fmaxf(hi, x[e]) : fmaxf(fabsf(hi), fabsf(x[e]));
    bad = fmaf(x[e], 0.0f, bad);                   // NaN with an infinity or a NaN
  }
  if constexpr (INT) lo = -quad_max(-lo);
  hi = quad_max(hi);
  bad = quad_max(bad == 0.0f ? 0.0f : 1.0f);
  if (bad > 0.0f) {
    meta = INT ? kNaN4 : 255u;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = NAN;
    return 0;
  }
  if (hi > 32768.0f || (INT && lo < -32768.0f)) {
    lo = fminf(fmaxf(lo, -32768.0f), 32768.0f);
    hi = fminf(fmaxf(hi, -32768.0f), 32768.0f);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fminf(fmaxf(x[e], -32768.0f), 32768.0f);
  }
  if constexpr (INT) {
    uint32_t zb = f16_rtz(lo);
    zb += f16_bits_to_f32(zb) > lo ? 1u : 0u;      // (towards zero is upwards below it)
    zb = zb == 0x8000u ? 0u : zb;
    const float z = f16_bits_to_f32(zb);
    // the smallest s with 15 s >= max - z: at most two steps above what a quotient that is a little too small gives
    const double range = fabs((double)hi - (double)z);      // (not -0)
    uint32_t sb = f16_rtz((float)range * (0.99999988f / 15.0f));
#pragma unroll
    for (int e = 0; e < 2; ++e) sb += 15.0 * (double)f16_bits_to_f32(sb) < range ? 1u : 0u;
    meta = sb | zb << 16;
    if (sb == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = z;
      return 0;
    }
    const float s = f16_bits_to_f32(sb), inv = __builtin_amdgcn_rcpf(s);
    // The product with the reciprocal is within 2^-18 of the quotient, and that in [0, 15]; next to a half the definition's own
    // steps decide.
    float r[8], off = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float q = (x[e] - z) * inv;
      r[e] = rintf(q);
      off = fmaxf(off, fabsf(q - r[e]));
    }
    if (off > 0.4999f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = (float)fmin(fmax(rint(((double)x[e] - (double)z) / (double)s), 0.0), 15.0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(s, r[e], z);
    const float w0 = fmaf(fmaf(fmaf(r[3], 16.0f, r[2]), 16.0f, r[1]), 16.0f, r[0]);
    const float w1 = fmaf(fmaf(fmaf(r[7], 16.0f, r[6]), 16.0f, r[5]), 16.0f, r[4]);
    return (uint32_t)w0 | (uint32_t)w1 << 16;
  } else {
    // hi = m 2^k with m in [1, 2): within 6 2^e = 1.5 2^(e + 2) from e = k - 2 on, or k - 1 when m > 1.5
    const uint32_t bits = __float_as_uint(hi);
    const int e = max((int)(bits >> 23) - 127 - 2 + ((bits & 0x7FFFFFu) > 0x400000u ? 1 : 0), kMinExp4);
    meta = (uint32_t)(e + 127);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * down, x[1] * down, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * down, x[3] * down, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * down, x[5] * down, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * down, x[7] * down, 1.0f, 3);
    values8<false>(w, meta, x);
    return w;
  }
}

// What a wave's lanes do at step s0 of a row's 2 Hkv heads: the lane's head, and where its row and its cached position begin.  EVEN: the
// wave's heads are all keys' or all values' (a whole number of steps each), so that all but the lane's offset is uniform (32768 rows of 8
// heads x 128: appending without rotation 54 us so, 61 in the general form, reading back 35 and 36.6).
template <int D, bool EVEN>
struct HeadOf {
  bool is_k, there;
  int h;
  __device__ __forceinline__ HeadOf(int s0, int sub, int heads) {
    const int s = EVEN ? s0 : s0 + sub;
    is_k = s < heads;
    h = (is_k ? s : s - heads) + (EVEN ? sub : 0);
    there = EVEN || s < 2 * heads;
  }
};

template <int D, bool INT, bool F16, bool EVEN>
__global__ __launch_bounds__(256) void paged4_append_kernel(Rows4Args a) {
  constexpr int CH = D / 8, HPW = 64 / CH;         // chunks of a head; heads of a wave at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * 4 + wave;
  if (t >= a.bt.T) return;
  const int c = lane % CH, sub = lane / CH;
  const int half = a.rt.table ? a.rt.rot / 16 : 0;                    // chunks of half the rotated part
  const bool turn = c < 2 * half, apart = a.rt.layout == FL_ROPE_HALF;
  const int mate = !turn || !apart ? c : c < half ? c + half : c - half;
  // a step's values are asked for one step ahead, the first before the row's place is known
  uint4 own = make_uint4(0, 0, 0, 0), other = own;
  auto load = [&](int s0) {
    const HeadOf<D, EVEN> o(s0, sub, a.pg.heads);
    if (s0 >= 2 * a.pg.heads || !o.there) return;
    const uint16_t* src = o.is_k ? a.k + (int64_t)t * a.ks : a.v + (int64_t)t * a.vs;
    own = *reinterpret_cast<const uint4*>(src + (uint32_t)(o.h * D + c * 8));
    if (o.is_k && apart && half > 0) other = *reinterpret_cast<const uint4*>(src + (uint32_t)(o.h * D + mate * 8));
  };
  load(0);
  const RowPlace w = place_of_row(a, t);
  if (w.at < 0) return;
  float cs[16];                                                       // cosines and sines of the chunk's pairs
#pragma unroll
  for (int e = 0; e < 16; ++e) cs[e] = 0.0f;
  if (turn) {
    const float4* row = reinterpret_cast<const float4*>(a.rt.table + (int64_t)w.pos * a.rt.rot + (apart ? 16 * min(c, mate) : 8 * c));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < 2 || apart) {
        const float4 f = row[e];
        cs[4 * e] = f.x; cs[4 * e + 1] = f.y; cs[4 * e + 2] = f.z; cs[4 * e + 3] = f.w;
      }
  }
  for (int s0 = 0; s0 < 2 * a.pg.heads; s0 += HPW) {
    const HeadOf<D, EVEN> o(s0, sub, a.pg.heads);
    if (!o.there) break;
    const uint32_t in_row = (uint32_t)(o.h * D + c * 8);
    const uint4 raw = own, raw2 = other;
    load(s0 + HPW);
    float x[8];
    unpack8<F16>(raw, x);
    if (o.is_k && turn) {
      // the products of 8- or 11-bit values with fp32 ones are exact in fp64: one rounding, by the sum, then fp32
      if (apart) {
        float y[8];
        unpack8<F16>(raw2, y);
        const double sign = c < half ? -1.0 : 1.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)fma((double)x[e], (double)cs[2 * e], sign * (double)y[e] * (double)cs[2 * e + 1]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double p = x[2 * e], q = x[2 * e + 1], co = cs[2 * e], si = cs[2 * e + 1];
          x[2 * e] = (float)fma(p, co, -(q * si));
          x[2 * e + 1] = (float)fma(p, si, q * co);
        }
      }
    }
    uint32_t meta;
    const uint32_t codes = encode_group<INT>(x, meta);
    const int64_t row0 = (w.at + (int64_t)(EVEN ? o.h - sub : 0) * a.pg.size) * (D / 2);      // bytes
    const uint32_t at = (uint32_t)(EVEN ? sub : o.h) * (uint32_t)a.pg.size;
    *reinterpret_cast<uint32_t*>((o.is_k ? a.kc : a.vc) + row0 + at * (D / 2) + c * 4) = codes;
    if ((c & 3) == 0) {
      constexpr int MB = meta_bytes<INT>(), NG = D / kGroup;
      uint8_t* m = (o.is_k ? a.km : a.vm) + row0 / (D / 2) * (NG * MB) + (at * NG + (uint32_t)(c / 4)) * MB;
      if constexpr (INT) *reinterpret_cast<uint32_t*>(m) = meta;
      else *m = (uint8_t)meta;
    }
    uint16_t* out = o.is_k ? a.kr : a.vr;
    if (out) *reinterpret_cast<uint4*>(out + (int64_t)t * (o.is_k ? a.krs : a.vrs) + in_row) = pack8<F16>(x);
  }
}

template <int D, bool INT, bool F16, bool EVEN>
__global__ __launch_bounds__(256) void paged4_read_kernel(Rows4Args a) {
  constexpr int CH = D / 8, HPW = 64 / CH, MB = meta_bytes<INT>(), NG = D / kGroup;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * 4 + wave;
  if (t >= a.bt.T) return;
  const RowPlace w = place_of_row(a, t);
  if (w.pos < 0) return;
  const int c = lane % CH, sub = lane / CH;
  for (int s0 = 0; s0 < 2 * a.pg.heads; s0 += HPW) {
    const HeadOf<D, EVEN> o(s0, sub, a.pg.heads);
    if (!o.there) break;
    uint16_t* out = o.is_k ? a.kr : a.vr;
    if (!out) continue;
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (w.at >= 0) {
      const int64_t row0 = (w.at + (int64_t)(EVEN ? o.h - sub : 0) * a.pg.size) * (D / 2);
      const uint32_t at = (uint32_t)(EVEN ? sub : o.h) * (uint32_t)a.pg.size;
      const uint32_t codes = *reinterpret_cast<const uint32_t*>((o.is_k ? a.kc : a.vc) + row0 + at * (D / 2) + c * 4);
      const uint32_t meta = load_meta<INT>((o.is_k ? a.km : a.vm) + row0 / (D / 2) * (NG * MB) + (at * NG + (uint32_t)(c / 4)) * MB);
      values8<INT>(codes, meta, x);
    }
    *reinterpret_cast<uint4*>(out + (int64_t)t * (o.is_k ? a.krs : a.vrs) + (uint32_t)(o.h * D + c * 8)) = pack8<F16>(x);
  }
}

template <int D, bool EVEN>
static void launch_append4(const Rows4Args& a, unsigned grid, int format, int dtype, hipStream_t st) {
  if (format == FL_KV4_INT) {
    if (dtype == FL_F16) paged4_append_kernel<D, true, true, EVEN><<<grid, 256, 0, st>>>(a);
    else paged4_append_kernel<D, true, false, EVEN><<<grid, 256, 0, st>>>(a);
  } else {
    if (dtype == FL_F16) paged4_append_kernel<D, false, true, EVEN><<<grid, 256, 0, st>>>(a);
    else paged4_append_kernel<D, false, false, EVEN><<<grid, 256, 0, st>>>(a);
  }
}
template <int D, bool EVEN>
static void launch_read4(const Rows4Args& a, unsigned grid, int format, int dtype, hipStream_t st) {
  if (format == FL_KV4_INT) {
    if (dtype == FL_F16) paged4_read_kernel<D, true, true, EVEN><<<grid, 256, 0, st>>>(a);
    else paged4_read_kernel<D, true, false, EVEN><<<grid, 256, 0, st>>>(a);
  } else {
    if (dtype == FL_F16) paged4_read_kernel<D, false, true, EVEN><<<grid, 256, 0, st>>>(a);
    else paged4_read_kernel<D, false, false, EVEN><<<grid, 256, 0, st>>>(a);
  }
}

}  // namespace fl

using namespace fl;

extern "C" int fl_paged4_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype, const int32_t* cu,
                                const int32_t* lens, int B, int T, int Hkv, int d, const float* table, int n_pos, int rot,
                                int layout, const int32_t* block_table, int max_pages, int num_pages, int page, int format,
                                void* k_cache, void* v_cache, void* k_meta, void* v_meta, void* k_rows, int64_t k_rows_stride,
                                void* v_rows, int64_t v_rows_stride, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_paged4_append";
  int rc = check_paged4(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page,
                        format, k_cache, v_cache, k_meta, v_meta);
  if (rc != FL_OK) return rc;
  if (T == 0) return FL_OK;
  struct Side {
    const char* name;
    const void* x;
    int64_t stride;
  };
  const Side in[2] = {{"k", k, k_stride}, {"v", v, v_stride}}, out[2] = {{"k_rows", k_rows, k_rows_stride}, {"v_rows", v_rows, v_rows_stride}};
  for (const Side& s : in) {
    rc = check_rows(fn, s.name, s.x, s.stride, Hkv, d);
    if (rc != FL_OK) return rc;
  }
  for (int o = 0; o < 2; ++o) {
    if (!out[o].x) continue;
    rc = check_rows(fn, out[o].name, out[o].x, out[o].stride, Hkv, d);
    for (int i = 0; i < 2 && rc == FL_OK; ++i)
      if (i != o || in[i].x != out[o].x || in[i].stride != out[o].stride)
        rc = check_apart(fn, out[o].name, out[o].x, out[o].stride, in[i].name, in[i].x, in[i].stride, T, Hkv * d);
    if (rc != FL_OK) return rc;
  }
  if (k_rows && v_rows) {
    rc = check_apart(fn, "k_rows", k_rows, k_rows_stride, "v_rows", v_rows, v_rows_stride, T, Hkv * d);
    if (rc != FL_OK) return rc;
  }
  hipStream_t st = as_stream(stream);
  Rows4Args a{};
  a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v); a.ks = k_stride; a.vs = v_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<uint8_t*>(k_cache); a.vc = static_cast<uint8_t*>(v_cache);
  a.km = static_cast<uint8_t*>(k_meta); a.vm = static_cast<uint8_t*>(v_meta);
  a.kr = static_cast<uint16_t*>(k_rows); a.vr = static_cast<uint16_t*>(v_rows); a.krs = k_rows_stride; a.vrs = v_rows_stride;
  rc = check_batch(fn, a.bt, a.pg, true, st);
  if (rc != FL_OK) return rc;
  const unsigned grid = ((unsigned)T + 3) / 4;
  const bool even = Hkv * d % 512 == 0;      // (a wave takes 512 channels at a time)
  if (d == 128) even ? launch_append4<128, true>(a, grid, format, dtype, st) : launch_append4<128, false>(a, grid, format, dtype, st);
  else even ? launch_append4<64, true>(a, grid, format, dtype, st) : launch_append4<64, false>(a, grid, format, dtype, st);
  return check_launch("paged4_append_kernel");
  FL_API_END
}

extern "C" int fl_paged4_read(const int32_t* cu, const int32_t* lens, int B, int T, int Hkv, int d, const int32_t* block_table,
                              int max_pages, int num_pages, int page, int format, const void* k_cache, const void* v_cache,
                              const void* k_meta, const void* v_meta, int dtype, void* k_out, int64_t k_out_stride, void* v_out,
                              int64_t v_out_stride, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_paged4_read";
  int rc = check_paged4(fn, dtype, cu, lens, B, T, Hkv, d, nullptr, 0, 0, 0, block_table, max_pages, num_pages, page, format,
                        k_cache, v_cache, k_meta, v_meta);
  if (rc != FL_OK) return rc;
  if (T == 0) return FL_OK;
  FL_REQUIRE(k_out || v_out, FL_E_NULL, "%s: k_out and v_out are NULL", fn);
  if (k_out) rc = check_rows(fn, "k_out", k_out, k_out_stride, Hkv, d);
  if (rc == FL_OK && v_out) rc = check_rows(fn, "v_out", v_out, v_out_stride, Hkv, d);
  if (rc == FL_OK && k_out && v_out) rc = check_apart(fn, "k_out", k_out, k_out_stride, "v_out", v_out, v_out_stride, T, Hkv * d);
  if (rc != FL_OK) return rc;
  hipStream_t st = as_stream(stream);
  Rows4Args a{};
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<uint8_t*>(const_cast<void*>(k_cache)); a.vc = static_cast<uint8_t*>(const_cast<void*>(v_cache));
  a.km = static_cast<uint8_t*>(const_cast<void*>(k_meta)); a.vm = static_cast<uint8_t*>(const_cast<void*>(v_meta));
  a.kr = static_cast<uint16_t*>(k_out); a.vr = static_cast<uint16_t*>(v_out); a.krs = k_out_stride; a.vrs = v_out_stride;
  rc = check_batch(fn, a.bt, a.pg, false, st);
  if (rc != FL_OK) return rc;
  const unsigned grid = ((unsigned)T + 3) / 4;
  const bool even = Hkv * d % 512 == 0;      // (a wave takes 512 channels at a time)
  if (d == 128) even ? launch_read4<128, true>(a, grid, format, dtype, st) : launch_read4<128, false>(a, grid, format, dtype, st);
  else even ? launch_read4<64, true>(a, grid, format, dtype, st) : launch_read4<64, false>(a, grid, format, dtype, st);
  return check_launch("paged4_read_kernel");
  FL_API_END
}
