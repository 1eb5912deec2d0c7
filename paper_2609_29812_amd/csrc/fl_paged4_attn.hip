// Dense attention of a ragged batch over the paged 4-bit cache.
#include "fl_simple_attn.h"

namespace fl {

struct Paged4Args {
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  int64_t qs, os;
  Batch bt;
  Rotary rt;
  Pages pg;
  const uint8_t *kc, *vc, *km, *vm;
  int Hq, G;
  float scale;
  int window, n_sink;
};

template <int D, bool INT>
struct PagedRows {
  const Paged4Args& a;
  int64_t table;
  int head;
  __device__ __forceinline__ int64_t row(int j) const {
    const int p = a.bt.table[table + (j >> a.pg.log2)];
    return (uint32_t)p < (uint32_t)a.pg.num ? ((int64_t)p * a.pg.heads + head) * a.pg.size + (j & (a.pg.size - 1)) : -1;
  }
  __device__ __forceinline__ bool there(int j) const { return row(j) >= 0; }
  __device__ __forceinline__ float spoilt(int j) const {
    bool ok = true;
    for (int g = 0; g < D / kGroup; ++g) {
      const int64_t at = (row(j) * (D / kGroup) + g) * meta_bytes<INT>();
      ok &= group_ok<INT>(load_meta<INT>(a.km + at)) && group_ok<INT>(load_meta<INT>(a.vm + at));
    }
    return ok ? 0.0f : NAN;
  }
  __device__ __forceinline__ float one(const uint8_t* codes, const uint8_t* meta, int j, int c) const {
    const int64_t r = row(j);
    float x[8];
    values8<INT>(reinterpret_cast<const uint32_t*>(codes + r * (D / 2))[c / 8],
                 load_meta<INT>(meta + (r * (D / kGroup) + c / kGroup) * meta_bytes<INT>()), x);
    float y = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) y = (c & 7) == e ? x[e] : y;
    return y;
  }
  __device__ __forceinline__ float key(int j, int c) const { return one(a.kc, a.km, j, c); }
  __device__ __forceinline__ float value(int j, int c) const { return one(a.vc, a.vm, j, c); }
};

// a wave a row and head
template <int D, bool INT, bool F16>
__global__ __launch_bounds__(256) void paged4_row_kernel(Paged4Args a) {
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = (int)(w / a.Hq), h = (int)(w % a.Hq);
  if (t >= a.bt.T) return;
  const Seq s = find_seq(a.bt, t, 0, [](int c) { return c; });
  if (s.b < 0 || t >= s.r1) return;
  const int cap = a.bt.max_pages * a.pg.size;
  const int pos = max(s.len, 0) - (s.r1 - t);
  const PagedRows<D, INT> src{a, (int64_t)s.b * a.bt.max_pages, h / a.G};
  float q[D / 64];
  turned_query<D, F16>(a.q + (int64_t)t * a.qs + (int64_t)h * D, a.rt, min(max(pos, 0), cap - 1), q);
  attend_row<D, F16>(src, q, a.scale, min(pos, cap - 1), a.window > 0 ? max(pos - a.window + 1, 0) : 0, a.n_sink,
                     a.o + (int64_t)t * a.os + (int64_t)h * D, a.lse ? a.lse + (int64_t)t * a.Hq + h : nullptr);
}

}  // namespace fl

using namespace fl;

extern "C" size_t fl_paged4_attn_ws(int, int, int, int, int, int, int, int, int, int, int) { return 0; }

extern "C" int fl_paged4_attn(const void* q, int64_t q_stride, int dtype, const int32_t* cu, const int32_t* lens, int B, int T,
                              int Hq, int Hkv, int d, const float* table, int n_pos, int rot, int layout,
                              const int32_t* block_table, int max_pages, int num_pages, int page, int format,
                              const void* k_cache, const void* v_cache, const void* k_meta, const void* v_meta, float sm_scale,
                              int window, int n_sink, int max_q, int max_len, void* o, int64_t o_stride, float* lse, void* ws,
                              size_t ws_bytes, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_paged4_attn";
  int rc = check_paged4(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page,
                        format, k_cache, v_cache, k_meta, v_meta);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(Hq >= Hkv && Hq % Hkv == 0 && Hq <= 65535, FL_E_SHAPE, "%s: Hq=%d must be a multiple of Hkv=%d, at most 65535", fn,
             Hq, Hkv);
  FL_REQUIRE((int64_t)T * Hq < (1ll << 31), FL_E_SHAPE, "%s: T * Hq must be below 2^31", fn);
  FL_REQUIRE(sm_scale > 0.0f && sm_scale < INFINITY, FL_E_RANGE, "%s: sm_scale must be positive and finite", fn);
  FL_REQUIRE(window >= 0 && n_sink >= 0, FL_E_RANGE, "%s: window and n_sink must be >= 0", fn);
  FL_REQUIRE(max_q >= 0 && max_len >= 0, FL_E_RANGE, "%s: max_q and max_len must be >= 0", fn);
  if (T == 0) return FL_OK;
  rc = check_rows(fn, "q", q, q_stride, Hq, d);
  if (rc != FL_OK) return rc;
  rc = check_rows(fn, "o", o, o_stride, Hq, d);
  if (rc != FL_OK) return rc;
  rc = check_apart(fn, "q", q, q_stride, "o", o, o_stride, T, Hq * d);
  if (rc != FL_OK) return rc;
  hipStream_t st = as_stream(stream);
  Paged4Args a{};
  a.q = static_cast<const uint16_t*>(q); a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.os = o_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<const uint8_t*>(k_cache); a.vc = static_cast<const uint8_t*>(v_cache);
  a.km = static_cast<const uint8_t*>(k_meta); a.vm = static_cast<const uint8_t*>(v_meta);
  a.Hq = Hq; a.G = Hq / Hkv; a.scale = sm_scale; a.window = window; a.n_sink = n_sink;
  rc = check_batch(fn, a.bt, a.pg, false, st);
  if (rc != FL_OK) return rc;
  const unsigned grid = (unsigned)(((int64_t)T * Hq + 3) / 4);
#define FL_ROW(DD)                                                                       \
  do {                                                                                   \
    if (format == FL_KV4_INT) {                                                          \
      if (dtype == FL_F16) paged4_row_kernel<DD, true, true><<<grid, 256, 0, st>>>(a);   \
      else paged4_row_kernel<DD, true, false><<<grid, 256, 0, st>>>(a);                  \
    } else {                                                                             \
      if (dtype == FL_F16) paged4_row_kernel<DD, false, true><<<grid, 256, 0, st>>>(a);  \
      else paged4_row_kernel<DD, false, false><<<grid, 256, 0, st>>>(a);                 \
    }                                                                                    \
  } while (0)
  if (d == 128) FL_ROW(128);
  else FL_ROW(64);
#undef FL_ROW
  return check_launch("paged4_row_kernel");
  FL_API_END
}
