// Dense attention of packed prompts.
#include "fl_simple_attn.h"

#include <algorithm>
#include <vector>

namespace fl {

struct PackedArgs {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;
  int64_t qs, ks, vs, os;
  Batch bt;                        // cu: cu_q, lens: cu_k
  Rotary rt;
  int n_pos, Tk, Hq, Hkv, G;
  float scale;
  int window, n_sink;
};

template <int D, bool F16>
struct PackedRows {
  const uint16_t *k, *v;
  int64_t ks, vs;
  __device__ __forceinline__ bool there(int) const { return true; }
  __device__ __forceinline__ float spoilt(int) const { return 0.0f; }
  __device__ __forceinline__ float key(int j, int c) const { return to_f32<F16>(k[(int64_t)j * ks + c]); }
  __device__ __forceinline__ float value(int j, int c) const { return to_f32<F16>(v[(int64_t)j * vs + c]); }
};

// a wave a row and head
template <int D, bool F16>
__global__ __launch_bounds__(256) void packed_row_kernel(PackedArgs a) {
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = (int)(w / a.Hq), h = (int)(w % a.Hq);
  if (t >= a.bt.T) return;
  const Seq s = find_seq(a.bt, t, 0, [](int c) { return c; });
  if (s.b < 0 || t >= s.r1) return;
  const int k0 = min(max(a.bt.lens[s.b], 0), a.Tk), k1 = min(max(a.bt.lens[s.b + 1], 0), a.Tk);
  const int pos = max(k1 - k0, 0) - (s.r1 - t);
  const PackedRows<D, F16> src{a.k + (int64_t)k0 * a.ks + (int64_t)(h / a.G) * D, a.v + (int64_t)k0 * a.vs + (int64_t)(h / a.G) * D, a.ks, a.vs};
  float q[D / 64];
  const bool ok = !a.rt.table || (uint32_t)pos < (uint32_t)a.n_pos;
  turned_query<D, F16>(a.q + (int64_t)t * a.qs + (int64_t)h * D, a.rt, ok ? max(pos, 0) : 0, q);
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
    if (a.rt.table) q[x] = ok || (int)(threadIdx.x & 63) + 64 * x >= a.rt.rot ? to_f32<F16>((F16 ? pack_f16x2(q[x], 0.0f) : pack_bf16x2(q[x], 0.0f)) & 0xFFFFu) : NAN;
  attend_row<D, F16>(src, q, a.scale, pos, a.window > 0 ? max(pos - a.window + 1, 0) : 0, a.n_sink,
                     a.o + (int64_t)t * a.os + (int64_t)h * D, a.lse ? a.lse + (int64_t)t * a.Hq + h : nullptr);
}

static int check_offsets(const char* fn, const char* name, const int32_t* cu, int B, int T, hipStream_t st) {
  std::vector<int32_t> c((size_t)B + 1);
  hipError_t e = hipStreamSynchronize(st);
  if (e == hipSuccess) e = hipMemcpy(c.data(), cu, c.size() * 4, hipMemcpyDeviceToHost);
  FL_REQUIRE(e == hipSuccess, FL_E_HIP, "%s: index check: copy of %s failed: %s", fn, name, hipGetErrorString(e));
  FL_REQUIRE(c[0] == 0, FL_E_RANGE, "%s: %s[0] = %d must be 0", fn, name, c[0]);
  for (int b = 0; b < B; ++b)
    FL_REQUIRE(c[b + 1] >= c[b] && c[b + 1] <= T, FL_E_RANGE, "%s: %s[%d] = %d after %d, of %d rows", fn, name, b + 1, c[b + 1], c[b], T);
  return FL_OK;
}

}  // namespace fl

using namespace fl;

extern "C" size_t fl_packed_attn_ws(int, int, int, int, int, int, int, int, int) { return 0; }

extern "C" int fl_packed_attn(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              int dtype, const int32_t* cu_q, const int32_t* cu_k, int B, int Tq, int Tk, int Hq, int Hkv, int d,
                              const float* table, int n_pos, int rot, int layout, float sm_scale, int window, int n_sink,
                              int max_k, void* o, int64_t o_stride, float* lse, void* ws, size_t ws_bytes, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_packed_attn";
  FL_REQUIRE(dtype == FL_BF16 || dtype == FL_F16, FL_E_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  FL_REQUIRE(d == 64 || d == 128, FL_E_SHAPE, "%s: d=%d must be 64 or 128", fn, d);
  FL_REQUIRE(B >= 1 && B <= 65536 && Tq >= 0 && Tk >= 0, FL_E_SHAPE, "%s: B=%d must be in [1, 65536], Tq=%d and Tk=%d >= 0", fn, B, Tq, Tk);
  FL_REQUIRE(Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 && Hq <= 65535, FL_E_SHAPE, "%s: Hq=%d must be a multiple of Hkv=%d, at most 65535",
             fn, Hq, Hkv);
  FL_REQUIRE((int64_t)Tq * Hq < (1ll << 31) && Tk <= INT_MAX - 4096, FL_E_SHAPE, "%s: Tq * Hq must be below 2^31, Tk below 2^31 - 4096", fn);
  FL_REQUIRE(cu_q && cu_k, FL_E_NULL, "%s: cu_q and cu_k are required", fn);
  int rc;
  if (table) {
    rc = check_rotary(fn, table, rot, layout, d);
    if (rc != FL_OK) return rc;
    FL_REQUIRE(n_pos >= 1, FL_E_RANGE, "%s: a table of %d positions", fn, n_pos);
  }
  FL_REQUIRE(sm_scale > 0.0f && sm_scale < INFINITY, FL_E_RANGE, "%s: sm_scale must be positive and finite", fn);
  FL_REQUIRE(window >= 0 && n_sink >= 0 && max_k >= 0, FL_E_RANGE, "%s: window, n_sink and max_k must be >= 0", fn);
  if (Tq == 0) return FL_OK;
  rc = check_rows(fn, "q", q, q_stride, Hq, d);
  if (rc == FL_OK) rc = check_rows(fn, "o", o, o_stride, Hq, d);
  if (rc == FL_OK && Tk > 0) rc = check_rows(fn, "k", k, k_stride, Hkv, d);
  if (rc == FL_OK && Tk > 0) rc = check_rows(fn, "v", v, v_stride, Hkv, d);
  if (rc != FL_OK) return rc;
  constexpr int64_t kMost = 1 << 24;
  FL_REQUIRE(q_stride <= kMost && o_stride <= kMost && (Tk == 0 || (k_stride <= kMost && v_stride <= kMost)), FL_E_SHAPE,
             "%s: row strides of at most 2^24 elements", fn);
  rc = check_disjoint(fn, "q", q, q_stride, Tq, Hq * d, "o", o, o_stride, Tq, Hq * d);
  if (rc == FL_OK && Tk > 0) rc = check_disjoint(fn, "k", k, k_stride, Tk, Hkv * d, "o", o, o_stride, Tq, Hq * d);
  if (rc == FL_OK && Tk > 0) rc = check_disjoint(fn, "v", v, v_stride, Tk, Hkv * d, "o", o, o_stride, Tq, Hq * d);
  if (rc != FL_OK) return rc;
  hipStream_t st = as_stream(stream);
  if (index_checks_on()) {
    rc = check_offsets(fn, "cu_q", cu_q, B, Tq, st);
    if (rc == FL_OK) rc = check_offsets(fn, "cu_k", cu_k, B, Tk, st);
    if (rc != FL_OK) return rc;
  }
  PackedArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.ks = k_stride; a.vs = v_stride; a.os = o_stride;
  a.bt = {cu_q, cu_k, nullptr, B, Tq, 0};
  a.rt = {table, rot, layout};
  a.n_pos = n_pos; a.Tk = Tk; a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv; a.scale = sm_scale; a.window = window; a.n_sink = n_sink;
  const unsigned grid = (unsigned)(((int64_t)Tq * Hq + 3) / 4);
  if (d == 128) {
    if (dtype == FL_F16) packed_row_kernel<128, true><<<grid, 256, 0, st>>>(a);
    else packed_row_kernel<128, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (dtype == FL_F16) packed_row_kernel<64, true><<<grid, 256, 0, st>>>(a);
    else packed_row_kernel<64, false><<<grid, 256, 0, st>>>(a);
  }
  return check_launch("packed_row_kernel");
  FL_API_END
}
