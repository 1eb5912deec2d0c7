// Dense attention of a ragged batch over the paged 8-bit cache.
#include "fl_paged.h"

namespace fl {

struct PagedAttnArgs {
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  int64_t qs, os;                  // row strides
  Batch bt;
  Rotary rt;
  Pages pg;
  const uint8_t *kc, *vc;
  const float *ksc, *vsc;
  int Hq, G;                       // query heads; of them per key/value head
  float scale_log2;                // sm_scale * log2(e)
  int window, n_sink;
};

template <bool I8>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if constexpr (I8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(w >> (8 * e));
  } else {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  }
}

// One wave per row and query head: lanes are keys for the scores, channels for the outputs.
template <int D, bool I8, bool F16>
__global__ __launch_bounds__(64) void paged_row_kernel(PagedAttnArgs a) {
  __shared__ float s_q[D], s_p[64];
  __shared__ int64_t s_at[64];
  const int lane = threadIdx.x, h = blockIdx.y, t = blockIdx.x, kvh = h / a.G;
  const int b = __builtin_amdgcn_readfirstlane(find_seq(a.bt, t, 0, [](int c) { return c; }));
  if (b < 0) return;
  const int r1 = row_of(a.bt, b + 1);
  if (t >= r1) return;
  const int64_t pos = (int64_t)a.bt.lens[b] - (r1 - t);      // the row's position
  const int last = (int)min(pos, (int64_t)a.bt.max_pages * a.pg.size - 1);
  for (int c = lane; c < D; c += 64) {
    const uint16_t* src = a.q + (int64_t)t * a.qs + (int64_t)h * D;
    float v = to_f32<F16>(src[c]);
    if (a.rt.table && c < a.rt.rot && pos >= 0 && last == pos) {
      const int half = a.rt.rot / 2;
      const bool hl = a.rt.layout == FL_ROPE_HALF;
      const int i = hl ? c % half : c / 2;
      const bool second = hl ? c >= half : (c & 1);
      const float other = to_f32<F16>(src[hl ? (second ? c - half : c + half) : c ^ 1]);
      const float2 cs = reinterpret_cast<const float2*>(a.rt.table)[pos * half + i];
      v = second ? other * cs.y + v * cs.x : v * cs.x - other * cs.y;
    }
    s_q[c] = v;
  }
  __syncthreads();
  float acc[D / 64] = {}, ref = -INFINITY, sum = 0.0f;
  for (int j0 = 0; j0 <= last; j0 += 64) {
    const int j = j0 + lane;
    bool seen = j <= last && (a.window == 0 || (int64_t)j > pos - a.window || j < a.n_sink);
    float x = -INFINITY, vs = 0.0f;
    if (seen) {
      const int pid = a.bt.table[(int64_t)b * a.bt.max_pages + (j >> a.pg.log2)];
      seen = (uint32_t)pid < (uint32_t)a.pg.num;
      if (seen) {
        const int64_t head = (int64_t)pid * a.pg.heads + kvh;
        const int64_t at = (head * a.pg.size + (j & (a.pg.size - 1))) * D;
        float dot = 0.0f;
        for (int c = 0; c < D; c += 4) {
          float k[4];
          decode4<I8>(*reinterpret_cast<const uint32_t*>(a.kc + at + c), k);
#pragma unroll
          for (int e = 0; e < 4; ++e) dot = fmaf(s_q[c + e], k[e], dot);
        }
        x = dot * (a.ksc[head] * a.scale_log2);
        vs = a.vsc[head];
        s_at[lane] = at;
      }
    }
    float top = x;
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (__builtin_amdgcn_ballot_w64(seen) == 0) continue;
    const float nref = fmaxf(ref, top);
    const float alpha = ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref - nref);
    const float p = seen ? __builtin_amdgcn_exp2f(x - nref) : 0.0f;
    ref = nref;
    sum = sum * alpha + p;
    s_p[lane] = seen ? p * vs : 0.0f;
    if (!seen) s_at[lane] = -1;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < D / 64; ++e) acc[e] *= alpha;
    for (int x2 = 0; x2 < 64; ++x2) {
      const int64_t at = s_at[x2];
      if (at < 0) continue;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const uint32_t c = a.vc[at + e * 64 + lane];
        float v[4];
        decode4<I8>(c, v);
        acc[e] = fmaf(s_p[x2], v[0], acc[e]);
      }
    }
    __syncthreads();
  }
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
  const bool none = ref == -INFINITY && sum == 0.0f;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    const float v = none ? 0.0f : acc[e] / sum;
    a.o[(int64_t)t * a.os + (int64_t)h * D + e * 64 + lane] =
        (uint16_t)((F16 ? pack_f16x2(v, 0.0f) : pack_bf16x2(v, 0.0f)) & 0xFFFFu);
  }
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.Hq + h] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace fl

using namespace fl;

extern "C" size_t fl_paged_attn_ws(int B, int T, int Hq, int Hkv, int d, int page, int max_pages, int window, int n_sink,
                                   int max_q, int max_len) {
  return 0;
}

extern "C" int fl_paged_attn(const void* q, int64_t q_stride, int dtype, const int32_t* cu, const int32_t* lens, int B, int T,
                             int Hq, int Hkv, int d, const float* table, int n_pos, int rot, int layout,
                             const int32_t* block_table, int max_pages, int num_pages, int page, int format,
                             const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                             float sm_scale, int window, int n_sink, int max_q, int max_len, void* o, int64_t o_stride,
                             float* lse, void* ws, size_t ws_bytes, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_paged_attn";
  int rc = check_paged(fn, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, block_table, max_pages, num_pages, page,
                       format, k_cache, v_cache, k_scale, v_scale);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(Hq >= Hkv && Hq % Hkv == 0 && Hq <= 65535, FL_E_SHAPE, "%s: Hq=%d must be a multiple of Hkv=%d, at most 65535", fn,
             Hq, Hkv);
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
  PagedAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.os = o_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<const uint8_t*>(k_cache); a.vc = static_cast<const uint8_t*>(v_cache); a.ksc = k_scale; a.vsc = v_scale;
  a.Hq = Hq; a.G = Hq / Hkv; a.scale_log2 = sm_scale * 1.4426950408889634f; a.window = window; a.n_sink = n_sink;
  rc = check_batch(fn, a.bt, a.pg, false, st);
  if (rc != FL_OK) return rc;
  const dim3 grid((unsigned)T, (unsigned)Hq);
#define FL_ROW(DD)                                                                                   \
  do {                                                                                               \
    if (format == FL_KV_I8) {                                                                        \
      if (dtype == FL_F16) paged_row_kernel<DD, true, true><<<grid, 64, 0, st>>>(a);                 \
      else paged_row_kernel<DD, true, false><<<grid, 64, 0, st>>>(a);                                \
    } else {                                                                                         \
      if (dtype == FL_F16) paged_row_kernel<DD, false, true><<<grid, 64, 0, st>>>(a);                \
      else paged_row_kernel<DD, false, false><<<grid, 64, 0, st>>>(a);                               \
    }                                                                                                \
  } while (0)
  if (d == 128) FL_ROW(128);
  else FL_ROW(64);
#undef FL_ROW
  return check_launch("paged_row_kernel");
  FL_API_END
}
