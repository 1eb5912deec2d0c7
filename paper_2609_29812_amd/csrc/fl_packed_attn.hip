// Dense attention of packed prompts: keys and values as rows in memory, for the kernel of many rows per sequence.
#include "fl_prompt.h"

#include <vector>

namespace fl {

struct PackedArgs : PagedAttnArgs {          // bt: cu = cu_q, lens = cu_k, one "page" of any length; pg.heads
  const uint16_t *k, *v;
  int64_t ks, vs;
  int Tk, n_pos;
};
__device__ __forceinline__ int key_row(const PackedArgs& a, int b) { return min(max(a.bt.lens[b], 0), a.Tk); }
// (lens[b] is the first key row: the length is that of the key rows)
__device__ __forceinline__ Seq seq_of(const PackedArgs& a, int b) {
  return {b, row_of(a.bt, b), row_of(a.bt, b + 1), max(key_row(a, b + 1) - key_row(a, b), 0)};
}
template <int R>
__device__ __forceinline__ Seq find_row_tile(const PackedArgs& a, int slot) {
  const int G = a.G;
  Seq s = find_seq(a.bt, slot, 1, [G](int c) { return (int)((int64_t)c * G / R); });
  if (s.b >= 0) s.len = max(key_row(a, s.b + 1) - key_row(a, s.b), 0);
  return s;
}

// Stages of 64 key and value rows by LDS-DMA, 16 bytes a lane, with the permutation of a row's chunks on the way (no bank conflicts);
// rows behind the sequence's last read zeros.  A key that a row does not see cannot reach it: its score is replaced.  A value can, as 0
// times an infinity: in stages that some row does not see in full, values that are not finite are set to 0 and noted, and what does see
// them gets NaN.
template <int D, bool F16>
struct PackedSource {
  using Args = PackedArgs;
  // (64 channels, 8192 positions of 16 heads: 186 us with two waves a SIMD, 173 with three; 128 channels need 250 registers)
  static constexpr int kD = D, kWavesPerSimd = D == 64 ? 3 : 2;
  static constexpr bool kF16 = F16, kOut16 = F16, kLow = false, kMixed = false, kOdd = true, kTwo = false;
  // Chunks of a row, rows of a load, loads of a wave, rows from one of these to the next: a lane's chunk is permuted alike in all.
  static constexpr int CH = D / 8, RPI = 64 / CH, NI = kStageKeys / RPI / 4, ROWS = 4 * RPI;

  const Args& a;
  const Span& sp;
  const uint16_t *k, *v;                     // row 0 of the sequence, the head's channels
  int n_k, t0, n, wave, lane;
  uint32_t kofs, vofs;                       // of the lane's chunk in a wave's first load (the others: ROWS rows on)

  __device__ __forceinline__ PackedSource(const Args& args, const Seq& sq, const Span& span, int kvh, int tid, int first, int stages)
      : a(args), sp(span), n_k(sq.len), t0(first), n(stages), wave(__builtin_amdgcn_readfirstlane(tid >> 6)), lane(tid & 63) {
    const int row0 = key_row(a, sq.b);
    k = a.k + (int64_t)row0 * a.ks + kvh * D;
    v = a.v + (int64_t)row0 * a.vs + kvh * D;
    const int c = wave * RPI + lane / CH;
    const uint32_t chunk = (uint32_t)((lane % CH) ^ swz32_f<D>(c)) * 16u;
    kofs = (uint32_t)c * (uint32_t)(2 * a.ks) + chunk;
    vofs = (uint32_t)c * (uint32_t)(2 * a.vs) + chunk;
  }
  // (offsets stay below 64 rows of at most 2^25 bytes)
  __device__ __forceinline__ void load(const uint16_t* rows, int64_t stride, uint32_t ofs, int key0, StageTile<D>& t) const {
    const int left = n_k - key0;
    const uint32_t step = ROWS * (uint32_t)(2 * stride);
    if (left >= kStageKeys) {                // uniform
      const rsrc_t r = make_rsrc(rows + key0 * stride, 0x7FFFFFFFu);
#pragma unroll
      for (int x = 0; x < NI; ++x)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, FL_LDS(t.x + (x * ROWS + wave * RPI) * D), 16, ofs, x * step, 0, 0);
    } else {
      const rsrc_t r = make_rsrc(rows + key0 * stride, left > 0 ? (uint32_t)(left - 1) * (uint32_t)(2 * stride) + 2u * D : 0u);
#pragma unroll
      for (int x = 0; x < NI; ++x)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, FL_LDS(t.x + (x * ROWS + wave * RPI) * D), 16, ofs + x * step, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void load_k(int st, StageTile<D>& t) { load(k, a.ks, kofs, key_of<kStageKeys>(sp, t0 + st), t); }
  __device__ __forceinline__ void load_v(int st, StageTile<D>& t) { load(v, a.vs, vofs, key_of<kStageKeys>(sp, t0 + st), t); }
  static constexpr int kItems = 0;
  __device__ __forceinline__ void item(int, StageTile<D>&, StageTile<D>&) const {}
  __device__ __forceinline__ void land() const { FL_WAIT_VM(0); }
  __device__ __forceinline__ void begin(StageTile<D>& k0, StageTile<D>& k1, StageTile<D>& v0) {
    load_k(0, k0);
    load_v(0, v0);
    if (n > 1) load_k(1, k1);
  }
  __device__ __forceinline__ void finish(StageTile<D>&, StageTile<D>&, StageTile<D>&) const { land(); }
  // The values that the wave's loads have brought: whether some of this lane's are not finite (those become 0), and which (`where` is
  // written if the wave has some).
  static __device__ __forceinline__ int wave_of(int key) { return key / RPI & 3; }
  __device__ __forceinline__ bool odd(StageTile<D>& t, uint32_t* where) const {
    constexpr uint32_t kExp = F16 ? 0x7C00u : 0x7F80u;
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    int l = lane;
    renew(l);                                // (places in LDS are formed anew: kept over the stages, they spilled)
    u32x4* at = reinterpret_cast<u32x4*>(t.x + wave * RPI * D + l * 8);
    u16x2 most = {0, 0};
#pragma unroll
    for (int x = 0; x < NI; ++x) {
      const u32x4 w = at[x * (ROWS * D / 8)];
#pragma unroll
      for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[e] & (kExp | kExp << 16)));
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(most[0] == kExp || most[1] == kExp) == 0, 1)) return false;      // uniform
    const int c = wave * RPI + l / CH;
    uint8_t* mark = reinterpret_cast<uint8_t*>(where) + c * CH + ((l % CH) ^ swz32_f<D>(c));
    bool any = false;
#pragma nounroll
    for (int x = 0; x < NI; ++x) {
      u32x4 w = *at;
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = (w[e] & kExp) == kExp, hi = (w[e] & (kExp << 16)) == (kExp << 16);
        bits |= (lo ? 1u : 0u) << (2 * e) | (hi ? 2u : 0u) << (2 * e);
        w[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
      }
      *mark = (uint8_t)bits;
      if (bits != 0) *at = w;
      any |= bits != 0;
      at += ROWS * D / 8;
      mark += ROWS * CH;
    }
    return any;
  }
  __device__ __forceinline__ void ahead(int) const {}
  __device__ __forceinline__ bool holes(int) const { return false; }
  __device__ __forceinline__ uint32_t there(int) const { return 15; }
  __device__ __forceinline__ float query(const Args& args, int t, int head, int pos, bool ok, int hw, u32x4* q, u32x4*) const {
    constexpr int KS = D / 16;
    const uint16_t* row = args.q + (int64_t)t * args.qs + (int64_t)head * D;
    if (!args.rt.table) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 w = reinterpret_cast<const u32x4*>(row)[2 * ks + hw];
        q[ks] = ok ? w : u32x4{};
      }
    } else {
      const bool in = (uint32_t)pos < (uint32_t)args.n_pos;
      float x[KS][8];
      turned_chunks<KS, F16, true>(args.rt, row, in ? pos : 0, x, [hw](int ks) { return 2 * ks + hw; });
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bool none = !in && 8 * (2 * ks + hw) < args.rt.rot;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = pack2<F16>(none ? NAN : x[ks][2 * e], none ? NAN : x[ks][2 * e + 1]);
          q[ks][e] = ok ? w : 0u;
        }
      }
    }
    return args.scale_log2;
  }
};

// (the compiler emits the launching side of one of the two forms alone unless both are named)
#define FL_FORMS(D, F16)                                                                      \
  template __global__ void prompt_kernel<PackedSource<D, F16>, PackedArgs, true>(PackedArgs); \
  template __global__ void prompt_kernel<PackedSource<D, F16>, PackedArgs, false>(PackedArgs);
FL_FORMS(128, true)
FL_FORMS(128, false)
FL_FORMS(64, true)
FL_FORMS(64, false)
#undef FL_FORMS

static PromptShape packed_shape(int B, int Tq, int Tk, int Hq, int Hkv, int window, int n_sink, int max_k) {
  int64_t keys = max_k > 0 ? std::min(max_k, Tk) : ((int64_t)Tk + B - 1) / B;
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + n_sink + kRowsOfTile);
  return {B, Tq, Hq / Hkv, Hkv, std::max(0, Tk - Tq) / B, keys, Tk};
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

extern "C" size_t fl_packed_attn_ws(int B, int Tq, int Tk, int Hq, int Hkv, int d, int window, int n_sink, int max_k) {
  if (B < 1 || Tq < 1 || Tk < 0 || Hkv < 1 || Hq < Hkv || Hq % Hkv || (d != 64 && d != 128) || window < 0 || n_sink < 0 || max_k < 0)
    return 0;
  return prompt_ws(packed_shape(B, Tq, Tk, Hq, Hkv, window, n_sink, max_k), d);
}

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
  const PromptShape shape = packed_shape(B, Tq, Tk, Hq, Hkv, window, n_sink, max_k);
  const size_t need = prompt_ws(shape, d);
  FL_REQUIRE(need == 0 || (ws && ws_bytes >= need), FL_E_WORKSPACE, "%s: workspace of %zu bytes required", fn, need);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 15) == 0, FL_E_SHAPE, "%s: ws must be 16-byte aligned", fn);
  PackedArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.ks = k_stride; a.vs = v_stride; a.os = o_stride;
  a.bt = {cu_q, cu_k, nullptr, B, Tq, INT_MAX - 4096};
  a.rt = {table, rot, layout};
  a.pg = {0, 1, 0, Hkv};
  a.n_pos = n_pos; a.Tk = Tk; a.Hq = Hq; a.G = Hq / Hkv; a.scale_log2 = sm_scale * 1.4426950408889634f;
  a.window = window; a.n_sink = n_sink;
  a.part = static_cast<float*>(ws);
  if (d == 128)
    return dtype == FL_F16 ? launch_prompt<PackedSource<128, true>, 128, true>(a, fn, shape, st)
                           : launch_prompt<PackedSource<128, false>, 128, false>(a, fn, shape, st);
  return dtype == FL_F16 ? launch_prompt<PackedSource<64, true>, 64, true>(a, fn, shape, st)
                         : launch_prompt<PackedSource<64, false>, 64, false>(a, fn, shape, st);
  FL_API_END
}
