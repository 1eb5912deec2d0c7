// Dense attention over the paged 4-bit cache for many rows per sequence (prompts and their chunks): a source of the prompt kernel.
// The codes of a stage are loaded while earlier ones are multiplied, widened to fp16 in registers and written to LDS once for the
// workgroup's 128 rows.
#include "fl_paged4_attn.h"
#include "fl_prompt.h"

namespace fl {

__device__ __forceinline__ Seq seq_of(const Paged4Args& a, int b) { return {b, row_of(a.bt, b), row_of(a.bt, b + 1), a.bt.lens[b]}; }
template <int R>
__device__ __forceinline__ Seq find_row_tile(const Paged4Args& a, int slot) {
  const int G = a.G;
  return find_seq(a.bt, slot, 1, [G](int c) { return (int)((int64_t)c * G / R); });
}

// A thread has a quarter of a key (and of a value) of each stage, which is of one group; a wave has 16 keys, which are of one page.
template <int D, bool INT, bool F16>
struct Paged4Source {
  static constexpr int kD = D;
  static constexpr bool kF16 = true, kOut16 = F16, kLow = F16, kMixed = INT;
  static constexpr int NW = D / 32, NG = D / kGroup, MB = meta_bytes<INT>();      // words of a thread, groups of a head

  const Paged4Args& a;
  const Span& sp;
  int b, kvh, t0, n, wave, lane;
  int pid[2];                                // the wave's page of stage 64 i + lane, by the parity of i
  uint64_t hole[2];                          // stages with a page that is not there
  int next[4];
  uint32_t kw[NW], vw[NW], km, kmv, vm;

  __device__ __forceinline__ Paged4Source(const Paged4Args& args, const Seq& sq, const Span& span, int head, int tid, int first, int stages)
      : a(args), sp(span), b(sq.b), kvh(head), t0(first), n(stages), wave(__builtin_amdgcn_readfirstlane(tid >> 6)), lane(tid & 63) {
    pages(0);
    use_pages(0);
    pid[1] = -1;
    hole[1] = 0;
  }
  __device__ __forceinline__ void pages(int block) {
    const int st = 64 * block + lane;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      next[g] = 0;
      if (st < n) {
        const int page = (key_of<kStageKeys>(sp, t0 + st) + 16 * g) >> a.pg.log2;
        next[g] = page < a.bt.max_pages ? a.bt.table[(int64_t)b * a.bt.max_pages + page] : -1;
      }
    }
  }
  __device__ __forceinline__ void use_pages(int block) {
    bool gone = false;
    int own = -1;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const bool none = (uint32_t)next[g] >= (uint32_t)a.pg.num;
      gone |= none;
      own = g == wave ? (none ? -1 : next[g]) : own;
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(gone);
    if (block & 1) {
      pid[1] = own;
      hole[1] = m;
    } else {
      pid[0] = own;
      hole[0] = m;
    }
  }
  __device__ __forceinline__ void ahead(int st) {
    if ((st & 63) == 0) pages((st >> 6) + 1);
    if ((st & 63) == 32) use_pages((st >> 6) + 1);
  }
  __device__ __forceinline__ bool holes(int st) const { return ((st & 64 ? hole[1] : hole[0]) >> (st & 63)) & 1; }
  __device__ __forceinline__ bool there(int st, int g) const {
    if (!holes(st)) return true;
    const int page = (key_of<kStageKeys>(sp, t0 + st) + 16 * g) >> a.pg.log2;
    return page < a.bt.max_pages && (uint32_t)a.bt.table[(int64_t)b * a.bt.max_pages + page] < (uint32_t)a.pg.num;
  }
  // row of the wave's 16 keys of a stage (a page that is not there: any other's, masked)
  __device__ __forceinline__ int64_t row_of_stage(int st) const {
    const int p = max(__builtin_amdgcn_readlane(st & 64 ? pid[1] : pid[0], st & 63), 0);
    return ((int64_t)p * a.pg.heads + kvh) * a.pg.size + ((key_of<kStageKeys>(sp, t0 + st) + 16 * wave) & (a.pg.size - 1));
  }
  __device__ __forceinline__ void codes(const uint8_t* at, uint32_t* w) const {
    if constexpr (NW == 4) {
      const u32x4 x = reinterpret_cast<const u32x4*>(at)[lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = x[e];
    } else {
      const u32x2 x = reinterpret_cast<const u32x2*>(at)[lane];
      w[0] = x[0];
      w[1] = x[1];
    }
  }
  __device__ __forceinline__ uint32_t number(const uint8_t* m, int64_t row) const {
    return load_meta<INT>(m + row * (NG * MB) + (uint32_t)(D == 128 ? lane : lane >> 1) * MB);
  }
  __device__ __forceinline__ void load_k(int st, StageTile<D>&) {
    const int64_t row = row_of_stage(st);
    codes(a.kc + row * (D / 2), kw);
    km = number(a.km, row);
    kmv = number(a.vm, row);
  }
  __device__ __forceinline__ void load_v(int st, StageTile<D>&) {
    const int64_t row = row_of_stage(st);
    codes(a.vc + row * (D / 2), vw);
    vm = number(a.vm, row);
  }
  __device__ __forceinline__ void put(StageTile<D>& t, const uint32_t* w, uint32_t meta, uint32_t bad) const {
    const int key = 16 * wave + (lane >> 2), g = swz32_f<D>(key & 31);
#pragma unroll
    for (int e = 0; e < NW; ++e) {
      u32x4 x = widen8<INT>(w[e], meta);
      if (e == 0) x[0] |= bad;
      *reinterpret_cast<u32x4*>(t.x + key * D + (((lane & 3) * NW + e) ^ g) * 8) = x;
    }
  }
  // a group that reads as NaN, of the key or the value, makes the key's scores NaN; the value's counts as 0
  __device__ __forceinline__ void land_k(StageTile<D>& t) const {
    put(t, kw, km, group_ok<INT>(km) & group_ok<INT>(kmv) ? 0u : 0x7E007E00u);
  }
  __device__ __forceinline__ void land(bool with_k, StageTile<D>& k, StageTile<D>& v) {
    if (with_k) land_k(k);
    if (!group_ok<INT>(vm)) {
      vm = 0;
#pragma unroll
      for (int e = 0; e < NW; ++e) vw[e] = 0;
    }
    put(v, vw, vm, 0);
  }
  static constexpr bool kOdd = false;        // (values are finite)
  __device__ __forceinline__ bool odd(StageTile<D>&, uint32_t*) const { return false; }
  __device__ __forceinline__ float query(const Paged4Args& args, int t, int head, int pos, bool ok, int hw, u32x4* q, u32x4* low) const {
    constexpr int KS = D / 16;
    f16x8 x[KS], y[F16 ? KS : 1];
    float m = load_query<KS, F16>(args, args.q + (int64_t)t * args.qs + (int64_t)head * D, ok, pos, args.bt.max_pages * args.pg.size, x, y,
                                  [hw](int k) { return 2 * k + hw; }, [](float v) { return xor32_max(v); });
    const bool none = !(m == m);             // a query that is not finite: NaN scores, and not the -inf of what it does not see
    m = none ? 1.0f : m;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      q[k] = __builtin_bit_cast(u32x4, in_order<INT>(x[k]));
      if constexpr (F16) low[k] = __builtin_bit_cast(u32x4, in_order<INT>(y[k]));
      if (none) q[k] = u32x4{0x7E007E00u, 0x7E007E00u, 0x7E007E00u, 0x7E007E00u};
    }
    return m;
  }
};

#define FL_FORMS(D, I, F16)                                                                           \
  template __global__ void prompt_kernel<Paged4Source<D, I, F16>, Paged4Args, true>(Paged4Args);      \
  template __global__ void prompt_kernel<Paged4Source<D, I, F16>, Paged4Args, false>(Paged4Args);
FL_FORMS(128, true, true)
FL_FORMS(128, true, false)
FL_FORMS(128, false, true)
FL_FORMS(128, false, false)
FL_FORMS(64, true, true)
FL_FORMS(64, true, false)
FL_FORMS(64, false, true)
FL_FORMS(64, false, false)
#undef FL_FORMS

size_t paged4_prompt_ws(int64_t slots, int Hkv, int d, int64_t cap, int64_t keys) { return prompt_ws(slots, Hkv, d, cap, keys); }

template <int D, bool INT, bool F16>
static int launch_prompt4(Paged4Args& a, int64_t keys, hipStream_t st) {
  return launch_prompt<Paged4Source<D, INT, F16>, D, F16>(a, "fl_paged4_attn", (int64_t)a.bt.max_pages * a.pg.size, keys, st);
}
int launch_paged4_prompt(const Paged4Args& args, int d, int format, bool f16, int64_t keys, hipStream_t st) {
  Paged4Args a = args;
  const bool i = format == FL_KV4_INT;
  if (d == 128) {
    if (i) return f16 ? launch_prompt4<128, true, true>(a, keys, st) : launch_prompt4<128, true, false>(a, keys, st);
    return f16 ? launch_prompt4<128, false, true>(a, keys, st) : launch_prompt4<128, false, false>(a, keys, st);
  }
  if (i) return f16 ? launch_prompt4<64, true, true>(a, keys, st) : launch_prompt4<64, true, false>(a, keys, st);
  return f16 ? launch_prompt4<64, false, true>(a, keys, st) : launch_prompt4<64, false, false>(a, keys, st);
}

}  // namespace fl
