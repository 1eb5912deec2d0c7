// Dense attention over the paged 4-bit cache for many rows per sequence (prompts and their chunks): a source of the prompt kernel.
// The codes of a stage are loaded while earlier ones are multiplied, widened to fp16 in registers beside the products and written to LDS
// once for the workgroup's 128 rows: 13 instructions for eight int4 codes, 4 for eight e2m1 ones, about a third of a stage's vector
// instructions for int4.  What bounds it: the vector units and the matrix cores in turn (chunks of 1009, 512 and 2000 of 32 / 8 heads x
// 128 with a window of 8192: busy for 60 and 38 % of the cycles; 490 us with plan and join; 8192 positions of 16 heads int4 367 us, e2m1
// 317, and 285 over bf16 rows).
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
// LOW: fp16 queries that are rotated, in two parts.
template <int D, bool INT, bool F16, bool LOW>
struct Paged4Source {
  // fp16 outputs of int4 codes: keys and probabilities in two parts, as for few rows; the keys' second parts double their stages in LDS
  static constexpr bool kTwo = INT && F16;
  static constexpr int kD = D, kWavesPerSimd = kTwo && D == 128 ? 1 : 2;    // (64 channels, 8192 positions of 16 heads: 231 us with 2, 236 with 3)
  using KTile = StageTile<D, kTwo ? 2 : 1>;
  static __device__ __forceinline__ uint32_t rest(float p0, float p1, uint32_t rounded) { return pack_rest(p0, p1, rounded); }
  static constexpr bool kF16 = true, kOut16 = F16, kLow = LOW, kMixed = INT;
  static constexpr int NW = D / 32, NG = D / kGroup, MB = meta_bytes<INT>();      // words of a thread, groups of a head

  const Paged4Args& a;
  const Span& sp;
  int b, kvh, t0, n, wave, lane;
  int pid[2];                                // the wave's page of stage 64 i + lane, by the parity of i
  uint64_t hole[2];                          // stages with a page that is not there
  uint32_t kw[NW], vw[NW], km, kmv, vm, place;
  Magic magic;

  __device__ __forceinline__ Paged4Source(const Paged4Args& args, const Seq& sq, const Span& span, int head, int tid, int first, int stages)
      : a(args), sp(span), b(sq.b), kvh(head), t0(first), n(stages), wave(__builtin_amdgcn_readfirstlane(tid >> 6)), lane(tid & 63) {
    place = place_of();
    km = kmv = vm = 0;
#pragma unroll
    for (int e = 0; e < NW; ++e) kw[e] = vw[e] = 0;
    pid[0] = pid[1] = -1;
    hole[0] = hole[1] = 0;
    pages(0);
  }
  __device__ __forceinline__ void pages(int block) {
    const int st = 64 * block + lane;
    bool gone = false;
    int own = -1;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      int p = 0;
      if (st < n) {
        const int page = (key_of<kStageKeys>(sp, t0 + st) + 16 * g) >> a.pg.log2;
        p = page < a.bt.max_pages ? a.bt.table[(int64_t)b * a.bt.max_pages + page] : -1;
      }
      const bool none = (uint32_t)p >= (uint32_t)a.pg.num;
      gone |= none;
      own = g == wave ? (none ? -1 : p) : own;
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(gone);
    pid[0] = block & 1 ? pid[0] : own;
    pid[1] = block & 1 ? own : pid[1];
    hole[0] = block & 1 ? hole[0] : m;
    hole[1] = block & 1 ? m : hole[1];
  }
  // (half way through a block the next one's, of 64 stages; waited for at once)
  __device__ __forceinline__ void ahead(int st) {
    if ((st & 63) == 32) pages((st >> 6) + 1);
  }
  __device__ __forceinline__ bool holes(int st) const {
    const uint64_t even = hole[0], odd = hole[1];
    return ((st & 64 ? odd : even) >> (st & 63)) & 1;
  }
  __device__ __forceinline__ uint32_t there(int st) const {  // a bit for 16 keys
    uint32_t bits = 15;
    if (holes(st)) {                         // uniform
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int page = (key_of<kStageKeys>(sp, t0 + st) + 16 * g) >> a.pg.log2;
        const bool here = page < a.bt.max_pages && (uint32_t)a.bt.table[(int64_t)b * a.bt.max_pages + page] < (uint32_t)a.pg.num;
        bits &= ~((here ? 0u : 1u) << g);
      }
    }
    return bits;
  }
  // row of the wave's 16 keys of a stage (a page that is not there: any other's, masked)
  __device__ __forceinline__ int64_t row_of_stage(int st) const {
    const int even = pid[0], odd = pid[1];
    const int p = max(__builtin_amdgcn_readlane(st & 64 ? odd : even, st & 63), 0);
    return ((int64_t)p * a.pg.heads + kvh) * a.pg.size + ((key_of<kStageKeys>(sp, t0 + st) + 16 * wave) & (a.pg.size - 1));
  }
  // (the lane's offset is formed anew beside a uniform address: added to it ahead of the stages, the sums spilled)
  __device__ __forceinline__ void codes(const uint8_t* at, uint32_t* w) const {
    int l = lane;
    renew(l);
    if constexpr (NW == 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(at + (uint32_t)(16 * l));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = x[e];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(at + (uint32_t)(8 * l));
      w[0] = x[0];
      w[1] = x[1];
    }
  }
  __device__ __forceinline__ uint32_t number(const uint8_t* m, int64_t row) const {
    int l = lane;
    renew(l);
    return load_meta<INT>(m + row * (NG * MB) + (uint32_t)((D == 128 ? l : l >> 1) * MB));
  }
  __device__ __forceinline__ void load_k(int st, KTile&) {
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
  // Word e of the thread's keys or values widened into its place.  Neighbouring threads write their words in different orders (e ^ turn),
  // so that 16 of them meet 16 different 16-byte groups of banks.
  __device__ __forceinline__ void place_words(uint32_t* w) const {
    const int turn = D == 128 ? lane >> 2 & 3 : lane >> 3 & 1;         // (of the thread's key)
#pragma unroll
    for (int bit = 1; bit < NW; bit *= 2)
#pragma unroll
      for (int e = 0; e < NW; ++e)
        if (!(e & bit)) {
          const uint32_t x = w[e], y = w[e | bit];
          w[e] = turn & bit ? y : x;
          w[e | bit] = turn & bit ? x : y;
        }
  }
  __device__ __forceinline__ uint32_t place_of() const {
    const int key = 16 * wave + (lane >> 2), turn = D == 128 ? lane >> 2 & 3 : lane >> 3 & 1;
    return (uint32_t)(key * D + ((((lane & 3) * NW) ^ turn ^ swz32_f<D>(key & 31)) * 8));
  }
  __device__ __forceinline__ void put_k(KTile& t, uint32_t w, uint32_t bad, int e) const {
    uint16_t* at = t.x + (place ^ (uint32_t)(8 * e));
    u32x4 x, low;
    if constexpr (kTwo) {
      widen8_two(w, km, magic, x, low);
      *reinterpret_cast<u32x4*>(at + kStageKeys * D) = low;
    } else {
      x = widen8<INT>(w, km, magic);
    }
    x[0] |= bad;
    *reinterpret_cast<u32x4*>(at) = x;
  }
  // The work of a stage beside its products: its loads, widened into their buffers, a word a time.  A group that reads as NaN, of the
  // key or the value, makes the key's scores NaN; the value's counts as 0.
  static constexpr int kItems = 2 * NW;
  __device__ __forceinline__ void item_k(int i, KTile& k) {
    if (i == 0) place_words(kw);
    put_k(k, kw[i], i == 0 && !(group_ok<INT>(km) & group_ok<INT>(kmv)) ? 0x7E007E00u : 0u, i);
  }
  __device__ __forceinline__ void item_v(int i, StageTile<D>& v) {
    if (i == 0) {
      place_words(vw);
      vm = group_ok<INT>(vm) ? vm : 0u;
    }
    *reinterpret_cast<u32x4*>(v.x + (place ^ (uint32_t)(8 * i))) = widen8<INT>(vw[i], vm, magic);
  }
  __device__ __forceinline__ void item(int i, KTile& k, StageTile<D>& v) {
    if (i < NW) item_k(i, k);
    else item_v(i - NW, v);
  }
  __device__ __forceinline__ void land_k(KTile& k) {
#pragma unroll
    for (int i = 0; i < NW; ++i) item_k(i, k);
  }
  __device__ __forceinline__ void begin(KTile& k0, KTile&, StageTile<D>& v0) {
    load_k(0, k0);
    load_v(0, v0);
  }
  __device__ __forceinline__ void finish(KTile& k0, KTile& k1, StageTile<D>& v0) {
    land_k(k0);
    if (n > 1) load_k(1, k1);
#pragma unroll
    for (int i = 0; i < NW; ++i) item_v(i, v0);
    if (n > 1) land_k(k1);
  }
  __device__ __forceinline__ void land() const {}
  static constexpr bool kOdd = false;        // (values are finite)
  static __device__ __forceinline__ int wave_of(int) { return 0; }
  __device__ __forceinline__ bool odd(StageTile<D>&, uint32_t*) const { return false; }
  __device__ __forceinline__ float query(const Paged4Args& args, int t, int head, int pos, bool ok, int hw, u32x4* q, u32x4* low) const {
    constexpr int KS = D / 16;
    f16x8 x[KS], y[F16 ? KS : 1];
    float m = load_query<KS, F16>(args, args.q + (int64_t)t * args.qs + (int64_t)head * D, ok, pos, args.bt.max_pages * args.pg.size, x, y,
                                  [hw](int k) { return 2 * k + hw; }, [](float v) { return xor32_max(v); });
    m = finite_factor<KS>(m, x);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      q[k] = __builtin_bit_cast(u32x4, in_order<INT>(x[k]));
      if constexpr (LOW) low[k] = __builtin_bit_cast(u32x4, in_order<INT>(y[k]));
    }
    return m;
  }
};

// (the compiler emits the launching side of one of the two forms alone unless both are named)
#define FL_FORMS(D, I, F16, LOW)                                                                           \
  template __global__ void prompt_kernel<Paged4Source<D, I, F16, LOW>, Paged4Args, true>(Paged4Args);      \
  template __global__ void prompt_kernel<Paged4Source<D, I, F16, LOW>, Paged4Args, false>(Paged4Args);
#define FL_FORMS_OF(D)            \
  FL_FORMS(D, true, false, false)  \
  FL_FORMS(D, true, true, false)   \
  FL_FORMS(D, true, true, true)    \
  FL_FORMS(D, false, false, false) \
  FL_FORMS(D, false, true, false)  \
  FL_FORMS(D, false, true, true)
FL_FORMS_OF(128)
FL_FORMS_OF(64)
#undef FL_FORMS_OF
#undef FL_FORMS

size_t paged4_prompt_ws(const PromptShape& s, int d) { return prompt_ws(s, d); }

template <int D, bool INT>
static int launch_prompt4(Paged4Args& a, bool f16, const PromptShape& shape, hipStream_t st) {
  const char* fn = "fl_paged4_attn";
  if (!f16) return launch_prompt<Paged4Source<D, INT, false, false>, D, false>(a, fn, shape, st);
  if (a.rt.table) return launch_prompt<Paged4Source<D, INT, true, true>, D, true>(a, fn, shape, st);
  return launch_prompt<Paged4Source<D, INT, true, false>, D, true>(a, fn, shape, st);
}
int launch_paged4_prompt(const Paged4Args& args, int d, int format, bool f16, const PromptShape& shape, hipStream_t st) {
  Paged4Args a = args;
  if (d == 128) return format == FL_KV4_INT ? launch_prompt4<128, true>(a, f16, shape, st) : launch_prompt4<128, false>(a, f16, shape, st);
  return format == FL_KV4_INT ? launch_prompt4<64, true>(a, f16, shape, st) : launch_prompt4<64, false>(a, f16, shape, st);
}

}  // namespace fl
