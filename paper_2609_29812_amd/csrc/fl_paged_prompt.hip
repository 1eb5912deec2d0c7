// Dense attention over the paged 8-bit cache for many rows per sequence: prompts and their chunks.
//
// A workgroup of 4 waves takes 128 rows (positions x query heads of one key/value head), 32 per wave, over stages of 64 keys.
// The codes of the next stage are loaded while this one is multiplied, widened to exact fp16 in registers and written to the
// other of two LDS buffers: one barrier a stage, each code widened once for 128 rows.
//   S^T = K Q^T     v_mfma_f32_32x32x16_f16, K rows as the A operand, so a lane holds 16 keys of one row per block;
//   O^T += V^T P^T  the same product, V read transposed (ds_read_b64_tr_b16), P rounded to fp16.
// Scales never touch the codes: a key scale multiplies its 16 scores inside the exponent's fma, a value scale enters as its
// logarithm there and leaves the row sum as its reciprocal, once per 16 keys.
//
// Bound by neither unit alone: vector instructions are issued in 56 % of the cycles and the matrix cores are busy in 41 %, one after
// the other, for a stage multiplies and then takes its scores through the exponent.  Per wave and stage 32 products (1024 matrix
// cycles; 48 with fp16 queries that are rotated) against about 360 vector instructions and 33 exponentials; 16 heads x 128, 16384
// positions 1.29 ms (850 TFLOP/s), where the dense loop over bf16 states, which widens no codes, takes 1.16.
//
// One workgroup for each row tile and head, the longest first, from two rounds of them on.  Fewer leave the chip idle, so there
// workgroups have equal shares of the work, whatever the lengths are: a first small kernel adds up the units of all row tiles,
// each of the 512 / Hkv workgroups of a key/value head takes an equal run of them, and row tiles that a border cuts are joined at
// the end from the sides' sums.  (1024 positions after 16000, 16 heads: 523 us without shares, 219 with; a whole prompt of 8192,
// 1040 workgroups: 411 without, 491 with.)
#include "fl_paged_attn.h"

#include <algorithm>

namespace fl {

// ends[s]: units of row tiles 0 .. s
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedAttnArgs a) {
  __shared__ int s_sum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  for (int s0 = 0; s0 < a.slots; s0 += 1024) {
    const int slot = s0 + threadIdx.x;
    int n = 0;
    if (slot < a.slots) {
      int lo = 0, hi = a.bt.B;                                // the last sequence whose first slot is at most this one
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (row_of(a.bt, mid) * a.G / kPromptRows + mid <= slot) lo = mid;
        else hi = mid;
      }
      const Seq q{lo, row_of(a.bt, lo), row_of(a.bt, lo + 1), a.bt.lens[lo]};
      const Span sp = span_of<kPromptRows, kPromptKeys>(a, q, slot - (q.r0 * a.G / kPromptRows + lo));
      n = sp.rows > 0 ? kTileUnits + max(sp.tiles, 1) : 0;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int x = __shfl_up(n, off, 64);
      n += lane >= off ? x : 0;
    }
    if (lane == 63) s_sum[wave] = n;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) n += s_sum[w];
      all += s_sum[w];
    }
    if (slot < a.slots) a.ends[slot] = before + n;
    before += all;
    __syncthreads();
  }
}

// first row tile whose end is beyond unit x (the wave looks at 64 places at a time)
__device__ __forceinline__ int tile_of_unit(const int* ends, int slots, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = slots;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = min(lo + (lane + 1) * step, lo + n) - 1;
    const uint64_t m = __builtin_amdgcn_ballot_w64(ends[at] > x);
    const int l = m ? __builtin_ctzll(m) : 63;
    const int next = min(lo + l * step, lo + n - 1);
    n = min(step, lo + n - next);
    lo = next;
  }
  return lo;
}

constexpr int kAhead = 32;                 // stages whose pages and scales are in LDS at a time

template <int D>
struct __attribute__((aligned(16))) PromptSlot {
  uint16_t k[kPromptKeys * D];             // blocks of 32 rows, 16-byte chunks permuted (swz32_f), fp16
  uint16_t v[kPromptKeys * D];
};

template <int D, bool I8, bool F16, bool SHARED>
__global__ __launch_bounds__(256, 2) void paged_prompt_kernel(PagedAttnArgs a) {
  constexpr int R = kPromptRows, COLS = kPromptKeys;
  constexpr int NBK = COLS / 32;           // 32-key blocks
  constexpr int KS = D / 16;               // k-steps of QK^T
  constexpr int DB = D / 32;               // 32-channel output blocks
  constexpr int LPK = D / 16;              // lanes (16 codes each) per key
  constexpr int NI = COLS * LPK / 256;     // loads of a thread, tensor and stage
  __shared__ PromptSlot<D> s0, s1;
  __shared__ float4 s_page[2][4 * kAhead]; // per 16 keys: key scale, log2 and reciprocal of the value scale, page

  const int kvh = blockIdx.x % a.pg.heads, wg = blockIdx.x / a.pg.heads;
  const int G = a.G;
  // the workgroup's run of units at .. end - 1 of its head, from row tile `slot` on; or all of one row tile
  int at = 0, end = 1, slot = gridDim.x / a.pg.heads - 1 - wg;          // (later rows see more keys: first)
  if constexpr (SHARED) {
    const Cut cut = cut_of(a);
    at = cut.begin(wg);
    end = cut.begin(wg + 1);
    if (at >= end) return;
    slot = tile_of_unit(a.ends, a.slots, at);
  }
  const int first = at;
  for (; at < end; ++slot) {
  int tid = threadIdx.x;
  // what a row tile derives from the lane is formed anew: kept over the stages, it spilled (128 channels with fp16 queries still
  // hold 3 to 9 registers of a lane in scratch, all but one of them read outside the stages)
  if constexpr (SHARED) asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = lane >> 5, r32 = lane & 31;
  const Seq sq = find_seq(a.bt, slot, 1, [G](int c) { return c * G / R; });
  const int b = sq.b;
  if (b < 0) return;
  const Span sp = span_of<R, COLS>(a, sq, slot - (sq.r0 * G / R + b));
  if (sp.rows == 0) {
    if constexpr (SHARED) continue;
    return;
  }
  // its stages t0 .. t0 + n - 1 of the row tile; `whole`: these are all
  int t0 = 0, n = sp.tiles;
  bool whole = true;
  int place = 0;
  if constexpr (SHARED) {
    const int tile_end = __builtin_amdgcn_readfirstlane(a.ends[slot]), units = max(sp.tiles, 1), unit0 = tile_end - units;
    t0 = max(at - unit0, 0);
    const int t1 = min(end - unit0, units);
    place = unit0 + t0 == first ? 0 : 1;                     // of the two row tiles that a share may cut
    at = min(tile_end, end);
    if (t0 >= t1) continue;                                  // (the tile's stages are the next share's)
    whole = t0 == 0 && t1 == units;
    n = min(t1, sp.tiles) - t0;
  } else {
    at = end;
  }

  const int cap = a.bt.max_pages * a.pg.size;
  const int rr = 32 * wave + r32;
  const bool row_ok = rr < sp.rows;
  const int rho = sp.rho0 + (row_ok ? rr : 0);
  const int tok = rho / G, head = kvh * G + rho % G, pos = sp.start + tok;
  // positions of the wave's first and last row (none: no key is seen)
  const int last_row = min(32 * wave + 31, sp.rows - 1);
  const bool wave_ok = 32 * wave < sp.rows;
  const int w_min = sp.start + (sp.rho0 + 32 * wave) / G;
  const int w_max = wave_ok ? min(sp.start + (sp.rho0 + last_row) / G, cap - 1) : -1;
  const int w_lo = a.window > 0 && w_min >= a.window ? w_min - a.window + 1 : 0;         // the first key (but for the leading) of any
  const int w_all = a.window > 0 && w_max >= a.window ? w_max - a.window + 1 : 0;        // ... of every row
  const int jmax = row_ok ? min(pos, cap - 1) : -1;
  const int jmin = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;

  // pages and scales of stages [from, from + kAhead): thread x < 128 has 16 keys
  auto page_of = [&](int from) {
    const int st = t0 + from + (tid >> 2);
    int p = -1;
    if (tid < 4 * kAhead && st < t0 + n) {
      const int page = (key_of<COLS>(sp, st) + (tid & 3) * 16) >> a.pg.log2;
      if (page < a.bt.max_pages) p = a.bt.table[(int64_t)b * a.bt.max_pages + page];
      if ((uint32_t)p >= (uint32_t)a.pg.num) p = -1;
    }
    return p;
  };
  auto scales_of = [&](int p) {
    float ks = 0.0f;
    ValueScale vs{0.0f, 1.0f};
    if (p >= 0) {
      ks = key_scale(a.ksc[(int64_t)p * a.pg.heads + kvh]);
      vs = value_scale(a.vsc[(int64_t)p * a.pg.heads + kvh]);
    }
    return make_float4(ks, vs.log2, vs.inv, __int_as_float(p));
  };

  const int page0 = page_of(0);                                       // (asked for before the queries)
  f16x8 qf[KS], ql[F16 ? KS : 1];
  float mul;
  {
    const uint16_t* src = a.q + (int64_t)(sp.r0 + tok) * a.qs + (int64_t)head * D;
    mul = load_query<KS, F16>(a, src, row_ok, pos, cap, qf, ql, [hw](int k) { return 2 * k + hw; },
                              [](float m) { return xor32_max(m); });
  }

  // loads: x of the wave covers keys of one 16-key group; a lane has 16 channels of a key
  typedef uint32_t v4u __attribute__((ext_vector_type(4)));
  v4u kw[NI], vw[NI];
  const int lane_key = tid / LPK, lane_ch = tid % LPK;
  auto fetch = [&](int st) __attribute__((always_inline)) {          // stage st (of the n)
    const int key0 = key_of<COLS>(sp, t0 + st);
#pragma unroll
    for (int x = 0; x < NI; ++x) {
      const int key = x * (256 / LPK) + lane_key;
      const int grp = __builtin_amdgcn_readfirstlane(key >> 4);
      const int p = __builtin_amdgcn_readfirstlane(__float_as_int(s_page[(st / kAhead) & 1][(st % kAhead) * 4 + grp].w));
      const int64_t base = (((int64_t)max(p, 0) * a.pg.heads + kvh) * a.pg.size + ((key0 + grp * 16) & (a.pg.size - 1))) * D;
      const uint32_t at = (uint32_t)((key & 15) * D + lane_ch * 16);
      kw[x] = *reinterpret_cast<const v4u*>(a.kc + base + at);
      vw[x] = *reinterpret_cast<const v4u*>(a.vc + base + at);
    }
  };
  auto store = [&](PromptSlot<D>& sl, int st) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NI; ++x) {
      const int key = x * (256 / LPK) + lane_key;
      if constexpr (!I8) {                                            // codes that no row sees may be NaN
        const float gone = s_page[(st / kAhead) & 1][(st % kAhead) * 4 + (key >> 4)].w;
        const bool there = (__float_as_int(gone) >= 0) & seen_by_any(a, sp, key_of<COLS>(sp, t0 + st) + key);
#pragma unroll
        for (int e = 0; e < 4; ++e) vw[x][e] = there ? vw[x][e] : 0u;
      }
      const int g = swz32_f<D>(key & 31);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int at = key * D + ((2 * lane_ch + c) ^ g) * 8;
        uint32_t w[4];
        widen4<I8>(kw[x][2 * c], w);
        widen4<I8>(kw[x][2 * c + 1], w + 2);
        *reinterpret_cast<u32x4*>(sl.k + at) = u32x4{w[0], w[1], w[2], w[3]};
        widen4<I8>(vw[x][2 * c], w);
        widen4<I8>(vw[x][2 * c + 1], w + 2);
        *reinterpret_cast<u32x4*>(sl.v + at) = u32x4{w[0], w[1], w[2], w[3]};
      }
    }
  };
  // LDS read offsets (elements), as in the dense kernel: K row r32, chunk 2 ks + hw; V transposed: lane (16 g + 4 t + q) at
  // V[16 kb + 4 (g >> 1) + t (+ 8)][32 db + 16 (g & 1) + 4 q]
  int koff[KS], voff[DB], voff8[DB];
  {
    const int g16 = lane >> 4, m16 = lane & 15;
    const int tq = m16 >> 2, q = m16 & 3;
    const int col0 = 4 * (g16 >> 1) + tq;
    const int c_lo = 2 * (g16 & 1) + (q >> 1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = r32 * D + ((2 * ks + hw) ^ swz32_f<D>(r32)) * 8;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      voff[db] = col0 * D + ((4 * db + c_lo) ^ swz32_f<D>(col0)) * 8 + 4 * (q & 1);
      voff8[db] = (col0 + 8) * D + ((4 * db + c_lo) ^ swz32_f<D>(col0 + 8)) * 8 + 4 * (q & 1);
    }
  }
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16{};
  float ref = -INFINITY, top = -INFINITY, lsum = 0.0f;

  auto compute = [&](const PromptSlot<D>& sl, int st) __attribute__((always_inline)) {
    const int key0 = key_of<COLS>(sp, t0 + st);
    if (key0 > w_max || (key0 + COLS <= w_lo && key0 >= a.n_sink)) return;     // uniform: no row of the wave sees a key of it
    const float4* pages = s_page[(st / kAhead) & 1] + (st % kAhead) * 4;
    f32x16 s[NBK];
#pragma unroll
    for (int x = 0; x < NBK; ++x) s[x] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < NBK; ++x) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(&sl.k[x * 32 * D + koff[ks]]);
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w), qf[ks], s[x], 0, 0, 0);
        if constexpr (F16)
          if (a.rt.table) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w), ql[ks], s[x], 0, 0, 0);
      }
    float mg[2 * NBK], lv[2 * NBK], iv[2 * NBK], least = INFINITY;
    int gone = 0;
    bool spoilt = false;
#pragma unroll
    for (int g = 0; g < 2 * NBK; ++g) {
      const float4 w = pages[g];
      mg[g] = w.x * mul;
      lv[g] = w.y;
      iv[g] = w.z;
      gone |= __float_as_int(w.w);
      spoilt |= w.z < 0.0f;
      least = fminf(least, w.y);
    }
    const bool holes = __builtin_amdgcn_readfirstlane(gone) < 0;
    if (key0 + COLS - 1 > w_min || (key0 < w_all && key0 + COLS > a.n_sink) || holes) {    // uniform
#pragma unroll
      for (int g = 0; g < 2 * NBK; ++g) {
        const int most = __float_as_int(pages[g].w) < 0 ? -1 : jmax;
#pragma unroll
        for (int v = 8 * (g & 1); v < 8 * (g & 1) + 8; ++v) {
          const int j = key0 + 32 * (g >> 1) + 8 * (v >> 2) + 4 * hw + (v & 3);
          const bool see = (j <= most) & ((j >= jmin) | (j < a.n_sink));
          s[g >> 1][v] = see ? s[g >> 1][v] * mg[g] : -INFINITY;
        }
        mg[g] = 1.0f;
      }
    }
    auto largest = [&](int g) {                                       // of a group's products
      const int x = g >> 1, v0 = 8 * (g & 1);
      const float m0 = max3(s[x][v0], s[x][v0 + 1], s[x][v0 + 2]), m1 = max3(s[x][v0 + 3], s[x][v0 + 4], s[x][v0 + 5]);
      return max3(max3(m0, s[x][v0 + 6], s[x][v0 + 7]), m1, m1);
    };
    float most = -INFINITY;                                           // contribution
#pragma unroll
    for (int g = 0; g < 2 * NBK; ++g) most = fmaxf(most, fmaf(largest(g), mg[g], lv[g]));
    most = xor32_max(most);
    auto lift = [&] {                                                 // the normaliser in units of the largest score
      float to = -INFINITY;
#pragma unroll
      for (int g = 0; g < 2 * NBK; ++g) to = fmaxf(to, largest(g) * mg[g]);
      to = xor32_max(to);
      if (to > top) {
        lsum *= __builtin_amdgcn_exp2f(top - to);
        top = to;
      }
    };
    const bool raise = most > ref + 8.0f;
    if (__builtin_amdgcn_ballot_w64(raise) != 0) {
      const float nm = raise ? most : ref;
      const float alpha = raise ? __builtin_amdgcn_exp2f(ref - nm) : 1.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] *= alpha;
      ref = nm;
      lift();
    }
    const float base = ref == -INFINITY ? 0.0f : ref;
    float share = ref_to_top(ref, top);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64((least <= kNoScale) | (ref - top - least > kRoom)) != 0, 0)) {
      lift();
      const float from = top == -INFINITY ? 0.0f : top;
      share = 0.0f;
#pragma unroll
      for (int g = 0; g < 2 * NBK; ++g) {
#pragma unroll
        for (int v = 8 * (g & 1); v < 8 * (g & 1) + 8; ++v)
          lsum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[g >> 1][v], mg[g], -from));
        lv[g] = lv[g] <= kNoScale ? -INFINITY : lv[g];
      }
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(spoilt) != 0, 0)) {                   // a value scale that is not finite: the rows that see it
      bool any = false;
#pragma unroll
      for (int x = 0; x < NBK; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) any |= iv[2 * x + (v >> 3)] < 0.0f && s[x][v] != -INFINITY;
      const float bad = xor32_add(any ? 1.0f : 0.0f) > 0.0f ? NAN : 0.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] += bad;
    }
    float sum = 0.0f;                                                 // the stage's part of the normaliser, in units of 2^ref
#pragma unroll
    for (int x = 0; x < NBK; ++x) {
      float pr[16];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float off = lv[2 * x + g] - base;
        float ts[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 8 * g; v < 8 * g + 8; ++v) {
          pr[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][v], mg[2 * x + g], off));
          ts[v & 1] += pr[v];
        }
        sum = fmaf(ts[0] + ts[1], fabsf(iv[2 * x + g]), sum);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4 pw = {pack_f16x2(pr[8 * kb + 0], pr[8 * kb + 1]), pack_f16x2(pr[8 * kb + 2], pr[8 * kb + 3]),
                          pack_f16x2(pr[8 * kb + 4], pr[8 * kb + 5]), pack_f16x2(pr[8 * kb + 6], pr[8 * kb + 7])};
        const f16x8 pf = __builtin_bit_cast(f16x8, pw);
        const uint16_t* vt = sl.v + x * 32 * D + 16 * kb * D;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const i16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16(FL_LDS4(vt + voff[db]));
          const i16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16(FL_LDS4(vt + voff8[db]));
          const i16x8 v8 = __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7);
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v8), pf, acc[db], 0, 0, 0);
        }
      }
    }
    lsum = fmaf(sum, share, lsum);
  };

  if (n > 0) {
    if constexpr (SHARED) __syncthreads();                                      // (the last row tile's stages are read)
    if (tid < 4 * kAhead) s_page[0][tid] = scales_of(page0);
    __syncthreads();
    fetch(0);
    store(s0, 0);
    __syncthreads();
    int ahead = -1;                                                   // page of the next block's 16 keys
    float4 ahead_s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto step = [&](PromptSlot<D>& cur, PromptSlot<D>& nxt, int st) __attribute__((always_inline)) {
      const int ph = st % kAhead;                                     // uniform; the next block's table in three steps
      if (ph == 0) ahead = page_of(st + kAhead);
      if (ph == 8) ahead_s = scales_of(ahead);
      if (ph == 16 && tid < 4 * kAhead) s_page[((st / kAhead) & 1) ^ 1][tid] = ahead_s;
      if (st + 1 < n) fetch(st + 1);
      compute(cur, st);
      if (st + 1 < n) store(nxt, st + 1);
      __syncthreads();
    };
    for (int st = 0; st < n; st += 2) {
      step(s0, s1, st);
      if (st + 1 < n) step(s1, s0, st + 1);
    }
  }
  lsum = xor32_add(lsum);
  const int64_t gr = (int64_t)(sp.r0 + tok) * a.Hq + head;
  const bool none = top == -INFINITY && lsum == 0.0f;
  if (SHARED && row_ok && !whole) {
    // a share cuts at most two row tiles: the one it begins with and the one it ends with
    const int64_t row = ((int64_t)(kvh * a.share + wg) * 2 + place) * R + rr;
    float* out = a.part + row * D + 4 * hw;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(out + db * 32 + 8 * j) =
            make_float4(acc[db][4 * j], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]);
    if (hw == 0) *reinterpret_cast<float4*>(a.part_ml + row * 4) = make_float4(ref, top, lsum, 0.0f);
  }
  if (row_ok && whole) {
  const float inv = none ? 0.0f : ref_to_top(ref, top) / lsum;
  uint16_t* out = a.o + (int64_t)(sp.r0 + tok) * a.os + (int64_t)head * D + 4 * hw;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = acc[db][4 * j + e] * inv;
      *reinterpret_cast<u32x2*>(out + db * 32 + 8 * j) = u32x2{F16 ? pack_f16x2(o[0], o[1]) : pack_bf16x2(o[0], o[1]),
                                                               F16 ? pack_f16x2(o[2], o[3]) : pack_bf16x2(o[2], o[3])};
    }
  if (hw == 0 && a.lse) a.lse[gr] = none ? -INFINITY : (top + __builtin_amdgcn_logf(lsum)) * 0.6931471805599453f;
 }
  }
}

// Row tiles that shares cut: a workgroup has 32 rows of one, d / 4 threads a row.
template <int D, bool F16>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int R = kPromptRows, LN = D / 4;
  const int kvh = blockIdx.x % a.pg.heads, rest = blockIdx.x / a.pg.heads;
  const int slot = rest / 4, r0 = (rest % 4) * 32;
  const Cut cut = cut_of(a);
  const int before = slot > 0 ? a.ends[slot - 1] : 0, end = a.ends[slot];
  if (before >= end) return;
  const int begin = before + kTileUnits;                     // its first stage
  const int p0 = cut.owner(begin), p1 = cut.owner(end - 1);
  if (p0 == p1) return;
  const int G = a.G;
  const Seq sq = find_seq(a.bt, slot, 1, [G](int c) { return c * G / R; });
  if (sq.b < 0) return;
  const Span sp = span_of<R, kPromptKeys>(a, sq, slot - (sq.r0 * G / R + sq.b));
  const int c = threadIdx.x % LN;
  for (int rr = r0 + threadIdx.x / LN; rr < min(r0 + 32, sp.rows); rr += 256 / LN) {
    auto place = [&](int p) { return ((int64_t)(kvh * a.share + p) * 2 + (max(begin, cut.begin(p)) == cut.begin(p) ? 0 : 1)) * R + rr; };
    const float4* ml = reinterpret_cast<const float4*>(a.part_ml);
    float m = -INFINITY, top = -INFINITY;
#pragma unroll 4
    for (int p = p0; p <= p1; ++p) {
      const float4 w = ml[place(p)];
      m = fmaxf(m, w.x);
      top = fmaxf(top, w.y);
    }
    float sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int p = p0; p <= p1; ++p) {
      const int64_t at = place(p);
      const float4 w = ml[at];
      const float4 x = *reinterpret_cast<const float4*>(a.part + at * D + 4 * c);
      const bool idle = w.y == -INFINITY && w.z == 0.0f;
      const float f = idle ? 0.0f : __builtin_amdgcn_exp2f(w.x - m);
      sum = fmaf(idle ? 0.0f : __builtin_amdgcn_exp2f(w.y - top), w.z, sum);
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    const bool none = top == -INFINITY && sum == 0.0f;
    const float inv = none ? 0.0f : ref_to_top(m, top) / sum;
    const int rho = sp.rho0 + rr, tok = rho / G, head = kvh * G + rho % G;
    *reinterpret_cast<u32x2*>(a.o + (int64_t)(sp.r0 + tok) * a.os + (int64_t)head * D + 4 * c) =
        u32x2{F16 ? pack_f16x2(o.x * inv, o.y * inv) : pack_bf16x2(o.x * inv, o.y * inv),
              F16 ? pack_f16x2(o.z * inv, o.w * inv) : pack_bf16x2(o.z * inv, o.w * inv)};
    if (a.lse && c == 0)
      a.lse[(int64_t)(sp.r0 + tok) * a.Hq + head] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

// Sums of cut row tiles, two for each share, and the ends of the row tiles.  No key is split where every row tile has a workgroup
// of its own.
static int shares_of(int Hkv) { return std::max(1, kPromptShares / Hkv); }
// (keys: that a row sees at most; below 1024 the two kernels more cost more than idle CUs.  cap: positions of a block table's row;
// all units of a head count below 2^31)
static bool is_shared(int64_t slots, int Hkv, int64_t cap, int64_t keys) {
  return slots * Hkv < 2 * kPromptShares && keys >= 1024 && slots * (cap / kPromptKeys + 16) < (1ll << 31) - 65536;
}
size_t paged_prompt_ws(int64_t slots, int Hkv, int d, int64_t cap, int64_t keys) {
  if (!is_shared(slots, Hkv, cap, keys)) return 0;
  return (size_t)shares_of(Hkv) * Hkv * 2 * kPromptRows * (d + 4) * sizeof(float) + (size_t)slots * sizeof(int);
}

int launch_paged_prompt(const PagedAttnArgs& args, int d, int format, bool f16, int64_t keys, hipStream_t st) {
  PagedAttnArgs a = args;
  const int64_t slots = (int64_t)a.bt.T * a.G / kPromptRows + a.bt.B;
  const bool shared = is_shared(slots, a.pg.heads, (int64_t)a.bt.max_pages * a.pg.size, keys);
  FL_REQUIRE(slots * a.pg.heads * 4 < (1ll << 31), FL_E_SHAPE, "fl_paged_attn: too many rows");
  a.slots = (int)slots;
  a.share = shares_of(a.pg.heads);
  int rc;
  if (shared) {
    const size_t places = (size_t)a.share * a.pg.heads * 2 * kPromptRows;
    a.part_ml = a.part + places * d;
    a.ends = reinterpret_cast<int*>(a.part_ml + places * 4);
    paged_plan_kernel<<<1, 1024, 0, st>>>(a);
    rc = check_launch("paged_plan_kernel");
    if (rc != FL_OK) return rc;
  }
  const unsigned grid = (unsigned)((shared ? a.share : slots) * a.pg.heads);
#define FL_PROMPT(DD, SS)                                                              \
  do {                                                                                 \
    if (format == FL_KV_I8) {                                                          \
      if (f16) paged_prompt_kernel<DD, true, true, SS><<<grid, 256, 0, st>>>(a);       \
      else paged_prompt_kernel<DD, true, false, SS><<<grid, 256, 0, st>>>(a);          \
    } else {                                                                           \
      if (f16) paged_prompt_kernel<DD, false, true, SS><<<grid, 256, 0, st>>>(a);      \
      else paged_prompt_kernel<DD, false, false, SS><<<grid, 256, 0, st>>>(a);         \
    }                                                                                  \
  } while (0)
  if (d == 128 && shared) FL_PROMPT(128, true);
  else if (d == 128) FL_PROMPT(128, false);
  else if (shared) FL_PROMPT(64, true);
  else FL_PROMPT(64, false);
#undef FL_PROMPT
  rc = check_launch("paged_prompt_kernel");
  if (rc != FL_OK || !shared) return rc;
  const unsigned join = (unsigned)(slots * 4 * a.pg.heads);
  if (d == 128) {
    if (f16) paged_join_kernel<128, true><<<join, 256, 0, st>>>(a);
    else paged_join_kernel<128, false><<<join, 256, 0, st>>>(a);
  } else {
    if (f16) paged_join_kernel<64, true><<<join, 256, 0, st>>>(a);
    else paged_join_kernel<64, false><<<join, 256, 0, st>>>(a);
  }
  return check_launch("paged_join_kernel");
}

}  // namespace fl
