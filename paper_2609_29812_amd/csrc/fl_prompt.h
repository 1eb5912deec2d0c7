// Dense causal attention for many rows per sequence, over keys and values from any source that can lay them out in LDS: the kernel,
// how its work is cut, and the joining of row tiles that a cut splits.
#pragma once

#include "fl_paged_attn.h"

#include <algorithm>
#include <cmath>

namespace fl {

constexpr int kStageKeys = 64;

// The keys or the values of a stage in LDS: blocks of 32 rows, 16-byte chunks permuted (swz32_f).  (Each buffer is an object of its
// own: the compiler orders reads of one behind loads into the same alone.)
template <int D, int PARTS = 1>
struct __attribute__((aligned(16))) StageTile {
  uint16_t x[PARTS * kStageKeys * D];        // (the second part of each behind all first ones)
};

// x, as if just computed
__device__ __forceinline__ void renew(int& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void renew(uint32_t& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void renew(float& x) { asm volatile("" : "+v"(x)); }

// The sources' own are found by their arguments; a template of the name has to be known for that.
template <int R> Seq find_row_tile();

// What the host knows of a call, as far as it decides how the work is cut.
struct PromptShape {
  int B, T, G, Hkv;                          // sequences, query positions, query heads of a key/value head, these
  int64_t past, keys, cap;                   // positions before the first query, on average; keys that a row sees at most; of a sequence at most
};

template <bool F16>
__device__ __forceinline__ f32x16 mma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) { return F16 ? pack_f16x2(a, b) : pack_bf16x2(a, b); }

// ends[s]: units of row tiles 0 .. s, for shares of equal work (SrcArgs: seq_of(a, b) gives a sequence).  One workgroup: 5 us, its chain
// of loads and sums.
template <class SrcArgs, int R>
__global__ __launch_bounds__(1024) void prompt_plan_kernel(SrcArgs a) {
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
        if ((int)((int64_t)row_of(a.bt, mid) * a.G / R) + mid <= slot) lo = mid;
        else hi = mid;
      }
      const Seq q = seq_of(a, lo);
      const Span sp = span_of<R, kStageKeys>(a, q, slot - ((int)((int64_t)q.r0 * a.G / R) + lo));
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
__device__ __forceinline__ int slot_of_unit(const int* ends, int slots, int x) {
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

// A workgroup has 128 rows of a sequence and key/value head (positions and the head's query heads), its four waves 32 each, and goes
// through the keys that they see in stages of 64, which the source lays out in LDS (two buffers for keys, two for values).
//   S^T = K Q^T     v_mfma_f32_32x32x16: a lane has one row (lane % 32) and half of the stage's keys, so that a row's largest score and
//                   sum stay in the lane but for one exchange with the other half.
//   O^T += V^T P^T  the same product: what a lane holds of P is the operand as it lies; V comes through transposing LDS reads.
// One pass: o and the sum are relative to a running reference, which is raised (and they rescaled) when a score is ahead of it by more
// than 8 octaves: probabilities reach 2^8 and are rounded to the products' type, scores, sums and outputs stay in fp32.
// Stages are a step apart: the scores of stage t + 1 are multiplied while the exponentials of stage t are taken, O of stage t while what
// is left of them and the largest scores of t + 1 are; a barrier a stage, loads waited for where the stage ends.
// What bounds it: the matrix cores (16384 positions of 16 heads x 128, bf16: busy for 63 % of the cycles, the vector units for 53 %; 990
// to 1080 us from card to card, 1020 to 1110 TFLOP/s, where a large product has 1224), with 64 channels the vector units (67 and 37 %; 32
// exponentials of 8 cycles and 100 instructions of 4 a wave and stage either way, beside half of the products; 8192 positions 172 us,
// 800 TFLOP/s), below a thousand positions the chain of a stage's loads, products and exponentials (300 positions 12 us).
// Taken against: 64 rows a wave, which halve the reads of LDS (512 registers, spilled: 3350 us for 1070); eight waves a workgroup (16384
// positions 1026 and 1033 us, windows of 1024 97 and 80); fragments read three or four ahead in place of two (0.5 %); wave priorities
// around the products (1 %).
template <class Src, class SrcArgs, bool SHARED>
__global__ __launch_bounds__(256, Src::kWavesPerSimd) void prompt_kernel(SrcArgs a) {
  constexpr int D = Src::kD, R = 128;
  constexpr int NBK = kStageKeys / 32;     // 32-key blocks of a stage
  constexpr int KS = D / 16;               // k-steps of QK^T
  constexpr int DB = D / 32;               // 32-channel output blocks
  using KTile = StageTile<D, Src::kTwo ? 2 : 1>;
  __shared__ KTile k0, k1;
  __shared__ StageTile<D> v0, v1;
  // Masked stages whose values are not all finite: the values are set to 0, their places are bits of `odd`, a byte for eight channels.
  __shared__ int s_bad[2][4];              // by the wave that looked: the stage where there are some
  __shared__ uint32_t odd[2][kStageKeys * D / 32];

  const int kvh = blockIdx.x % a.pg.heads, wg = blockIdx.x / a.pg.heads;
  const int G = a.G;
  // the workgroup's run of units at .. end - 1 of its head, from row tile `slot` on; or all of one row tile
  int at = 0, end = 1, slot = gridDim.x / a.pg.heads - 1 - wg;          // (later rows see more keys: first)
  if constexpr (SHARED) {
    const Cut cut = cut_of(a);
    at = cut.begin(wg);
    end = cut.begin(wg + 1);
    if (at >= end) return;
    slot = slot_of_unit(a.ends, a.slots, at);
  }
  const int first = at;
  // (offsets that do not ascend: the plan may give units to row tiles that have no rows here, so units alone do not end the walk)
  for (; at < end && (!SHARED || slot < a.slots); ++slot) {
    int tid = threadIdx.x;
    if constexpr (SHARED) renew(tid);                        // (what a row tile derives from the lane is formed anew)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hw = lane >> 5, r32 = lane & 31;
    const Seq sq = find_row_tile<R>(a, slot);
    if (sq.b < 0) return;
    const Span sp = span_of<R, kStageKeys>(a, sq, slot - ((int)((int64_t)sq.r0 * G / R) + sq.b));
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
      place = unit0 + t0 == first ? 0 : 1;                   // of the two row tiles that a share may cut
      at = min(tile_end, end);
      if (t0 >= t1) continue;                                // (the tile's stages are the next share's)
      whole = t0 == 0 && t1 == units;
      n = min(t1, sp.tiles) - t0;
    } else {
      at = end;
    }

    const int cap = a.bt.max_pages * a.pg.size;
    const int row = 32 * wave + r32;
    const bool row_ok = row < sp.rows;
    const int rho_q = sp.rho0 + (row_ok ? row : 0), pos = sp.start + rho_q / G;
    const int jmax = row_ok ? min(pos, cap - 1) : -1;
    const int jmin = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
    // positions of the wave's first and last row, also behind the last key (a wave without rows: -1)
    const int row0 = 32 * wave;
    const int w_min = sp.start + (sp.rho0 + row0) / G;
    const int w_max = row0 < sp.rows ? sp.start + (sp.rho0 + min(row0 + 32, sp.rows) - 1) / G : -1;
    // the first key (but for the leading) that all rows up to position `last` see
    auto first_of_all = [&](int last) { return a.window > 0 && last >= a.window ? min(last - a.window + 1, cap) : 0; };
    const int w_all = first_of_all(w_max);

    Src src(a, sq, sp, kvh, tid, t0, n);
    if (n > 0) {
      if constexpr (SHARED) __syncthreads();                 // (the last row tile's stages are read)
      src.begin(k0, k1, v0);                                 // (the first loads, before those of the queries)
    }
    u32x4 qf[KS], ql[Src::kLow ? KS : 1];
    const float mul = src.query(a, sp.r0 + rho_q / G, kvh * G + rho_q % G, pos, row_ok, hw, qf, ql);
    // LDS read offsets (elements).  Keys (A operand): row r32, chunk 2 ks + hw.  Values (transposed reads): lane (16 g + 4 t + q)
    // at V[16 kb + 4 (g >> 1) + t (+ 8)][32 db + 16 (g & 1) + 4 q]
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
    float ref = -INFINITY, lsum = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x16{};
    auto key0_of = [&](int st) { return key_of<kStageKeys>(sp, t0 + st); };
    // stages from .. from + len - 1, uniform: every row sees every key (the tiles of leading positions count as masked)
    struct Clear {
      int from;
      uint32_t len;
      __device__ __forceinline__ bool operator()(int st) const { return (uint32_t)(st - from) < len; }
    };
    auto clear_of = [&](int least, int low) {                // least: the first row's position; low: first key that all see
      const int c0 = sp.n_lead + max((low + kStageKeys - 1) / kStageKeys - sp.first, 0) - t0;
      const int c1 = sp.n_lead + ((least + 1) >> 6) - sp.first - t0;         // (kStageKeys is 64; -1 >> 6 is -1)
      return Clear{max(c0, 0), (uint32_t)max(c1 - max(c0, 0), 0)};
    };
    const Clear wave_clear = clear_of(w_min, w_all);
    const Clear tile_clear = clear_of(sp.i_min, first_of_all(sp.i_max));
    auto masked = [&](int st) { return !wave_clear(st) || src.holes(st); };
    auto tile_masked = [&](int st) { return !tile_clear(st); };

    // scores of a stage, S^T = K Q^T: a lane has 16 keys of one row per block
    auto scores = [&](f32x16 (&s)[NBK], const KTile& kt) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < NBK; ++b) s[b] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int b = 0; b < NBK; ++b) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(&kt.x[b * 32 * D + koff[ks]]);
          s[b] = mma32<Src::kF16>(w, qf[ks], s[b]);
          if constexpr (Src::kLow) s[b] = mma32<Src::kF16>(w, ql[ks], s[b]);
          if constexpr (Src::kTwo)
            s[b] = mma32<Src::kF16>(*reinterpret_cast<const u32x4*>(&kt.x[kStageKeys * D + b * 32 * D + koff[ks]]), qf[ks], s[b]);
        }
    };
    auto largest = [&](const f32x16 (&s)[NBK], int g) __attribute__((always_inline)) {        // of half a block
      const f32x16& y = s[g / 2];
      const int v = 8 * (g & 1);
      const float m0 = max3(y[v], y[v + 1], y[v + 2]), m1 = max3(y[v + 3], y[v + 4], y[v + 5]);
      return max3(max3(m0, y[v + 6], y[v + 7]), m1, m1);
    };
    auto largest_of = [&](const f32x16 (&s)[NBK]) __attribute__((always_inline)) {
      float m = largest(s, 0);
#pragma unroll
      for (int g = 1; g < 2 * NBK; ++g) m = fmaxf(m, largest(s, g));
      return m;
    };
    // What a row does not see is -inf: a word of bits for the lane's keys, taken by two instructions a score.
    auto mask = [&](f32x16 (&s)[NBK], int st) __attribute__((always_inline)) {
      const int origin = key0_of(st) + 4 * hw;               // the lane's keys count from here: 0 .. 3, 8 .. 11, .. 56 .. 59
      auto until = [&](int j) {                              // keys 0 .. j
        const uint32_t n = min(4u * (uint32_t)(j >> 3) + min((uint32_t)(j & 7), 3u), 31u);
        return j < 0 ? 0u : ~0u >> (31u - n);
      };
      const uint32_t here = ((src.there(st) * 0x00204081u) & 0x01010101u) * 0xFFu;         // uniform: a byte of bits for 16 keys
      const uint32_t see = until(jmax - origin) & (~until(jmin - origin - 1) | until(a.n_sink - origin - 1)) & here;
#pragma unroll
      for (int b = 0; b < NBK; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)see, 16 * b + v, 1);
          s[b][v] = __uint_as_float((__float_as_uint(s[b][v]) & all) | (0xFF800000u & ~all));
        }
    };
    // the running references follow the largest scores of a stage, where those are ahead by more than 8 octaves
    auto refer = [&](float& most) __attribute__((always_inline)) {
      const float m = xor32_max(most) * mul;
      const bool raise = m > ref + 8.0f;
      if (__builtin_amdgcn_ballot_w64(raise) != 0) {
        const float nm = raise ? m : ref;
        const float alpha = raise ? __builtin_amdgcn_exp2f(ref - nm) : 1.0f;
        lsum *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] *= alpha;
        ref = nm;
      }
    };
    // One pair of a stage's probabilities (16 pairs a row), as half a word of the operands.
    float ts[2];
    auto weigh = [&](const f32x16 (&s)[NBK], u32x4 (&pf)[NBK][2], u32x4 (&pl)[NBK][2], float base, int i) __attribute__((always_inline)) {
      const int b = i / 8, v = 2 * (i % 8);
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][v], mul, -base));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][v + 1], mul, -base));
      ts[0] += p0;
      ts[1] += p1;
      uint32_t two = pack2<Src::kF16>(p0, p1);
      renew(ts[0]);                                          // (here: summed and packed later, the probabilities would stay in registers)
      renew(ts[1]);
      renew(two);
      pf[b][v / 8][(v % 8) / 2] = two;
      if constexpr (Src::kTwo) {
        uint32_t rest = Src::rest(p0, p1, two);
        renew(rest);
        pl[b][v / 8][(v % 8) / 2] = rest;
      }
    };
    auto read_k = [&](const KTile& kt, int i, int part) __attribute__((always_inline)) {       // k-step i / NBK, block i % NBK
      return *reinterpret_cast<const u32x4*>(&kt.x[part * kStageKeys * D + (i % NBK) * 32 * D + koff[i / NBK]]);
    };
    auto read_v = [&](const StageTile<D>& vt, int i) __attribute__((always_inline)) {          // keys 16 (i / DB), channels 32 (i % DB)
      const uint16_t* at_v = vt.x + 16 * (i / DB) * D;
      const i16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16(FL_LDS4(at_v + voff[i % DB]));
      const i16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16(FL_LDS4(at_v + voff8[i % DB]));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto score = [&](f32x16 (&s)[NBK], const u32x4& w, int i) __attribute__((always_inline)) {
      s[i % NBK] = mma32<Src::kF16>(w, qf[i / NBK], s[i % NBK]);
      if constexpr (Src::kLow) s[i % NBK] = mma32<Src::kF16>(w, ql[i / NBK], s[i % NBK]);
    };
    // NaN for what sees a value that is not finite
    auto poison = [&](int st) __attribute__((always_inline)) {
      const int key0 = key0_of(st);
      uint32_t m[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) m[db] = 0;
#pragma nounroll
      for (int i = 0; i < kStageKeys; ++i) {
        const int j = key0 + i;
        const bool see = (j <= jmax) & ((j >= jmin) | (j < a.n_sink)) & (s_bad[st & 1][Src::wave_of(i)] == st);
#pragma unroll
        for (int db = 0; db < DB; ++db) m[db] |= see ? odd[st & 1][i * DB + db] : 0u;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        m[db] >>= 4 * hw;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] = (m[db] >> (8 * (v >> 2) + (v & 3))) & 1u ? NAN : acc[db][v];
      }
    };
    // A stage: the scores of the next one (nxt) beside the probabilities of this one (cur), then O^T += V^T P^T beside what is left of
    // them and the largest scores of the next.  Each matrix instruction is followed by vector instructions that do not wait for it.
    // (With a second part of 128-channel queries the registers hold one stage's scores alone: there they are formed behind the products;
    // beside them, 6000 rows of 16 heads after 2000 positions take 543 us and not 461.)
    constexpr bool kBeside = !(Src::kLow && D == 128);
    constexpr int NQ = KS * NBK, NP = NBK * 2 * DB, EARLY = 12, LATE = NP * 3 / 4, LA = 2, MG = 2 * NBK;
    auto stage = [&](f32x16 (&cur)[NBK], f32x16 (&nxt)[NBK], KTile& K, const KTile& KN, const StageTile<D>& V,
                     StageTile<D>& VN, float& most)
        __attribute__((always_inline)) {
      u32x4 pf[NBK][2], pl[NBK][2], fr[LA + 1], fl[LA + 1];  // (second parts: kTwo)
      const float base = ref == -INFINITY ? 0.0f : ref;
      ts[0] = ts[1] = 0.0f;
      if constexpr (kBeside) {
#pragma unroll
        for (int b = 0; b < NBK; ++b) nxt[b] = f32x16{};
      }
      // the probabilities' pairs up to which each scores' and each products' instruction goes
      auto early = [](int i) { return EARLY * i / NQ; };
      auto late = [](int i) { return min(EARLY + (16 - EARLY) * i / LATE, 16); };
      auto score_all = [&](bool beside) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LA; ++i) {
          fr[i] = read_k(KN, i, 0);
          if constexpr (Src::kTwo) fl[i] = read_k(KN, i, 1);
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          if (i + LA < NQ) fr[(i + LA) % (LA + 1)] = read_k(KN, i + LA, 0);
          else if (beside) fr[(i + LA) % (LA + 1)] = read_v(V, i + LA - NQ);
          score(nxt, fr[i % (LA + 1)], i);
          if constexpr (Src::kTwo) {
            if (i + LA < NQ) fl[(i + LA) % (LA + 1)] = read_k(KN, i + LA, 1);
            nxt[i % NBK] = mma32<Src::kF16>(fl[i % (LA + 1)], qf[i / NBK], nxt[i % NBK]);
          }
          if (beside) {
#pragma unroll
            for (int y = early(i); y < early(i + 1); ++y) weigh(cur, pf, pl, base, y);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto multiply = [&](int first) __attribute__((always_inline)) {       // (first: of the fragments' registers)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if (i + LA < NP) fr[(first + i + LA) % (LA + 1)] = read_v(V, i + LA);
          acc[i % DB] = mma32<Src::kF16>(fr[(first + i) % (LA + 1)], pf[i / DB / 2][i / DB % 2], acc[i % DB]);
          if constexpr (Src::kTwo) acc[i % DB] = mma32<Src::kF16>(fr[(first + i) % (LA + 1)], pl[i / DB / 2][i / DB % 2], acc[i % DB]);
#pragma unroll
          for (int y = late(i); y < late(i + 1); ++y) weigh(cur, pf, pl, base, y);
          // (the source's own work; behind the last stages into buffers that are not read again)
#pragma unroll
          for (int y = Src::kItems * i / NP; y < Src::kItems * (i + 1) / NP; ++y) src.item(y, K, VN);
          if constexpr (kBeside) {
#pragma unroll
            for (int g = MG * i / NP; g < MG * (i + 1) / NP; ++g) {
              const float m = largest(nxt, g);
              most = g == 0 ? m : fmaxf(most, m);
              if (g == MG - 1) renew(most);                  // (here, beside the products)
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if constexpr (kBeside) {
        score_all(true);
        multiply(NQ);
      } else {
#pragma unroll
        for (int y = 0; y < EARLY; ++y) weigh(cur, pf, pl, base, y);
#pragma unroll
        for (int i = 0; i < LA; ++i) fr[i] = read_v(V, i);
        __builtin_amdgcn_sched_barrier(0);
        multiply(0);
#pragma unroll
        for (int b = 0; b < NBK; ++b) nxt[b] = f32x16{};
        score_all(false);
        most = largest_of(nxt);
      }
      lsum += ts[0] + ts[1];
    };
    // masked stages: the values that the wave's loads have brought
    auto look = [&](int st, StageTile<D>& v) __attribute__((always_inline)) {
      if constexpr (Src::kOdd)
        if (tile_masked(st)) {                               // uniform
          const bool any = __builtin_amdgcn_ballot_w64(src.odd(v, odd[st & 1])) != 0;
          if (lane == 0) s_bad[st & 1][wave] = any ? st : -1;
        }
    };
    if (n > 0) {
      // stages go K(t), then V(t), one behind: the scores of stage t + 1 are formed beside the probabilities of stage t
      src.finish(k0, k1, v0);
      look(0, v0);
      __syncthreads();
      f32x16 sa[NBK], sb[NBK];
      float most;
      auto enter = [&](f32x16 (&s)[NBK], int st) __attribute__((always_inline)) {
        if (masked(st)) {                                    // uniform
          mask(s, st);
          most = largest_of(s);
        }
        refer(most);
      };
      scores(sa, k0);
      most = largest_of(sa);
      enter(sa, 0);
      __syncthreads();                                       // (the first keys are read)
      // K: where stage st's keys were and st + 2's come; KN: st + 1's; V: st's values; VN: where st + 1's come
      auto step = [&](f32x16 (&cur)[NBK], f32x16 (&nxt)[NBK], int st, KTile& K, KTile& KN, StageTile<D>& V,
                      StageTile<D>& VN) __attribute__((always_inline)) {
        const bool more = st + 1 < n;                        // uniform
        if (st + 2 < n) src.load_k(st + 2, K);
        if (more) src.load_v(st + 1, VN);
        if constexpr (Src::kOdd)
          if (tile_masked(st)) {                             // uniform
            const int* bad = s_bad[st & 1];
            if (__builtin_expect(bad[0] == st || bad[1] == st || bad[2] == st || bad[3] == st, 0)) poison(st);
          }
        // (behind the last stage the next one's scores are of no use, and without harm)
        stage(cur, nxt, K, KN, V, VN, most);
        if (more) enter(nxt, st + 1);
        src.land();
        if (more) look(st + 1, VN);
        src.ahead(st);
        __syncthreads();
      };
      for (int st = 0; st < n; st += 2) {
        step(sa, sb, st, k0, k1, v0, v1);
        if (st + 1 < n) step(sb, sa, st + 1, k1, k0, v1, v0);
      }
    }
    if constexpr (Src::kMixed) {
      // values lie in the order 0 4 1 5 2 6 3 7: a half-wave's four become channels 0 .. 3 or 4 .. 7 of eight
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x16& o = acc[db];
          const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[4 * j]), __float_as_uint(o[4 * j + 1]), false, false);
          const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[4 * j + 2]), __float_as_uint(o[4 * j + 3]), false, false);
          o[4 * j] = __uint_as_float(p[0]);
          o[4 * j + 1] = __uint_as_float(q[0]);
          o[4 * j + 2] = __uint_as_float(p[1]);
          o[4 * j + 3] = __uint_as_float(q[1]);
        }
    }
    lsum = xor32_add(lsum);
    if (row_ok) {
      const int rho = sp.rho0 + row, tok = rho / G, head = kvh * G + rho % G;
      const bool none = ref == -INFINITY && lsum == 0.0f;
      if (SHARED && !whole) {
        // a share cuts at most two row tiles: the one it begins with and the one it ends with
        const int64_t pr = ((int64_t)(kvh * a.share + wg) * 2 + place) * R + row;
        float* out = a.part + pr * D + 4 * hw;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<float4*>(out + db * 32 + 8 * j) =
                make_float4(acc[db][4 * j], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]);
        if (hw == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = make_float2(ref, lsum);
      } else {
        const float inv = none ? 0.0f : 1.0f / lsum;
        uint16_t* out = a.o + (int64_t)(sp.r0 + tok) * a.os + (int64_t)head * D + 4 * hw;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x16& o = acc[db];
            *reinterpret_cast<u32x2*>(out + db * 32 + 8 * j) = u32x2{pack2<Src::kOut16>(o[4 * j] * inv, o[4 * j + 1] * inv),
                                                                     pack2<Src::kOut16>(o[4 * j + 2] * inv, o[4 * j + 3] * inv)};
          }
        if (hw == 0 && a.lse)
          a.lse[(int64_t)(sp.r0 + tok) * a.Hq + head] = none ? -INFINITY : (ref + __builtin_amdgcn_logf(lsum)) * 0.6931471805599453f;
      }
    }
  }
}

// Row tiles that shares cut: a workgroup has 32 rows of one, d / 4 threads a row.  The parts are read once, in fp32 as they were summed
// (912 tiles of 130 stages in 512 shares: 70 MB of parts, 19 us).
template <class Args, int D, bool OUT16, int R>
__global__ __launch_bounds__(256) void prompt_join_kernel(Args a) {
  constexpr int LN = D / 4, PER = R / 32;
  const int kvh = blockIdx.x % a.pg.heads, rest = blockIdx.x / a.pg.heads;
  const int slot = rest / PER, r0 = (rest % PER) * 32;
  const Cut cut = cut_of(a);
  const int before = slot > 0 ? a.ends[slot - 1] : 0, end = a.ends[slot];
  if (before >= end) return;
  const int begin = before + kTileUnits;                     // its first stage
  const int p0 = cut.owner(begin), p1 = cut.owner(end - 1);
  if (p0 == p1) return;
  const int G = a.G;
  const Seq sq = find_row_tile<R>(a, slot);
  if (sq.b < 0) return;
  const Span sp = span_of<R, kStageKeys>(a, sq, slot - ((int)((int64_t)sq.r0 * G / R) + sq.b));
  const int c = threadIdx.x % LN;
  for (int rr = r0 + threadIdx.x / LN; rr < min(r0 + 32, sp.rows); rr += 256 / LN) {
    auto place = [&](int p) { return ((int64_t)(kvh * a.share + p) * 2 + (max(begin, cut.begin(p)) == cut.begin(p) ? 0 : 1)) * R + rr; };
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
    float m = -INFINITY;
#pragma unroll 4
    for (int p = p0; p <= p1; ++p) m = fmaxf(m, ml[place(p)].x);
    float sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int p = p0; p <= p1; ++p) {
      const int64_t at = place(p);
      const float2 w = ml[at];
      const float4 x = *reinterpret_cast<const float4*>(a.part + at * D + 4 * c);
      // (a part with NaN scores alone has no reference, but counts)
      const float f = w.x == -INFINITY ? (w.y == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(w.x - m);
      sum = fmaf(f, w.y, sum);
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    const bool none = m == -INFINITY && sum == 0.0f;
    const float inv = none ? 0.0f : 1.0f / sum;
    const int rho = sp.rho0 + rr, tok = rho / G, head = kvh * G + rho % G;
    *reinterpret_cast<u32x2*>(a.o + (int64_t)(sp.r0 + tok) * a.os + (int64_t)head * D + 4 * c) =
        u32x2{pack2<OUT16>(o.x * inv, o.y * inv), pack2<OUT16>(o.z * inv, o.w * inv)};
    if (a.lse && c == 0)
      a.lse[(int64_t)(sp.r0 + tok) * a.Hq + head] = none ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

constexpr int kRowsOfTile = 128;
inline int prompt_shares(int Hkv) { return std::max(1, 512 / Hkv); }
// How a call is cut: a workgroup for each row tile, or equal shares of all tiles' stages for 512 workgroups (two a CU), which the plan,
// the join and the parts' way through memory make 35 to 45 us dearer.  Cut where tiles one by one would leave CUs idle for longer, as far
// as the host can tell: the longest tile beyond an even share of the stages, at 1.0 us a stage then and at 1.75 where its keys are read
// by few tiles (a chunk after a long context); or the last round's free places, where all tiles are about as long, at 2.
// Tiles one by one against shares: prompts of 16 heads x 128, 1500 positions 33 and 42 us, 4096 90 and 103, 8192 272 and 307; of 4
// heads, 4096 positions 74 and 48 us, 16384 326 and 285; 512 rows of 16 heads after 3584 keys 109 and 83 us; from the 4-bit cache, 100
// rows of 8 heads after 5000 positions 122 and 37 us, 512 after each of 4 x 4000 (32 / 8 heads) 177 and 202, chunks of 1009, 512 and
// 2000 after 15000, 0 and 6001 (912 tiles: 1.8 rounds) 728 and 602.
inline bool prompt_shared(const PromptShape& s) {
  const int64_t slots = (int64_t)s.T * s.G / kRowsOfTile + s.B;
  if (slots * (s.cap / kStageKeys + 16) >= (1ll << 31) - 65536) return false;      // (units of a head fit an int)
  const double rows = (double)s.T / s.B, keys = (double)s.keys;
  const double least = std::min((double)s.past, keys), most = std::min((double)s.past + rows, keys), grow = most - least;
  const double seen = rows > 0 ? (grow * (least + most) / 2 + (rows - grow) * keys) / rows : 0;      // of a row, on average
  const double rounds = s.B * std::ceil(rows * s.G / kRowsOfTile) * s.Hkv / 512;
  // (a long sequence among short ones has many of the rows)
  const double longest = std::min((double)s.T, keys - least) * s.G / kRowsOfTile * s.Hkv / 512 * (least + keys) / 2;
  const double alone = (keys - std::max(rounds * seen, longest)) * (keys > 0 ? 1 + 0.75 * least / keys : 1.0);
  const double idle = std::max(alone, rounds > 1 ? 2 * least * (std::ceil(rounds) - rounds) : 0.0);
  return idle >= 36 * kStageKeys;
}
inline size_t prompt_ws(const PromptShape& s, int d) {
  if (!prompt_shared(s)) return 0;
  const int64_t slots = (int64_t)s.T * s.G / kRowsOfTile + s.B;
  return (size_t)prompt_shares(s.Hkv) * s.Hkv * 2 * kRowsOfTile * (d + 2) * sizeof(float) + (size_t)slots * sizeof(int);
}
template <class Src, int D, bool OUT16, class SrcArgs>
int launch_prompt(SrcArgs& a, const char* fn, const PromptShape& shape, hipStream_t st) {
  constexpr int R = kRowsOfTile;
  const int64_t slots = (int64_t)a.bt.T * a.G / R + a.bt.B;
  FL_REQUIRE(slots * a.pg.heads * 4 < (1ll << 31), FL_E_SHAPE, "%s: too many rows", fn);
  a.slots = (int)slots;
  if (!prompt_shared(shape)) {
    prompt_kernel<Src, SrcArgs, false><<<(unsigned)(slots * a.pg.heads), 256, 0, st>>>(a);
    return check_launch("prompt_kernel");
  }
  a.share = prompt_shares(a.pg.heads);
  const size_t places = (size_t)a.share * a.pg.heads * 2 * R;
  a.part_ml = a.part + places * D;
  a.ends = reinterpret_cast<int*>(a.part_ml + places * 2);
  prompt_plan_kernel<SrcArgs, R><<<1, 1024, 0, st>>>(a);
  int rc = check_launch("prompt_plan_kernel");
  if (rc != FL_OK) return rc;
  prompt_kernel<Src, SrcArgs, true><<<(unsigned)(a.share * a.pg.heads), 256, 0, st>>>(a);
  rc = check_launch("prompt_kernel");
  if (rc != FL_OK) return rc;
  prompt_join_kernel<SrcArgs, D, OUT16, R><<<(unsigned)(slots * (R / 32) * a.pg.heads), 256, 0, st>>>(a);
  return check_launch("prompt_join_kernel");
}

}  // namespace fl
