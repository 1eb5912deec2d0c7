// Dense attention of a ragged batch over the paged 4-bit cache: few rows per sequence (single positions), the joining of split keys,
// and the entry points.
#include "fl_paged4_attn.h"
#include "fl_prompt.h"

#include <algorithm>
#include <type_traits>

namespace fl {

constexpr int kKeys4 = 32;         // keys of a wave's tile

// Few rows: a workgroup has R = 16 NR rows of one key/value head (positions and the head's query heads) and a part of the keys;
// its four waves take tiles of 32 keys in turn, each by itself.
//   S^T = K Q^T   v_mfma_f32_16x16x32_f16: a lane loads a quarter of a key's codes as they lie, which are of one group, and widens
//                 them in registers; the contraction runs over the channels in the order that this gives.
//   O^T += V^T P^T  the same product: a lane of S^T holds 2 x 4 keys of one row, which is the P^T operand for keys in that order;
//                 the lane's words of V (8 keys x d / 16 channels) are transposed while they are widened.  Row m of 16 keys is key
//                 4 (m % 4) + m / 4, so that the wave's load of one value a lane takes four neighbouring keys, whole cache lines.
// No LDS in the loop: the next tile's keys are fetched into the registers that the scores leave, its values into those that the
// outputs leave.  Page numbers of 32 tiles are fetched by the lanes at once and handed out by v_readlane.
// What bounds it: memory, and the 300 to 400 vector instructions of a tile close behind (32 sequences of up to 8191 positions, 32 / 8
// heads x 128, int4: 147 MB in 43 us, 3.4 TB/s, vector units busy for 69 % of the cycles; 131072 positions, e2m1: 142 MB in 33 us, 4.3
// TB/s, 55 %), at both ends the chain from the lengths over the block table to the first product, about 9 us (a single sequence of 300).
// Taken against: codes through the caches' default policy (48 and 47 us, 39.8 and 38; windows of 4096 26 and 28.5), the first tile's
// loads ahead of the queries (40.5 and 38).
// fp16 outputs of int4 codes: keys and probabilities are each rounded to fp16 in two parts (widen8_two, pack_rest).  An output has one
// rounding to fp16 of its own; with those of keys, values and probabilities in one part each it would be off by 1.9 times that, with the
// values' alone it is by 1.35 times.
// (Workgroups of a CU: 16 rows three, as there are shares; with four, fp16 queries of 128 channels spill, 58 us for 131072 positions and
// not 37, and bf16 ones gain nothing.  32 rows two; with three 54.5 us for eight sequences of 8000 and not 53.)
template <int D, bool INT, bool F16, int NR>
__global__ __launch_bounds__(256, NR == 1 ? 3 : 2) void paged4_token_kernel(Paged4Args a) {
  constexpr bool TWO = INT && F16;
  constexpr int R = 16 * NR, KS = D / 32, DT = D / 16, NG = D / kGroup, MB = meta_bytes<INT>();
  constexpr int LD = D + 4;               // row stride of the waves' sums in LDS
  __shared__ float s_ref[4][R], s_sum[4][R];
  __shared__ __attribute__((aligned(16))) float s_acc[4][16][LD];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int r16 = lane & 15, g4 = lane >> 4;
  const int kvh = blockIdx.x % a.pg.heads;
  const int slot = blockIdx.x / a.pg.heads;
  const int G = a.G;
  Seq sq;
  Span sp;
  int split = 0;
  if (a.n_split == 1) {
    sq = find_seq(a.bt, slot, 1, [G](int c) { return (int)((int64_t)c * G / R); });
    if (sq.b < 0) return;
    sp = span_of<R, kKeys4>(a, sq, slot - ((int)((int64_t)sq.r0 * G / R) + sq.b));
    cut(sp, 1);
  } else {
    const Shares<R, kKeys4> shares(a);
    int tile;
    sq = shares.find(slot, tile, split);
    if (sq.b < 0) return;
    sp = span_of<R, kKeys4>(a, sq, tile);
    cut(sp, shares.parts(sq.r1 - sq.r0, sq.len));
  }
  if (sp.rows == 0) return;
  const int b = sq.b;
  const int t0 = split * sp.per, t1 = min(t0 + sp.per, sp.tiles);

  // pages of the wave's next 32 tiles: lane l has tile l % 32, key group l / 32
  int pid_v = -1;
  auto fetch_pages = [&](int c0) {
    const int tile = t0 + wave + 4 * (c0 + (lane & 31));
    pid_v = -1;
    if (tile < t1) {
      const int page = (key_of<kKeys4>(sp, tile) + (lane >> 5) * 16) >> a.pg.log2;
      if (page < a.bt.max_pages) pid_v = a.bt.table[(int64_t)b * a.bt.max_pages + page];
      if ((uint32_t)pid_v >= (uint32_t)a.pg.num) pid_v = -1;
    }
  };
  fetch_pages(0);

  // the lane's rows
  f16x8 qf[NR][KS], ql[NR][F16 ? KS : 1];
  float mul[NR];
  int jmax[NR], jmin[NR];
  const int cap = a.bt.max_pages * a.pg.size;
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int rr = x * 16 + r16;
    const bool ok = rr < sp.rows;
    const int rho = sp.rho0 + (ok ? rr : 0);
    const int t = rho / G, pos = sp.start + t;
    const uint16_t* src = a.q + (int64_t)(sp.r0 + t) * a.qs + (int64_t)(kvh * G + rho % G) * D;
    // (the order in which keys lie in the lanes)
    mul[x] = load_query<KS, F16>(a, src, ok, pos, cap, qf[x], ql[x], [g4](int k) { return KS * g4 + k; },
                                 [](float m) { return row4_max(m); });
    mul[x] = finite_factor<KS>(mul[x], qf[x]);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[x][k] = in_order<INT>(qf[x][k]);
      if constexpr (F16) ql[x][k] = in_order<INT>(ql[x][k]);
    }
    jmax[x] = ok ? min(pos, cap - 1) : -1;
    jmin[x] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  }
  // a tile that every row sees in full needs no mask: its keys are at most all_max and at least all_min (or leading)
  const int all_max = sp.i_min, all_min = a.window > 0 && sp.i_max >= a.window ? sp.i_max - a.window + 1 : 0;

  f32x4 acc[NR][DT];
  float ref[NR], lsum[NR];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    ref[x] = -INFINITY;
    lsum[x] = 0.0f;
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[x][t] = f32x4{};
  }

  uint32_t wk[2][KS], mk[2], mkv[2];                         // the tile's codes of the lane, the group's numbers, the values' ones
  uint32_t wv[8];
  const Magic magic;
  // lane offsets; the lane that has the numbers of the lane's first value
  const int key = 4 * (r16 & 3) + (r16 >> 2);
  const uint32_t k_at = (uint32_t)(key * (D / 2) + g4 * (D / 8)), m_at = (uint32_t)(key * NG + g4 * NG / 4) * MB;
  const uint32_t v_at = (uint32_t)(g4 * (D / 2) + (DT == 8 ? r16 * 4 : (r16 >> 1) * 4));
  const int from = 4 * (4 * g4 + 16 * (DT == 8 ? r16 >> 2 : 2 * (r16 >> 3)));
  auto base_of = [&](int c, int h) {                         // row of key group h of the wave's tile c
    const int key0 = key_of<kKeys4>(sp, t0 + wave + 4 * c);
    const int p = max(__builtin_amdgcn_readlane(pid_v, (c & 31) + 32 * h), 0);        // (a page that is not there: masked)
    return ((int64_t)p * a.pg.heads + kvh) * a.pg.size + ((key0 + 16 * h) & (a.pg.size - 1));
  };
  auto load_k = [&](int c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t row = base_of(c, h);
      const uint8_t* kb = a.kc + row * (D / 2);
      if constexpr (KS == 4) {
        const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kb + k_at));
#pragma unroll
        for (int k = 0; k < 4; ++k) wk[h][k] = w[k];
      } else {
        const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(kb + k_at));
        wk[h][0] = w[0];
        wk[h][1] = w[1];
      }
      mk[h] = load_meta<INT>(a.km + row * (NG * MB) + m_at);
      mkv[h] = load_meta<INT>(a.vm + row * (NG * MB) + m_at);
    }
  };
  auto load_v = [&](int c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* vb = a.vc + base_of(c, h) * (D / 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) wv[4 * h + e] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(vb + 4 * e * (D / 2) + v_at));
    }
  };
  auto compute = [&](int c, bool more) {
    const int key0 = key_of<kKeys4>(sp, t0 + wave + 4 * c);
    const int pid0 = __builtin_amdgcn_readlane(pid_v, c & 31), pid1 = __builtin_amdgcn_readlane(pid_v, (c & 31) + 32);
    const bool masked = key0 + kKeys4 - 1 > all_max || (key0 < all_min && key0 + kKeys4 > a.n_sink) || (pid0 | pid1) < 0;
    // a group that reads as NaN, of the key or the value, makes the key's scores NaN; the value's counts as 0
    uint32_t bad[2];
    bool fine = true;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool ok = group_ok<INT>(mkv[h]);
      bad[h] = ok & group_ok<INT>(mk[h]) ? 0u : 0x7E007E00u;
      fine &= ok;
    }
    const bool spoilt = __builtin_amdgcn_ballot_w64(!fine) != 0;      // uniform
    // the values' numbers go from the lane that has loaded them to those that have the values
    uint32_t mv[8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) mv[4 * h + e] = (uint32_t)__builtin_amdgcn_ds_bpermute(from + 4 * e, (int)mkv[h]);
    f32x4 s[NR][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int x = 0; x < NR; ++x) s[x][h] = f32x4{};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32x4 w, rest;
        if constexpr (TWO) widen8_two(wk[h][k], mk[h], magic, w, rest);
        else w = widen8<INT>(wk[h][k], mk[h], magic);
        if (k == 0) w[0] |= bad[h];
        const f16x8 kf = __builtin_bit_cast(f16x8, w);
        if constexpr (TWO) {
#pragma unroll
          for (int x = 0; x < NR; ++x) s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, rest), qf[x][k], s[x][h], 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < NR; ++x) s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[x][k], s[x][h], 0, 0, 0);
        if constexpr (F16)
          if (a.rt.table) {
#pragma unroll
            for (int x = 0; x < NR; ++x) s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, ql[x][k], s[x][h], 0, 0, 0);
          }
      }
    }
    if (more) load_k(c + 1);
    f16x8 pf[NR], pl[TWO ? NR : 1];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      f32x4(&y)[2] = s[x];
      if (masked) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = key0 + 16 * h + 4 * i + g4;
            const bool see = (j <= jmax[x]) & ((j >= jmin[x]) | (j < a.n_sink)) & ((h ? pid1 : pid0) >= 0);
            y[h][i] = see ? y[h][i] : -INFINITY;
          }
      }
      const float most = mul[x] * row4_max(max3(max3(y[0][0], y[0][1], y[0][2]), max3(y[0][3], y[1][0], y[1][1]), max3(y[1][2], y[1][3], y[1][3])));
      const bool raise = most > ref[x] + 8.0f;
      if (__builtin_amdgcn_ballot_w64(raise) != 0) {
        const float nm = raise ? most : ref[x];
        const float alpha = raise ? __builtin_amdgcn_exp2f(ref[x] - nm) : 1.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[x][t] *= alpha;
        lsum[x] *= alpha;
        ref[x] = nm;
      }
      const float base = ref[x] == -INFINITY ? 0.0f : ref[x];
      float p[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[h][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[h][i], mul[x], -base));
      lsum[x] += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
      const u32x4 pw = {pack_f16x2(p[0][0], p[0][1]), pack_f16x2(p[0][2], p[0][3]), pack_f16x2(p[1][0], p[1][1]),
                        pack_f16x2(p[1][2], p[1][3])};
      pf[x] = __builtin_bit_cast(f16x8, pw);
      if constexpr (TWO)
        pl[x] = __builtin_bit_cast(f16x8, u32x4{pack_rest(p[0][0], p[0][1], pw[0]), pack_rest(p[0][2], p[0][3], pw[1]),
                                                pack_rest(p[1][0], p[1][1], pw[2]), pack_rest(p[1][2], p[1][3], pw[3])});
    }
    if (__builtin_expect(spoilt, 0)) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!group_ok<INT>(mv[e])) wv[e] = mv[e] = 0;
    }
    if constexpr (DT == 4) {                                 // the lane's half of a word
#pragma unroll
      for (int e = 0; e < 8; ++e) wv[e] = r16 & 1 ? wv[e] >> 16 : wv[e];
    }
    auto pair_of = [&](auto byte) {                          // channels 2 y and the next of the lane, eight keys
      constexpr int y = decltype(byte)::value;
      u32x4 va, vb;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (INT) {
          const f16x2 sc = both_low(mv[2 * e], mv[2 * e + 1]), z = both_high(mv[2 * e], mv[2 * e + 1]);
          const uint32_t two = __builtin_amdgcn_perm(wv[2 * e + 1], wv[2 * e], 0x0c000c00u | (uint32_t)(4 + y) << 16 | (uint32_t)y);
          va[e] = apply(low_pair(two, magic), sc, z);
          vb[e] = apply(high_pair(two, magic), sc, z);
        } else {
          const uint32_t p0 = widen_byte<y>(wv[2 * e], __uint_as_float(mv[2 * e] << 23));
          const uint32_t p1 = widen_byte<y>(wv[2 * e + 1], __uint_as_float(mv[2 * e + 1] << 23));
          va[e] = __builtin_amdgcn_perm(p1, p0, 0x05040100u);
          vb[e] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
        }
      }
#pragma unroll
      for (int x = 0; x < NR; ++x) {
        acc[x][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, va), pf[x], acc[x][2 * y], 0, 0, 0);
        acc[x][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, vb), pf[x], acc[x][2 * y + 1], 0, 0, 0);
        if constexpr (TWO) {
          acc[x][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, va), pl[x], acc[x][2 * y], 0, 0, 0);
          acc[x][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, vb), pl[x], acc[x][2 * y + 1], 0, 0, 0);
        }
      }
    };
    pair_of(std::integral_constant<int, 0>{});
    pair_of(std::integral_constant<int, 1>{});
    if constexpr (DT == 8) {
      pair_of(std::integral_constant<int, 2>{});
      pair_of(std::integral_constant<int, 3>{});
    }
  };

  const int mine = t1 - t0 - wave <= 0 ? 0 : (t1 - t0 - wave + 3) / 4;     // tiles of this wave
  for (int c0 = 0; c0 < mine; c0 += 32) {
    if (c0 > 0) fetch_pages(c0);
    const int c1 = min(c0 + 32, mine);
    load_k(c0);
    load_v(c0);
    for (int c = c0; c < c1; ++c) {
      compute(c, c + 1 < c1);
      if (c + 1 < c1) load_v(c + 1);
    }
  }

  // the four waves' states of a row meet in LDS (the lane's place is formed anew: kept over the loop, it spilled)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  r16 = tid & 15;
  g4 = (tid & 63) >> 4;
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    lsum[x] = row4_add(lsum[x]);
    if (g4 == 0) {
      s_ref[wave][x * 16 + r16] = ref[x];
      s_sum[wave][x * 16 + r16] = lsum[x];
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int rr = x * 16 + r16;
    const float m = fmaxf(fmaxf(s_ref[0][rr], s_ref[1][rr]), fmaxf(s_ref[2][rr], s_ref[3][rr]));
    const float f = ref[x] == -INFINITY ? (lsum[x] == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(ref[x] - m);
    if (x > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)                              // channels (4 g4 + i) DT + t, t < DT
#pragma unroll
      for (int t = 0; t < DT; t += 4)
        *reinterpret_cast<float4*>(&s_acc[wave][r16][(4 * g4 + i) * DT + t]) =
            make_float4(acc[x][t][i] * f, acc[x][t + 1][i] * f, acc[x][t + 2][i] * f, acc[x][t + 3][i] * f);
    __syncthreads();
    constexpr int CPR = D / 4;                               // four channels a thread
    for (int w = tid; w < 16 * CPR; w += 256) {
      const int row = w / CPR, c = (w % CPR) * 4, rx = x * 16 + row;
      if (rx >= sp.rows) continue;
      const float mm = fmaxf(fmaxf(s_ref[0][rx], s_ref[1][rx]), fmaxf(s_ref[2][rx], s_ref[3][rx]));
      float sum = 0.0f;
#pragma unroll
      for (int v = 0; v < 4; ++v)                            // (a sum of NaN scores has no reference, but counts)
        sum += s_ref[v][rx] == -INFINITY ? s_sum[v][rx] : s_sum[v][rx] * __builtin_amdgcn_exp2f(s_ref[v][rx] - mm);
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (s_acc[0][row][c + e] + s_acc[1][row][c + e]) + (s_acc[2][row][c + e] + s_acc[3][row][c + e]);
      const int rho = sp.rho0 + rx, t = rho / G, h = kvh * G + rho % G;
      const int64_t gr = (int64_t)(sp.r0 + t) * a.Hq + h;
      if (sp.parts > 1) {
        const int64_t at = (int64_t)blockIdx.x * R + rx;
        *reinterpret_cast<float4*>(a.part + at * D + c) = make_float4(o[0], o[1], o[2], o[3]);
        if (c == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mm, sum);
      } else {
        const bool none = mm == -INFINITY && sum == 0.0f;
        const float inv = none ? 0.0f : 1.0f / sum;
        const u32x2 two = {F16 ? pack_f16x2(o[0] * inv, o[1] * inv) : pack_bf16x2(o[0] * inv, o[1] * inv),
                           F16 ? pack_f16x2(o[2] * inv, o[3] * inv) : pack_bf16x2(o[2] * inv, o[3] * inv)};
        *reinterpret_cast<u32x2*>(a.o + (int64_t)(sp.r0 + t) * a.os + (int64_t)h * D + c) = two;
        if (c == 0 && a.lse) a.lse[gr] = none ? -INFINITY : (mm + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
      }
    }
  }
}

// The parts of a row's keys joined: a workgroup a row, d / 4 threads across its channels and 1024 / d groups that take the
// parts in turn, so that the loads of one part are never waited for before those of the next.
// (1024 rows of about 4 parts 5.3 us, 32 rows of 96 4.7: a launch and two rounds of loads)
constexpr int kMaxSplit = 256;
template <int D, int R, bool F16>
__global__ __launch_bounds__(256) void paged4_merge_kernel(Paged4Args a) {
  constexpr int LN = D / 4, NG = 256 / LN;
  __shared__ float s_f[kMaxSplit], s_w[2][4];
  __shared__ float4 s_o[NG][LN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
  const Seq sq = find_seq(a.bt, t, 0, [](int c) { return c; });
  if (sq.b < 0 || t >= sq.r1) return;
  const Shares<R, kKeys4> shares(a);
  const int parts = shares.parts(sq.r1 - sq.r0, sq.len);
  if (parts <= 1) return;
  const int rho = (t - sq.r0) * a.G + h % a.G;
  const int item = shares.before(sq.b) + rho / R * parts;    // the row tile's first; the parts follow
  if (item < 0 || item + parts > a.slots) return;            // (offsets that do not ascend: nothing was written)
  const int64_t first = ((int64_t)item * a.pg.heads + h / a.G) * R + rho % R, step = (int64_t)a.pg.heads * R;
  float2 w = make_float2(-INFINITY, 0.0f);                   // ref, normaliser
  if ((int)threadIdx.x < parts) w = reinterpret_cast<const float2*>(a.part_ml)[first + threadIdx.x * step];
  float m = w.x;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if (lane == 0) s_w[0][wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_w[0][0], s_w[0][1]), fmaxf(s_w[0][2], s_w[0][3]));
  const float f = w.x == -INFINITY ? (w.y == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(w.x - m);
  float sum = f * w.y;
  s_f[threadIdx.x] = f;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
  if (lane == 0) s_w[1][wave] = sum;
  __syncthreads();
  sum = (s_w[1][0] + s_w[1][1]) + (s_w[1][2] + s_w[1][3]);
  const int c = threadIdx.x % LN, grp = threadIdx.x / LN;
  const float4* src = reinterpret_cast<const float4*>(a.part + first * D) + c;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int s = grp; s < parts; s += NG) {
    const float4 x = src[s * step * LN];
    const float g = s_f[s];
    o.x = fmaf(g, x.x, o.x);
    o.y = fmaf(g, x.y, o.y);
    o.z = fmaf(g, x.z, o.z);
    o.w = fmaf(g, x.w, o.w);
  }
  s_o[grp][c] = o;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int s = 1; s < NG; ++s) {
    const float4 x = s_o[s][c];
    o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
  }
  const bool none = m == -INFINITY && sum == 0.0f;
  const float inv = none ? 0.0f : 1.0f / sum;
  *reinterpret_cast<u32x2*>(a.o + (int64_t)t * a.os + (int64_t)h * D + 4 * c) =
      u32x2{F16 ? pack_f16x2(o.x * inv, o.y * inv) : pack_bf16x2(o.x * inv, o.y * inv),
            F16 ? pack_f16x2(o.z * inv, o.w * inv) : pack_bf16x2(o.z * inv, o.w * inv)};
  if (a.lse && c == 0) a.lse[blockIdx.x] = none ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// Work items of a head: row tiles, and with split keys as many parts more as the tiles are shared out to.
static int64_t items_of(int T, int G, int B, int Hkv, int rows, int n_split, int share) {
  return (int64_t)T * G / rows + B + (n_split > 1 ? share / Hkv + 1 : 0);
}

template <int NR>
static int launch_token4(const Paged4Args& args, int d, int format, bool f16, hipStream_t st) {
  Paged4Args a = args;
  const int64_t items = items_of(a.bt.T, a.G, a.bt.B, a.pg.heads, 16 * NR, a.n_split, a.share), n = items * a.pg.heads;
  FL_REQUIRE(n < (1ll << 31), FL_E_SHAPE, "fl_paged4_attn: too many rows");
  a.slots = (int)items;
  a.part_ml = a.part ? a.part + n * 16 * NR * d : nullptr;
  const unsigned grid = (unsigned)n;
#define FL_TOKEN(DD)                                                                         \
  do {                                                                                       \
    if (format == FL_KV4_INT) {                                                              \
      if (f16) paged4_token_kernel<DD, true, true, NR><<<grid, 256, 0, st>>>(a);             \
      else paged4_token_kernel<DD, true, false, NR><<<grid, 256, 0, st>>>(a);                \
    } else {                                                                                 \
      if (f16) paged4_token_kernel<DD, false, true, NR><<<grid, 256, 0, st>>>(a);            \
      else paged4_token_kernel<DD, false, false, NR><<<grid, 256, 0, st>>>(a);               \
    }                                                                                        \
  } while (0)
  if (d == 128) FL_TOKEN(128);
  else FL_TOKEN(64);
#undef FL_TOKEN
  const int rc = check_launch("paged4_token_kernel");
  if (rc != FL_OK || a.n_split == 1) return rc;
  const unsigned rows = (unsigned)((int64_t)a.bt.T * a.Hq);
  if (d == 128) {
    if (f16) paged4_merge_kernel<128, 16 * NR, true><<<rows, 256, 0, st>>>(a);
    else paged4_merge_kernel<128, 16 * NR, false><<<rows, 256, 0, st>>>(a);
  } else {
    if (f16) paged4_merge_kernel<64, 16 * NR, true><<<rows, 256, 0, st>>>(a);
    else paged4_merge_kernel<64, 16 * NR, false><<<rows, 256, 0, st>>>(a);
  }
  return check_launch("paged4_merge_kernel");
}

// How a call is cut: up to 32 rows of a key/value head in a sequence (up to 64 where sequences and heads are few) the kernel for few
// rows, whose keys are split while sequences and heads alone are fewer than its shares, in parts of kLeastTiles tiles or more; more rows
// the kernel for prompts.  (32 / 8 heads x 128, int4.  16 rows after each of eight times 4000 positions: 23 us, and 32 in the form for 32
// rows.  32 rows after eight times 32000: 101 us, in the form for 16 rows 123, in the kernel for prompts 167.  64 rows after one, four
// and eight contexts of 4000, 2000 and 32000: 18, 24 and 178 us, in the kernel for prompts 36, 35 and 175; after 32 of 4000 123 and
// 102.  Shares: 512 and 1024 take 49 and 52 us for 32 sequences where 768 take 47, 39 and 44 for 131072 positions where 768 take 37.
// Least tiles: 4 and 16 take 73 and 71 us for eight sequences of 32000 where 8 take 70, and are within 5 % elsewhere.)
constexpr int kShare = 768, kLeastTiles = 8;
struct Plan4 {
  int rows, n_split, min_tiles, share;
  PromptShape shape;              // (the kernel for prompts)
  size_t ws;
};
static Plan4 plan4_of(int B, int T, int Hq, int Hkv, int d, int page, int max_pages, int window, int n_sink, int max_q, int max_len) {
  Plan4 p{};
  const int64_t G = Hq / Hkv;
  const int64_t per_seq = std::max<int64_t>(1, std::min<int64_t>(max_q > 0 ? max_q : 1, T)) * G;
  p.rows = per_seq <= 16 ? 16 : per_seq <= ((int64_t)B * Hkv <= 128 ? 64 : 32) ? 32 : 128;
  const int64_t cap = (int64_t)max_pages * page;
  int64_t len = max_len > 0 ? std::min<int64_t>(max_len, cap) : cap;
  const int64_t past = std::max<int64_t>(0, len - T / B);
  if (window > 0) len = std::min<int64_t>(len, (int64_t)window + n_sink + std::max(max_q, 1));
  p.n_split = p.min_tiles = 1;
  if (p.rows == 128) {
    p.shape = {B, T, (int)G, Hkv, past, len, cap};
    p.ws = paged4_prompt_ws(p.shape, d);
    return p;
  }
  const int64_t tiles = std::max<int64_t>(1, (len + kKeys4 - 1) / kKeys4);
  const int64_t units = std::max<int64_t>(1, std::max<int64_t>(B, T * G / p.rows)) * Hkv;
  p.share = kShare;
  p.min_tiles = kLeastTiles;
  const int64_t split = units < kShare ? std::min<int64_t>(std::max<int64_t>(tiles / kLeastTiles, 1), kMaxSplit) : 1;
  p.n_split = (int)split;
  // (a place for each row of each work item, however long the contexts are)
  p.ws = split > 1 ? (size_t)items_of(T, (int)G, B, Hkv, p.rows, p.n_split, p.share) * Hkv * p.rows * (d + 2) * sizeof(float) : 0;
  return p;
}

}  // namespace fl

using namespace fl;

extern "C" size_t fl_paged4_attn_ws(int B, int T, int Hq, int Hkv, int d, int page, int max_pages, int window, int n_sink,
                                    int max_q, int max_len) {
  if (B < 1 || T < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv || (d != 64 && d != 128) || page < 16 || max_pages < 1 || window < 0 ||
      n_sink < 0 || max_q < 0 || max_len < 0)
    return 0;
  return plan4_of(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len).ws;
}

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
  const Plan4 p = plan4_of(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len);
  FL_REQUIRE(p.ws == 0 || (ws && ws_bytes >= p.ws), FL_E_WORKSPACE, "%s: workspace of %zu bytes required", fn, p.ws);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 15) == 0, FL_E_SHAPE, "%s: ws must be 16-byte aligned", fn);
  hipStream_t st = as_stream(stream);
  Paged4Args a{};
  a.q = static_cast<const uint16_t*>(q); a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.os = o_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<const uint8_t*>(k_cache); a.vc = static_cast<const uint8_t*>(v_cache);
  a.km = static_cast<const uint8_t*>(k_meta); a.vm = static_cast<const uint8_t*>(v_meta);
  a.Hq = Hq; a.G = Hq / Hkv; a.scale_log2 = sm_scale * 1.4426950408889634f; a.window = window; a.n_sink = n_sink;
  a.n_split = p.n_split; a.min_tiles = p.min_tiles; a.share = p.share;
  a.part = static_cast<float*>(ws);
  rc = check_batch(fn, a.bt, a.pg, false, st);
  if (rc != FL_OK) return rc;
  if (p.rows == 16) return launch_token4<1>(a, d, format, dtype == FL_F16, st);
  if (p.rows == 32) return launch_token4<2>(a, d, format, dtype == FL_F16, st);
  return launch_paged4_prompt(a, d, format, dtype == FL_F16, p.shape, st);
  FL_API_END
}
