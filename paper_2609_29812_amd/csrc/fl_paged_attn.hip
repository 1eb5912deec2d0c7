// Dense attention of a ragged batch over the paged 8-bit cache: few rows per sequence (single positions), the joining of
// split keys, and the entry points.
#include "fl_paged_attn.h"

#include <algorithm>

namespace fl {

constexpr int kTokenKeys = 32;     // keys of a wave's tile

// Few rows: a workgroup has R = 16 NR rows of one key/value head (positions and the head's query heads) and a part of the
// keys; its four waves take tiles of 32 keys in turn, each by itself.
//   S^T = K Q^T   v_mfma_f32_16x16x32_f16: a lane loads a quarter of a key's codes as they lie, widened in registers to exact
//                 fp16; the contraction runs over the channels in the order that this gives.
//   O^T += V^T P^T  the same product: a lane of S^T holds 2 x 4 keys of one row, which is the P^T operand for keys in that
//                 order; the lane's V bytes (8 keys x d / 16 channels) are transposed by byte permutes while they are widened.
// No LDS in the loop: the next tile's keys are fetched into the registers that the scores leave, its values into those that the
// outputs leave.  Page numbers and scales of 32 tiles are fetched by the lanes at once and handed out by v_readlane.  Each code is
// read once, non-temporally (131072 positions: 53 us against 60 under the default policy).
//
// Bound by HBM for long contexts, by the chain of loads before the first product (sequences; pages and queries; scales and codes)
// for short ones.  8 heads x 128: 131072 positions of one sequence 50 us, 5.4 TB/s; 32 sequences of 1 to 8191 positions 53 us, 4.5
// TB/s (64 us with the same number of parts for every sequence); 16 heads, 299 positions 9.5 us.
template <int D, bool I8, bool F16, int NR>
__global__ __launch_bounds__(256, NR == 1 ? (F16 ? 3 : 4) : 2) void paged_token_kernel(PagedAttnArgs a) {
  constexpr int R = 16 * NR, KS = D / 32, DT = D / 16;
  constexpr int KW = D / 64;              // 16-byte loads of a lane per key group
  constexpr int VW = D / 64;              // words of a lane per key of V
  constexpr int LD = D + 4;               // row stride of the waves' sums in LDS
  __shared__ float s_ref[4][R], s_top[4][R], s_sum[4][R];
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
    sq = find_seq(a.bt, slot, 1, [G](int c) { return c * G / R; });
    if (sq.b < 0) return;
    sp = span_of<R, kTokenKeys>(a, sq, slot - (sq.r0 * G / R + sq.b));
    cut(sp, 1);
  } else {
    const Shares<R, kTokenKeys> shares(a);
    int tile;
    sq = shares.find(slot, tile, split);
    if (sq.b < 0) return;
    sp = span_of<R, kTokenKeys>(a, sq, tile);
    cut(sp, shares.parts(sq.r1 - sq.r0, sq.len));
  }
  if (sp.rows == 0) return;
  const int b = sq.b;
  const int t0 = split * sp.per, t1 = min(t0 + sp.per, sp.tiles);

  // pages and scales of the wave's next 32 tiles: lane l has tile l % 32, key group l / 32.  The pages are asked for before the
  // queries, and their scales before the first codes but waited for after them.
  int pid_v = -1;
  float ks_v = 0.0f, lv_v = 1.0f, iv_v = 0.0f;
  auto fetch_pages = [&](int c0) {
    const int tile = t0 + wave + 4 * (c0 + (lane & 31));
    pid_v = -1;
    if (tile < t1) {
      const int page = (key_of<kTokenKeys>(sp, tile) + (lane >> 5) * 16) >> a.pg.log2;
      if (page < a.bt.max_pages) pid_v = a.bt.table[(int64_t)b * a.bt.max_pages + page];
    }
  };
  auto fetch_scales = [&] {
    const bool there = (uint32_t)pid_v < (uint32_t)a.pg.num;
    pid_v = there ? pid_v : -1;
    const int64_t at = (int64_t)max(pid_v, 0) * a.pg.heads + kvh;
    ks_v = a.ksc[at];
    lv_v = a.vsc[at];
  };
  auto use_scales = [&] {
    const ValueScale vs = value_scale(pid_v < 0 ? 1.0f : lv_v);
    ks_v = pid_v < 0 ? 0.0f : key_scale(ks_v);
    lv_v = vs.log2;
    iv_v = vs.inv;
  };
  fetch_pages(0);

  // the lane's rows
  f16x8 qf[NR][KS], ql[NR][F16 ? KS : 1];
  float mul[NR];
  int jmax[NR], jmin[NR];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int rr = x * 16 + r16;
    const bool ok = rr < sp.rows;
    const int rho = sp.rho0 + (ok ? rr : 0);
    const int t = rho / G, pos = sp.start + t;
    const uint16_t* src = a.q + (int64_t)(sp.r0 + t) * a.qs + (int64_t)(kvh * G + rho % G) * D;
    const int cap = a.bt.max_pages * a.pg.size;
    // (the order in which keys lie in the lanes)
    mul[x] = load_query<KS, F16>(a, src, ok, pos, cap, qf[x], ql[x], [g4](int k) { return 8 * (k / 2) + 2 * g4 + k % 2; },
                                 [](float m) { return row4_max(m); });
    jmax[x] = ok ? min(pos, cap - 1) : -1;
    jmin[x] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  }
  // a tile that every row sees in full needs no mask: its keys are at most all_max and at least all_min (or leading)
  const int all_max = sp.i_min, all_min = a.window > 0 && sp.i_max >= a.window ? sp.i_max - a.window + 1 : 0;

  f32x4 acc[NR][DT];
  float ref[NR], top[NR], lsum[NR];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    ref[x] = top[x] = -INFINITY;
    lsum[x] = 0.0f;
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[x][t] = f32x4{};
  }

  u32x4 wk[2][KW];                                           // the tile's codes of the lane
  uint32_t wv[8][VW];
  auto base_of = [&](int c, int h) {                         // first code of key group h of the wave's tile c
    const int key0 = key_of<kTokenKeys>(sp, t0 + wave + 4 * c);
    const int p = max(__builtin_amdgcn_readlane(pid_v, (c & 31) + 32 * h), 0);        // (a page that is not there: masked)
    return (((int64_t)p * a.pg.heads + kvh) * a.pg.size + ((key0 + 16 * h) & (a.pg.size - 1))) * D;
  };
  auto load_k = [&](int c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* kb = a.kc + base_of(c, h);
#pragma unroll
      for (int x = 0; x < KW; ++x) wk[h][x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kb + (uint32_t)(r16 * D + 64 * x + 16 * g4)));
    }
  };
  auto load_v = [&](int c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* vb = a.vc + base_of(c, h);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t at = (uint32_t)((g4 * 4 + e) * D + r16 * DT);
        if constexpr (VW == 2) {
          const u32x2 d2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(vb + at));
          wv[4 * h + e][0] = d2[0];
          wv[4 * h + e][1] = d2[1];
        } else {
          wv[4 * h + e][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(vb + at));
        }
      }
    }
  };
  auto compute = [&](int c, bool more) {
    const int key0 = key_of<kTokenKeys>(sp, t0 + wave + 4 * c);
    const int pid0 = __builtin_amdgcn_readlane(pid_v, c & 31), pid1 = __builtin_amdgcn_readlane(pid_v, (c & 31) + 32);
    float ks[2], lv[2], iv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ks[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_v), (c & 31) + 32 * h));
      lv[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lv_v), (c & 31) + 32 * h));
      iv[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(iv_v), (c & 31) + 32 * h));
    }
    const bool spoilt = iv[0] < 0.0f || iv[1] < 0.0f;
    const float least = fminf(lv[0], lv[1]);
    const bool masked = key0 + kTokenKeys - 1 > all_max || (key0 < all_min && key0 + kTokenKeys > a.n_sink) || (pid0 | pid1) < 0;
    f32x4 s[NR][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int x = 0; x < NR; ++x) s[x][h] = f32x4{};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32x4 kw;
        uint32_t two[2];
        widen4<I8>(wk[h][k / 2][2 * (k % 2)], two);
        kw[0] = two[0]; kw[1] = two[1];
        widen4<I8>(wk[h][k / 2][2 * (k % 2) + 1], two);
        kw[2] = two[0]; kw[3] = two[1];
#pragma unroll
        for (int x = 0; x < NR; ++x)
          s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kw), qf[x][k], s[x][h], 0, 0, 0);
        if constexpr (F16)
          if (a.rt.table) {
#pragma unroll
            for (int x = 0; x < NR; ++x)
              s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kw), ql[x][k], s[x][h], 0, 0, 0);
          }
      }
    }
    if (more) load_k(c + 1);
    if (__builtin_expect((masked && !I8) || least <= kNoScale, 0)) {              // codes that no row sees may be NaN; those of a scale of 0 count as 0
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool there = seen_by_any(a, sp, key0 + (e >> 2) * 16 + g4 * 4 + (e & 3)) && (e < 4 ? pid0 : pid1) >= 0 &&
                           lv[e >> 2] > kNoScale;
#pragma unroll
        for (int y = 0; y < VW; ++y) wv[e][y] = there ? wv[e][y] : 0u;
      }
    }
    f16x8 pf[NR];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      float y[2][4], most = -INFINITY;                       // scores; the largest contribution
      bool see[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float m = ks[h] * mul[x];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[h][i] = s[x][h][i] * m;
        if (masked) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = key0 + 16 * h + 4 * g4 + i;
            see[h][i] = (j <= jmax[x]) & ((j >= jmin[x]) | (j < a.n_sink)) & ((h ? pid1 : pid0) >= 0);
            y[h][i] = see[h][i] ? y[h][i] : -INFINITY;
          }
        }
        most = fmaxf(most, max3(max3(y[h][0], y[h][1], y[h][2]), y[h][3], y[h][3]) + lv[h]);
      }
      most = row4_max(most);
      auto best = [&] {                                      // the largest score
        return row4_max(max3(max3(y[0][0], y[0][1], y[0][2]), max3(y[0][3], y[1][0], y[1][1]), max3(y[1][2], y[1][3], y[1][3])));
      };
      auto lift = [&](float to) {                            // the normaliser in units of a larger 2^top
        if (to > top[x]) {
          lsum[x] *= __builtin_amdgcn_exp2f(top[x] - to);
          top[x] = to;
        }
      };
      const bool raise = most > ref[x] + 8.0f;
      if (__builtin_amdgcn_ballot_w64(raise) != 0) {
        const float nm = raise ? most : ref[x];
        const float alpha = raise ? __builtin_amdgcn_exp2f(ref[x] - nm) : 1.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[x][t] *= alpha;
        ref[x] = nm;
        lift(best());
      }
      const float base = ref[x] == -INFINITY ? 0.0f : ref[x];
      const bool apart = __builtin_amdgcn_ballot_w64(ref[x] - top[x] - least > kRoom) != 0;
      if (__builtin_expect(apart, 0)) {                      // (out of the way of the loop's code)
        lift(best());
        const float from = top[x] == -INFINITY ? 0.0f : top[x];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) lsum[x] += __builtin_amdgcn_exp2f(y[h][i] - from);
      }
      float p[2][4], sum = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float off = lv[h] - base;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[h][i] = __builtin_amdgcn_exp2f(y[h][i] + off);
        }
        const float part = (p[h][0] + p[h][1]) + (p[h][2] + p[h][3]);
        sum = fmaf(part, fabsf(iv[h]), sum);
      }
      lsum[x] = fmaf(sum, apart ? 0.0f : ref_to_top(ref[x], top[x]), lsum[x]);
      if (__builtin_expect(spoilt, 0)) {                                          // a value scale that is not finite: the rows that see it
        bool any = false;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) any |= iv[h] < 0.0f && (!masked || see[h][i]);
        const float bad = row4_add(any ? 1.0f : 0.0f) > 0.0f ? NAN : 0.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[x][t] += bad;
      }
      const u32x4 pw = {pack_f16x2(p[0][0], p[0][1]), pack_f16x2(p[0][2], p[0][3]), pack_f16x2(p[1][0], p[1][1]),
                        pack_f16x2(p[1][2], p[1][3])};
      pf[x] = __builtin_bit_cast(f16x8, pw);
    }
#pragma unroll
    for (int y = 0; y < VW; ++y)
#pragma unroll
      for (int u = 0; u < 2; ++u) {                          // channels 4 y + 2 u and the next of the lane, eight keys
        u32x4 va, vb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t two[2];
          widen4<I8>(__builtin_amdgcn_perm(wv[2 * e + 1][y], wv[2 * e][y], u ? 0x07030602u : 0x05010400u), two);
          va[e] = two[0];
          vb[e] = two[1];
        }
#pragma unroll
        for (int x = 0; x < NR; ++x) {
          const int t = 4 * y + 2 * u;
          acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, va), pf[x], acc[x][t], 0, 0, 0);
          acc[x][t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, vb), pf[x], acc[x][t + 1], 0, 0, 0);
        }
      }
  };

  const int mine = t1 - t0 - wave <= 0 ? 0 : (t1 - t0 - wave + 3) / 4;     // tiles of this wave
  for (int c0 = 0; c0 < mine; c0 += 32) {
    if (c0 > 0) fetch_pages(c0);
    fetch_scales();
    const int c1 = min(c0 + 32, mine);
    load_k(c0);
    load_v(c0);
    use_scales();
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
      s_top[wave][x * 16 + r16] = top[x];
      s_sum[wave][x * 16 + r16] = lsum[x];
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int rr = x * 16 + r16;
    const float m = fmaxf(fmaxf(s_ref[0][rr], s_ref[1][rr]), fmaxf(s_ref[2][rr], s_ref[3][rr]));
    const float f = ref[x] == -INFINITY && lsum[x] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ref[x] - m);
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
      const float mt = fmaxf(fmaxf(s_top[0][rx], s_top[1][rx]), fmaxf(s_top[2][rx], s_top[3][rx]));
      float sum = 0.0f;
#pragma unroll
      for (int v = 0; v < 4; ++v)                            // (a sum of NaN scores has no reference, but counts)
        sum += s_top[v][rx] == -INFINITY && s_sum[v][rx] == 0.0f ? 0.0f : s_sum[v][rx] * __builtin_amdgcn_exp2f(s_top[v][rx] - mt);
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (s_acc[0][row][c + e] + s_acc[1][row][c + e]) + (s_acc[2][row][c + e] + s_acc[3][row][c + e]);
      const int rho = sp.rho0 + rx, t = rho / G, h = kvh * G + rho % G;
      const int64_t gr = (int64_t)(sp.r0 + t) * a.Hq + h;
      if (sp.parts > 1) {
        const int64_t at = (int64_t)blockIdx.x * R + rx;
        *reinterpret_cast<float4*>(a.part + at * D + c) = make_float4(o[0], o[1], o[2], o[3]);
        if (c == 0) *reinterpret_cast<float4*>(a.part_ml + at * 4) = make_float4(mm, mt, sum, 0.0f);
      } else {
        const bool none = mt == -INFINITY && sum == 0.0f;
        const float inv = none ? 0.0f : ref_to_top(mm, mt) / sum;
        const u32x2 two = {F16 ? pack_f16x2(o[0] * inv, o[1] * inv) : pack_bf16x2(o[0] * inv, o[1] * inv),
                           F16 ? pack_f16x2(o[2] * inv, o[3] * inv) : pack_bf16x2(o[2] * inv, o[3] * inv)};
        *reinterpret_cast<u32x2*>(a.o + (int64_t)(sp.r0 + t) * a.os + (int64_t)h * D + c) = two;
        if (c == 0 && a.lse) a.lse[gr] = none ? -INFINITY : (mt + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
      }
    }
  }
}

// The parts of a row's keys joined: a workgroup a row, d / 4 threads across its channels and 1024 / d groups that take the
// parts in turn, so that the loads of one part are never waited for before those of the next.
constexpr int kMaxSplit = 256;
template <int D, int R, int KT, bool F16>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int LN = D / 4, NG = 256 / LN;
  __shared__ float s_f[kMaxSplit], s_w[3][4];
  __shared__ float4 s_o[NG][LN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
  const Seq sq = find_seq(a.bt, t, 0, [](int c) { return c; });
  if (sq.b < 0 || t >= sq.r1) return;
  const Shares<R, KT> shares(a);
  const int parts = shares.parts(sq.r1 - sq.r0, sq.len);
  if (parts <= 1) return;
  const int rho = (t - sq.r0) * a.G + h % a.G;
  const int item = shares.before(sq.b) + rho / R * parts;    // the row tile's first; the parts follow
  if (item < 0 || item + parts > a.slots) return;            // (offsets that do not ascend: nothing was written)
  const int64_t gr = blockIdx.x;
  const int64_t first = ((int64_t)item * a.pg.heads + h / a.G) * R + rho % R, step = (int64_t)a.pg.heads * R;
  float4 w = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);  // ref, top, normaliser
  if ((int)threadIdx.x < parts) w = reinterpret_cast<const float4*>(a.part_ml)[first + threadIdx.x * step];
  float m = w.x, top = w.y;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    m = fmaxf(m, __shfl_xor(m, off, 64));
    top = fmaxf(top, __shfl_xor(top, off, 64));
  }
  if (lane == 0) {
    s_w[0][wave] = m;
    s_w[2][wave] = top;
  }
  __syncthreads();
  m = fmaxf(fmaxf(s_w[0][0], s_w[0][1]), fmaxf(s_w[0][2], s_w[0][3]));
  top = fmaxf(fmaxf(s_w[2][0], s_w[2][1]), fmaxf(s_w[2][2], s_w[2][3]));
  const bool idle = w.y == -INFINITY && w.z == 0.0f;
  float sum = idle ? 0.0f : w.z * __builtin_amdgcn_exp2f(w.y - top);
  s_f[threadIdx.x] = idle ? 0.0f : __builtin_amdgcn_exp2f(w.x - m);
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
  const bool none = top == -INFINITY && sum == 0.0f;
  const float inv = none ? 0.0f : ref_to_top(m, top) / sum;
  *reinterpret_cast<u32x2*>(a.o + (int64_t)t * a.os + (int64_t)h * D + 4 * c) =
      u32x2{F16 ? pack_f16x2(o.x * inv, o.y * inv) : pack_bf16x2(o.x * inv, o.y * inv),
            F16 ? pack_f16x2(o.z * inv, o.w * inv) : pack_bf16x2(o.z * inv, o.w * inv)};
  if (a.lse && c == 0) a.lse[gr] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

template <int R, int KT>
static int launch_merge(const PagedAttnArgs& a, int d, bool f16, hipStream_t st) {
  const unsigned grid = (unsigned)((int64_t)a.bt.T * a.Hq);
  if (d == 128) {
    if (f16) paged_merge_kernel<128, R, KT, true><<<grid, 256, 0, st>>>(a);
    else paged_merge_kernel<128, R, KT, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (f16) paged_merge_kernel<64, R, KT, true><<<grid, 256, 0, st>>>(a);
    else paged_merge_kernel<64, R, KT, false><<<grid, 256, 0, st>>>(a);
  }
  return check_launch("paged_merge_kernel");
}

// Work items of a head: row tiles, and with split keys as many parts more as the tiles are shared out to.
static int64_t items_of(int T, int G, int B, int Hkv, int rows, int n_split, int share) {
  return (int64_t)T * G / rows + B + (n_split > 1 ? share / Hkv + 1 : 0);
}

template <int NR>
static int launch_token(const PagedAttnArgs& args, int d, int format, bool f16, hipStream_t st) {
  PagedAttnArgs a = args;
  const int64_t items = items_of(a.bt.T, a.G, a.bt.B, a.pg.heads, 16 * NR, a.n_split, a.share), n = items * a.pg.heads;
  FL_REQUIRE(n < (1ll << 31), FL_E_SHAPE, "fl_paged_attn: too many rows");
  a.slots = (int)items;
  a.part_ml = a.part ? a.part + n * 16 * NR * d : nullptr;
  const unsigned grid = (unsigned)n;
#define FL_TOKEN(DD)                                                                        \
  do {                                                                                      \
    if (format == FL_KV_I8) {                                                               \
      if (f16) paged_token_kernel<DD, true, true, NR><<<grid, 256, 0, st>>>(a);             \
      else paged_token_kernel<DD, true, false, NR><<<grid, 256, 0, st>>>(a);                \
    } else {                                                                                \
      if (f16) paged_token_kernel<DD, false, true, NR><<<grid, 256, 0, st>>>(a);            \
      else paged_token_kernel<DD, false, false, NR><<<grid, 256, 0, st>>>(a);               \
    }                                                                                       \
  } while (0)
  if (d == 128) FL_TOKEN(128);
  else FL_TOKEN(64);
#undef FL_TOKEN
  int rc = check_launch("paged_token_kernel");
  if (rc != FL_OK || a.n_split == 1) return rc;
  return launch_merge<16 * NR, kTokenKeys>(a, d, f16, st);
}

// How a call is cut.  Up to 16 or 32 rows of a key/value head in a sequence: the kernel for few rows, whose keys are split while
// sequences and heads alone are fewer than its 768 shares (three workgroups per CU: 32 uneven sequences of 8 heads 57 us, 62 with
// 512, 59 with 1024; 131072 positions 55, 55, 56), in parts of 8 tiles or more (299 positions: 9.0 us in one part, 13 in two).
// More rows: the kernel for prompts.
constexpr int kShare = 768, kLeastTiles = 8;
struct Plan {
  int rows, n_split, min_tiles, share;
  int64_t keys;                   // that a row sees at most, as far as the caller knows
  size_t ws;
};
static Plan plan_of(int B, int T, int Hq, int Hkv, int d, int page, int max_pages, int window, int n_sink, int max_q, int max_len) {
  Plan p{};
  const int64_t G = Hq / Hkv;
  const int64_t per_seq = std::max<int64_t>(1, std::min<int64_t>(max_q > 0 ? max_q : 1, T)) * G;
  p.rows = per_seq <= 16 ? 16 : per_seq <= 32 ? 32 : 128;
  const int64_t cap = (int64_t)max_pages * page;
  int64_t len = max_len > 0 ? std::min<int64_t>(max_len, cap) : cap;
  if (window > 0) len = std::min<int64_t>(len, (int64_t)window + n_sink + std::max(max_q, 1));
  p.n_split = p.min_tiles = 1;
  p.keys = len;
  if (p.rows == 128) {
    p.ws = paged_prompt_ws((int64_t)T * G / kPromptRows + B, Hkv, d, cap, len);
    return p;
  }
  const int64_t tiles = std::max<int64_t>(1, (len + kTokenKeys - 1) / kTokenKeys);
  const int64_t units = std::max<int64_t>(1, std::max<int64_t>(B, T * G / p.rows)) * Hkv;
  p.share = kShare;
  p.min_tiles = kLeastTiles;
  const int64_t split = units < kShare ? std::min<int64_t>(std::max<int64_t>(tiles / kLeastTiles, 1), kMaxSplit) : 1;
  p.n_split = (int)split;
  // (a place for each row of each work item, however long the contexts are)
  p.ws = split > 1 ? (size_t)items_of(T, (int)G, B, Hkv, p.rows, p.n_split, p.share) * Hkv * p.rows * (d + 4) * sizeof(float) : 0;
  return p;
}

}  // namespace fl

using namespace fl;

extern "C" size_t fl_paged_attn_ws(int B, int T, int Hq, int Hkv, int d, int page, int max_pages, int window, int n_sink,
                                   int max_q, int max_len) {
  if (B < 1 || T < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv || (d != 64 && d != 128) || page < 16 || max_pages < 1 || window < 0 ||
      n_sink < 0 || max_q < 0 || max_len < 0)
    return 0;
  return plan_of(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len).ws;
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
  const Plan p = plan_of(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len);
  FL_REQUIRE(p.ws == 0 || (ws && ws_bytes >= p.ws), FL_E_WORKSPACE, "%s: workspace of %zu bytes required", fn, p.ws);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 15) == 0, FL_E_SHAPE, "%s: ws must be 16-byte aligned", fn);
  hipStream_t st = as_stream(stream);
  PagedAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.o = static_cast<uint16_t*>(o); a.lse = lse; a.qs = q_stride; a.os = o_stride;
  a.bt = {cu, lens, block_table, B, T, max_pages};
  a.rt = {table, rot, layout};
  a.pg = {num_pages, page, log2_of(page), Hkv};
  a.kc = static_cast<const uint8_t*>(k_cache); a.vc = static_cast<const uint8_t*>(v_cache); a.ksc = k_scale; a.vsc = v_scale;
  a.Hq = Hq; a.G = Hq / Hkv; a.scale_log2 = sm_scale * 1.4426950408889634f; a.window = window; a.n_sink = n_sink;
  a.n_split = p.n_split; a.min_tiles = p.min_tiles; a.share = p.share;
  a.part = static_cast<float*>(ws);
  rc = check_batch(fn, a.bt, a.pg, false, st);
  if (rc != FL_OK) return rc;
  if (p.rows == 16) return launch_token<1>(a, d, format, dtype == FL_F16, st);
  if (p.rows == 32) return launch_token<2>(a, d, format, dtype == FL_F16, st);
  return launch_paged_prompt(a, d, format, dtype == FL_F16, p.keys, st);
  FL_API_END
}
