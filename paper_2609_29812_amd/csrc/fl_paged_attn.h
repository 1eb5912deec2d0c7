// The paged attention's kernels: their arguments, how rows and keys are cut into work, and pieces that both kernels use.
#pragma once

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
  int n_split, min_tiles;          // at most n_split parts of the keys, each of about min_tiles tiles or more
  int share;                       // workgroups that the tiles of a batch are shared out to (many rows: per key/value head)
  int* ends;                       // many rows, shared out: units up to and with each row tile's
  int slots;                       // work items of a head at most: row tiles, with split keys of few rows their parts too
  float *part, *part_ml;           // rows of a split work item: [..][d] sums and [..][4]: ref, top and normaliser (below), unused
};

// What a row tile works on: rows rho0 .. rho0 + rows - 1 of a sequence, a row being (position, head of the group) with the
// heads fastest, and the tiles of KT keys that some row of it may see, in order: the n_lead tiles of the leading positions,
// then tiles first .. last.
struct Span {
  int r0, rho0, rows;              // rows == 0: nothing to do
  int start;                       // position of the sequence's first row
  int i_min, i_max;                // positions of the tile's first and last row
  int n_lead, first, tiles;        // tiles: in all
  int parts, per;                  // parts that have work, tiles in each but the last
};

// tiles `slot` of R rows: slots cu[b] G / R + b .. belong to sequence b
template <int R, int KT>
__device__ __forceinline__ Span span_of(const PagedAttnArgs& a, const Seq& q, int tile) {
  Span s{};
  s.r0 = q.r0;
  const int n = q.r1 - q.r0;
  s.rho0 = tile * R;
  s.rows = min(n * a.G - s.rho0, R);
  if (s.rows <= 0 || tile < 0) {
    s.rows = 0;
    return s;
  }
  const int cap = a.bt.max_pages * a.pg.size;                // positions that have a block table entry
  s.start = max(q.len, 0) - n;
  s.i_min = s.start + s.rho0 / a.G;
  s.i_max = s.start + (s.rho0 + s.rows - 1) / a.G;
  const int hi = min(s.i_max, cap - 1);
  int lo = 0;
  if (a.window > 0 && s.i_min >= a.window) lo = min(s.i_min - a.window + 1, cap);    // (a length beyond the block table)
  s.n_lead = (min(a.n_sink, lo) + KT - 1) / KT;
  s.first = max(s.n_lead, lo / KT);
  s.tiles = hi < 0 ? 0 : s.n_lead + max(hi / KT - s.first + 1, 0);
  s.parts = 1;
  s.per = s.tiles;
  return s;
}
// whether some row of the tile sees key j (when its page is there)
__device__ __forceinline__ bool seen_by_any(const PagedAttnArgs& a, const Span& s, int j) {
  const int lo = a.window > 0 && s.i_min >= a.window ? s.i_min - a.window + 1 : 0;
  return (j <= s.i_max) & ((j >= lo) | (j < a.n_sink));
}

// Split keys of few rows: the tiles of all sequences are shared out evenly, whatever the lengths are.  With `per` = all
// (sequence, row tile, key/value head, tile)s / share, a sequence of t tiles gets ceil(t / per) parts (at most n_split), and
// work item u of a head goes to sequences in order: rt_b * parts_b items each.  t is the number of tiles that a row tile sees at
// most; span_of then cuts what it does see into that many parts.
template <int R, int KT>
struct Shares {
  int per;
  int r0, r1, len;                                           // the lane's sequence of the first 64
  const PagedAttnArgs& a;
  __device__ __forceinline__ Shares(const PagedAttnArgs& args) : a(args) {
    float total = 0.0f;                                      // (a share: exactness is of no matter, and every wave has the same)
    const int lane = threadIdx.x & 63;
    load(lane, r0, r1, len);
    if (lane < a.bt.B) total = (float)row_tiles(r1 - r0) * (float)tiles(r1 - r0, len);
    for (int b = lane + 64; b - lane < a.bt.B; b += 64) {
      int x0, x1, l;
      load(b, x0, x1, l);
      if (b < a.bt.B) total += (float)row_tiles(x1 - x0) * (float)tiles(x1 - x0, l);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) total += __shfl_xor(total, off, 64);
    const float share = ceilf(total * (float)a.pg.heads / (float)a.share);
    per = __builtin_amdgcn_readfirstlane(max(a.min_tiles, (int)fminf(share, 1073741824.0f)));
  }
  __device__ __forceinline__ void load(int b, int& x0, int& x1, int& l) const {
    const int bc = min(b, a.bt.B - 1);
    x0 = row_of(a.bt, bc);
    x1 = row_of(a.bt, bc + 1);
    l = a.bt.lens[bc];
  }
  __device__ __forceinline__ int row_tiles(int n) const { return n <= 0 ? 0 : (n * a.G + R - 1) / R; }
  __device__ __forceinline__ int tiles(int n, int len) const {
    int64_t l = min(max(len, 0), a.bt.max_pages * a.pg.size);
    if (a.window > 0) l = min(l, (int64_t)a.window + a.n_sink + n);
    return (int)((l + KT - 1) / KT);
  }
  __device__ __forceinline__ int parts(int n, int len) const {
    return min(max((tiles(n, len) + per - 1) / per, 1), a.n_split);
  }
  // items of the sequences before sequence `seq`
  __device__ __forceinline__ int before(int seq) const {
    const int lane = threadIdx.x & 63;
    int sum = 0;
    for (int b0 = 0; b0 < seq; b0 += 64) {
      int x0 = r0, x1 = r1, xl = len;
      if (b0 > 0) load(b0 + lane, x0, x1, xl);
      sum += b0 + lane < seq ? row_tiles(x1 - x0) * parts(x1 - x0, xl) : 0;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    return sum;
  }
  // the sequence of item u, the row tile and the part; seq.b = -1 behind the last
  __device__ __forceinline__ Seq find(int u, int& tile, int& part) const {
    const int lane = threadIdx.x & 63;
    Seq s{-1, 0, 0, 0};
    tile = part = 0;
    int before = 0;                                          // items of the sequences looked at
    for (int b0 = 0; b0 < a.bt.B; b0 += 64) {
      int x0 = r0, x1 = r1, xl = len;
      if (b0 > 0) load(b0 + lane, x0, x1, xl);
      const int p = parts(x1 - x0, xl);
      const int items = b0 + lane < a.bt.B ? row_tiles(x1 - x0) * p : 0;
      int end = items;                                       // items up to and with the lane's
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(end, off, 64);
        end += lane >= off ? x : 0;
      }
      const uint64_t m = __builtin_amdgcn_ballot_w64(before + end > u);
      if (m != 0) {
        const int l = __builtin_ctzll(m);
        s = {b0 + l, __builtin_amdgcn_readlane(x0, l), __builtin_amdgcn_readlane(x1, l), __builtin_amdgcn_readlane(xl, l)};
        const int at = u - before - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(items, l));
        const int ps = __builtin_amdgcn_readlane(p, l);
        tile = at / ps;
        part = at % ps;
        break;
      }
      before += __builtin_amdgcn_readlane(end, 63);
    }
    return s;
  }
};
// cuts a span into the parts that its sequence has (some may have no tile)
__device__ __forceinline__ void cut(Span& s, int parts) {
  s.parts = parts;
  s.per = (s.tiles + parts - 1) / parts;
}
template <int KT>
__device__ __forceinline__ int key_of(const Span& s, int tile) { return (tile < s.n_lead ? tile : tile - s.n_lead + s.first) * KT; }

// The chunks of eight channels ch(0) .. ch(N - 1) of a row in fp32, turned by row `pos` of the table when there is one.  Loads stand in
// front and under no branch that lanes could take apart: a row costs two rounds of them.  AS_ROPE: the bits of rope_kernel (interleaved
// pairs' products are otherwise joined as the compiler likes; those of halves are its bits in any case).
template <int N, bool F16, bool AS_ROPE = false, class Ch>
__device__ __forceinline__ void turned_chunks(const Rotary& rt, const uint16_t* row, int pos, float (*v)[8], Ch ch) {
  uint4 raw[N], par[N];
#pragma unroll
  for (int k = 0; k < N; ++k) raw[k] = reinterpret_cast<const uint4*>(row)[ch(k)];
  if (!rt.table) {
#pragma unroll
    for (int k = 0; k < N; ++k) unpack8<F16>(raw[k], v[k]);
  } else {
    const float* tr = rt.table + (int64_t)pos * rt.rot;
    const int half = rt.rot / 16;                          // chunks of half the rotated part
    if (rt.layout == FL_ROPE_HALF) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = ch(k);
        par[k] = reinterpret_cast<const uint4*>(row)[c < half ? c + half : c < 2 * half ? c - half : c];
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = ch(k);
        const bool turn = c < 2 * half;
        const float sign = c < half ? -1.0f : 1.0f;
        const float4* p = reinterpret_cast<const float4*>(tr + 16 * (turn ? (c < half ? c : c - half) : 0));
        float y[8];
        unpack8<F16>(raw[k], v[k]);
        unpack8<F16>(par[k], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 w = p[e];
          const float r0 = fmaf(v[k][2 * e], w.x, y[2 * e] * (sign * w.y)), r1 = fmaf(v[k][2 * e + 1], w.z, y[2 * e + 1] * (sign * w.w));
          v[k][2 * e] = turn ? r0 : v[k][2 * e];
          v[k][2 * e + 1] = turn ? r1 : v[k][2 * e + 1];
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = ch(k);
        const bool turn = c < 2 * half;
        const float4* p = reinterpret_cast<const float4*>(tr + 8 * (turn ? c : 0));
        unpack8<F16>(raw[k], v[k]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 w = p[e];
          float* x = v[k] + 4 * e;
          float r0 = x[0] * w.x - x[1] * w.y, r1 = x[0] * w.y + x[1] * w.x;
          float r2 = x[2] * w.z - x[3] * w.w, r3 = x[2] * w.w + x[3] * w.z;
          if constexpr (AS_ROPE) {
            r0 = fmaf(x[0], w.x, -(x[1] * w.y)), r1 = fmaf(x[0], w.y, x[1] * w.x);
            r2 = fmaf(x[2], w.z, -(x[3] * w.w)), r3 = fmaf(x[2], w.w, x[3] * w.z);
          }
          x[0] = turn ? r0 : x[0];
          x[1] = turn ? r1 : x[1];
          x[2] = turn ? r2 : x[2];
          x[3] = turn ? r3 : x[3];
        }
      }
    }
  }
}

// The chunks of eight channels ch(0) .. ch(N - 1) of a query row as fp16 relative to the row's largest magnitude (2^-e, e its
// exponent, so that no range is lost), rotated by its position `pos` in fp32 when there is a table (a position outside the block
// table as if at its border).  `most` takes the largest magnitude of the lane to that of the row.  The row's
// factor comes back.
__device__ __forceinline__ float row_down(float m) {
  const int e = min(max((int)(__float_as_uint(m) >> 23), 1), 253);
  return __uint_as_float((uint32_t)(254 - e) << 23);
}
// fp16 queries get a second part, what the rounding of the rotated values to fp16 left (`low`; bf16 ones do not: their outputs are
// rounded eight times as coarsely).
template <int N, bool F16, class Ch, class Most>
__device__ __forceinline__ float load_query(const PagedAttnArgs& a, const uint16_t* row, bool ok, int pos, int cap, f16x8* q,
                                            f16x8* low, Ch ch, Most most) {
  float v[N][8];
  turned_chunks<N, F16>(a.rt, row, min(max(pos, 0), cap - 1), v, ch);
  float top = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[k][e]));
  top = most(top);
  const float down = row_down(top);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = ok ? pack_f16x2(v[k][2 * e] * down, v[k][2 * e + 1] * down) : 0u;
    q[k] = __builtin_bit_cast(f16x8, w);
    if constexpr (F16) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = ok ? pack_f16x2(v[k][2 * e] * down - (float)q[k][2 * e], v[k][2 * e + 1] * down - (float)q[k][2 * e + 1]) : 0u;
      low[k] = __builtin_bit_cast(f16x8, w);
    }
  }
  return top < INFINITY ? a.scale_log2 / down : NAN;         // (scores of an infinite query may all be -inf: NaN, not unseen)
}

// Four codes of one word as two fp16 pairs (exact).  Int8: c + 128 under the exponent of 1024, less 1152.
template <bool I8>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t* out) {
  if constexpr (I8) {
    w ^= 0x80808080u;
    const f16x2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    out[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off);
    out[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off);
  } else {
    out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true));
  }
}

// The largest of three in one instruction (v_maximum3_f32; a NaN comes through, where a maximum would first quiet its operands).
__device__ __forceinline__ float max3(float x, float y, float z) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z);
}

// What the value scale does.  A row has two references.  `ref` follows the contributions x + log2 s of its keys (x: a score in
// octaves, s: its page's scale), so exp2(x + log2 s - ref), a probability times its page's scale, stays within fp16's range whatever
// the scales are; `top` follows the scores, and the normaliser is held in units of 2^top.  A page's part of it is the
// sum of its contributions, times 2^(ref - top) / s.  That sum has room for 2^-126, so where ref - top - log2 s stays below kRoom
// octaves, what it loses is below 2^-62 of the normaliser.  Above (a page of values far smaller than those that carry the row) the
// page's exponentials are taken once more, relative to `top`.  The output is sums * 2^(ref - top) / normaliser.
// A scale below 2^-112 (the append writes none between 0 and 2^-109) counts as 0: it has kNoScale, one octave below any other, and
// its products are 0.
// One that is negative or not finite counts as 1 with a negative reciprocal (the normaliser does not depend on it), and the rows
// that see the page are made NaN.
constexpr float kRoom = 64.0f, kNoScale = -113.0f;
__device__ __forceinline__ float key_scale(float s) { return s >= 0.0f && s < INFINITY ? s : NAN; }
struct ValueScale {
  float log2, inv;
};
__device__ __forceinline__ ValueScale value_scale(float s) {
  if (!(s >= 0.0f && s < INFINITY)) return {0.0f, -1.0f};
  if (s < 0x1p-112f) return {kNoScale, 0x1p113f};
  return {__builtin_amdgcn_logf(s), 1.0f / s};
}
// 2^(ref - top); 1 for a row that has seen nothing, or nothing but NaN
__device__ __forceinline__ float ref_to_top(float ref, float top) {
  return ref == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - top);
}

// The work of a head, row tile after row tile, cut into shares of `per`: unit x belongs to workgroup owner(x).  A row tile is
// kTileUnits for its queries and what stands before its first product, then one unit a stage (at least one, so that the rows of a
// tile that sees no key are written).
constexpr int kTileUnits = 6;
struct Cut {
  int total, per;
  __device__ __forceinline__ int begin(int p) const { return (int)min((int64_t)total, (int64_t)per * p); }
  __device__ __forceinline__ int owner(int x) const { return x / per; }
};
// Units of a share at least: its queries, its sums and their join cost about ten.  Where few row tiles stand against many CUs
// (100 rows of 8 heads over 5000 positions, 320 units a head) 8, 12, 16 and 24 took 44, 48, 55 and 67 us; 64 rows over 32000
// positions 132, 116, 96 and 99 us, being joined from more parts then.
constexpr int kLeastUnits = 12;
__device__ __forceinline__ Cut cut_of(const PagedAttnArgs& a) {
  const int total = __builtin_amdgcn_readfirstlane(a.ends[a.slots - 1]);
  return {total, __builtin_amdgcn_readfirstlane(max(kLeastUnits, (total + a.share - 1) / a.share))};
}

// many rows
constexpr int kPromptRows = 128, kPromptKeys = 64;
constexpr int kPromptShares = 512;         // two workgroups per CU
size_t paged_prompt_ws(int64_t slots, int Hkv, int d, int64_t cap, int64_t keys);
int launch_paged_prompt(const PagedAttnArgs& a, int d, int format, bool f16, int64_t keys, hipStream_t st);

}  // namespace fl
