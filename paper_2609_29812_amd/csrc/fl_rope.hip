// Rotary positions: the table of cosines and sines, and the rotation of dense rows.
#include "fl_paged.h"

#include <cmath>
#include <vector>

namespace fl {

struct TableArgs {
  int n_pos, half, scaling, per;   // positions per thread
  double base, factor, orig_len, low, high, m;
  float2* out;
};

// The frequency of pair i (header, (9)).
__device__ __forceinline__ double frequency(const TableArgs& a, int i) {
  const double share = (double)i / (double)a.half;
  double f = pow(a.base, -share);
  if (a.scaling == FL_ROPE_LINEAR) f /= a.factor;
  if (a.scaling == FL_ROPE_YARN) {
    const double turns = a.orig_len * f / 6.283185307179586476925;
    const double g = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
    f = f * (g + (1.0 - g) / a.factor);
  }
  return f;
}

// A thread has one pair and `per` positions, so that the fp64 power is paid once for all of them.  The angle is reduced in turns,
// in fp64 (p f / 2 pi less its nearest integer: exact but for the product's rounding, 2^-53 of it); the remainder's sine and
// cosine are fp32 ones of its high part, corrected to first order by its low part.  Bound by the vector ALU (busy in all of the
// compute units' cycles): 131072 positions x 64 pairs, 67 MB, in 19 us, 3.6 TB/s (28 us with fp64 sines and cosines).
__global__ __launch_bounds__(256) void rope_table_kernel(TableArgs a) {
  const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int i = (int)(g % a.half);
  const int64_t p0 = g / a.half * a.per;
  if (p0 >= a.n_pos) return;
  const double turns = frequency(a, i) * 0.15915494309189533577;    // of a position: f / 2 pi
  const float m = (float)a.m;
  const int n = (int)min((int64_t)a.per, (int64_t)a.n_pos - p0);
  for (int x = 0; x < n; ++x) {
    const double t = (double)(p0 + x) * turns, r = 2.0 * (t - rint(t));     // half turns, in [-1, 1]
    const float hi = (float)r, lo = (float)(r - (double)hi) * 3.14159265358979f;
    float s, c;
    sincospif(hi, &s, &c);
    a.out[(p0 + x) * a.half + i] = make_float2(m * fmaf(-s, lo, c), m * fmaf(c, lo, s));
  }
}

struct RopeArgs {
  const uint16_t* x;
  uint16_t* y;
  const int32_t* pos;
  const float* table;
  int64_t xs, ys, n;               // row strides; work items
  int H, d, n_pos, rot, units;     // units of a head
  float sign;
};

// A unit is 16 channels of a head: chunks i and i + rot / 16 of its rotated part (FL_ROPE_HALF) or two neighbouring chunks
// of eight, so that a thread holds both values of every pair and the rotation may be in place.  A thread has one unit; the heads of a
// row find its cosines and sines in the caches.  Bound by HBM: 32768 rows of 16 heads x 128 in 47 us, 285 MB at 6.1 TB/s; eight
// rows 2.9 us.
template <bool HALF, bool F16>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (g >= a.n) return;
  const int u = (int)(g % a.units);
  const int64_t w = g / a.units;
  const int h = (int)(w % a.H);
  const int t = (int)(w / a.H);
  const int turned = a.rot / 16;
  const bool turn = u < turned;
  const int c0 = HALF && turn ? u : 2 * u;
  const int c1 = HALF && turn ? u + turned : 2 * u + 1;
  const bool two = c1 * 8 < a.d;
  float cs[16];
  if (turn) {
    const int p = a.pos ? a.pos[t] : t;
    const bool ok = (uint32_t)p < (uint32_t)a.n_pos;
    const float4* row = reinterpret_cast<const float4*>(a.table + (int64_t)(ok ? p : 0) * a.rot + u * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 v = row[e];
      cs[4 * e] = ok ? v.x : NAN;
      cs[4 * e + 1] = ok ? v.y * a.sign : NAN;
      cs[4 * e + 2] = ok ? v.z : NAN;
      cs[4 * e + 3] = ok ? v.w * a.sign : NAN;
    }
  }
  const uint16_t* src = a.x + (int64_t)t * a.xs + (int64_t)h * a.d;
  uint16_t* dst = a.y + (int64_t)t * a.ys + (int64_t)h * a.d;
  uint4 w0 = *reinterpret_cast<const uint4*>(src + c0 * 8);
  uint4 w1 = two ? *reinterpret_cast<const uint4*>(src + c1 * 8) : make_uint4(0, 0, 0, 0);
  if (turn) {
    float v[16], r[16];
    unpack8<F16>(w0, v);
    unpack8<F16>(w1, v + 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) {           // pair e: (v[e], v[e + 8]) or (v[2e], v[2e + 1])
      const int i0 = HALF ? e : 2 * e, i1 = HALF ? e + 8 : 2 * e + 1;
      r[i0] = v[i0] * cs[2 * e] - v[i1] * cs[2 * e + 1];
      r[i1] = v[i0] * cs[2 * e + 1] + v[i1] * cs[2 * e];
    }
    w0 = pack8<F16>(r);
    w1 = pack8<F16>(r + 8);
  }
  *reinterpret_cast<uint4*>(dst + c0 * 8) = w0;
  if (two) *reinterpret_cast<uint4*>(dst + c1 * 8) = w1;
}

int check_rows(const char* fn, const char* name, const void* x, int64_t stride, int H, int d) {
  FL_REQUIRE(x, FL_E_NULL, "%s: %s is NULL", fn, name);
  FL_REQUIRE(stride >= (int64_t)H * d && stride % 8 == 0, FL_E_SHAPE,
             "%s: the row stride of %s must be a multiple of 8 and at least H * d, got %lld", fn, name, (long long)stride);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(x) & 15) == 0, FL_E_SHAPE, "%s: %s must be 16-byte aligned", fn, name);
  return FL_OK;
}

int check_apart(const char* fn, const char* xn, const void* x, int64_t xs, const char* yn, const void* y, int64_t ys, int T,
                int width) {
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
  const uint64_t w = 2 * (uint64_t)width;
  const uint64_t xe = x0 + 2 * (uint64_t)(T - 1) * xs + w, ye = y0 + 2 * (uint64_t)(T - 1) * ys + w;
  // rows of the one may lie between the rows of the other, as the parts of a fused projection do
  const uint64_t gap = (x0 > y0 ? x0 - y0 : y0 - x0) % (2 * (uint64_t)xs);
  FL_REQUIRE(xe <= y0 || ye <= x0 || (xs == ys && gap >= w && gap <= 2 * (uint64_t)xs - w), FL_E_SHAPE, "%s: %s and %s overlap",
             fn, xn, yn);
  return FL_OK;
}

int check_rotary(const char* fn, const float* table, int rot, int layout, int d) {
  FL_REQUIRE(layout == FL_ROPE_HALF || layout == FL_ROPE_INTERLEAVED, FL_E_UNSUPPORTED, "%s: unknown layout %d", fn, layout);
  FL_REQUIRE(rot >= 16 && rot % 16 == 0 && rot <= d, FL_E_SHAPE, "%s: rot=%d must be a multiple of 16 in [16, %d]", fn, rot, d);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(table) & 15) == 0, FL_E_SHAPE, "%s: table must be 16-byte aligned", fn);
  return FL_OK;
}

}  // namespace fl

using namespace fl;

extern "C" int fl_rope_table(int n_pos, int rot, double base, int scaling, double factor, double orig_len, double low,
                             double high, float* table, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_rope_table";
  FL_REQUIRE(table, FL_E_NULL, "%s: table is NULL", fn);
  FL_REQUIRE((reinterpret_cast<uintptr_t>(table) & 15) == 0, FL_E_SHAPE, "%s: table must be 16-byte aligned", fn);
  FL_REQUIRE(scaling >= FL_ROPE_NONE && scaling <= FL_ROPE_YARN, FL_E_UNSUPPORTED, "%s: unknown scaling %d", fn, scaling);
  FL_REQUIRE(n_pos >= 1, FL_E_SHAPE, "%s: n_pos=%d must be positive", fn, n_pos);
  FL_REQUIRE(rot >= 16 && rot % 16 == 0 && rot <= 1024, FL_E_SHAPE, "%s: rot=%d must be a multiple of 16 in [16, 1024]", fn, rot);
  FL_REQUIRE(std::isfinite(base) && base > 1.0, FL_E_RANGE, "%s: base must be finite and above 1", fn);
  if (scaling != FL_ROPE_NONE)
    FL_REQUIRE(std::isfinite(factor) && factor >= 1.0, FL_E_RANGE, "%s: factor must be finite and at least 1", fn);
  if (scaling == FL_ROPE_YARN)
    FL_REQUIRE(std::isfinite(orig_len) && orig_len > 0.0 && std::isfinite(low) && std::isfinite(high) && low < high, FL_E_RANGE,
               "%s: YARN needs orig_len > 0 and low < high", fn);
  TableArgs a{};
  a.n_pos = n_pos; a.half = rot / 2; a.scaling = scaling;
  a.base = scaling == FL_ROPE_NTK ? base * std::pow(factor, (double)rot / (rot - 2)) : base;
  a.factor = factor; a.orig_len = orig_len; a.low = low; a.high = high;
  a.m = scaling == FL_ROPE_YARN ? 1.0 + 0.1 * std::log(factor) : 1.0;
  a.out = reinterpret_cast<float2*>(table);
  a.per = n_pos >= 65536 ? 32 : n_pos >= 8192 ? 4 : 1;
  const int64_t threads = ((int64_t)n_pos + a.per - 1) / a.per * a.half;
  rope_table_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, as_stream(stream)>>>(a);
  return check_launch("rope_table_kernel");
  FL_API_END
}

extern "C" int fl_rope(const void* x, int64_t x_stride, const int32_t* pos, const float* table, int n_pos, int rot,
                       int layout, int inverse, int dtype, int T, int H, int d, void* y, int64_t y_stride, void* stream) {
  FL_API_BEGIN
  const char* fn = "fl_rope";
  FL_REQUIRE(dtype == FL_BF16 || dtype == FL_F16, FL_E_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  FL_REQUIRE(T >= 0 && H >= 1, FL_E_SHAPE, "%s: T=%d must be >= 0 and H=%d positive", fn, T, H);
  FL_REQUIRE(d >= 16 && d % 8 == 0 && d <= 1024, FL_E_SHAPE, "%s: d=%d must be a multiple of 8 in [16, 1024]", fn, d);
  FL_REQUIRE(table, FL_E_NULL, "%s: table is NULL", fn);
  int rc = check_rotary(fn, table, rot, layout, d);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(n_pos >= 1 && (pos || T <= n_pos), FL_E_RANGE, "%s: %d rows without positions need a table of as many, got %d", fn,
             T, n_pos);
  if (T == 0) return FL_OK;
  rc = check_rows(fn, "x", x, x_stride, H, d);
  if (rc != FL_OK) return rc;
  rc = check_rows(fn, "y", y, y_stride, H, d);
  if (rc != FL_OK) return rc;
  if (x != y || x_stride != y_stride) {
    rc = check_apart(fn, "x", x, x_stride, "y", y, y_stride, T, H * d);
    if (rc != FL_OK) return rc;
  }
  hipStream_t st = as_stream(stream);
  if (index_checks_on() && pos) {
    hipError_t e = hipStreamSynchronize(st);
    std::vector<int32_t> p((size_t)T);
    if (e == hipSuccess) e = hipMemcpy(p.data(), pos, p.size() * 4, hipMemcpyDeviceToHost);
    FL_REQUIRE(e == hipSuccess, FL_E_HIP, "%s: index check: copy of pos failed: %s", fn, hipGetErrorString(e));
    for (int t = 0; t < T; ++t)
      FL_REQUIRE(p[t] >= 0 && p[t] < n_pos, FL_E_RANGE, "%s: pos[%d] = %d outside [0, %d)", fn, t, p[t], n_pos);
  }
  RopeArgs a{};
  a.x = static_cast<const uint16_t*>(x); a.y = static_cast<uint16_t*>(y); a.pos = pos; a.table = table;
  a.xs = x_stride; a.ys = y_stride; a.H = H; a.d = d; a.n_pos = n_pos; a.rot = rot;
  a.units = (d + 15) / 16;
  a.n = (int64_t)T * H * a.units;
  a.sign = inverse ? -1.0f : 1.0f;
  FL_REQUIRE((a.n + 255) / 256 < (1ll << 31), FL_E_SHAPE, "%s: T * H * d too large", fn);
  const unsigned grid = (unsigned)((a.n + 255) / 256);
  if (layout == FL_ROPE_HALF) {
    if (dtype == FL_F16) rope_kernel<true, true><<<grid, 256, 0, st>>>(a);
    else rope_kernel<true, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (dtype == FL_F16) rope_kernel<false, true><<<grid, 256, 0, st>>>(a);
    else rope_kernel<false, false><<<grid, 256, 0, st>>>(a);
  }
  return check_launch("rope_kernel");
  FL_API_END
}
