// Rotary positions of queries and keys, by themselves and behind a norm over each head, for gfx950.
#include "ad_device.h"
#include "ad_kernels.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace ad {

constexpr int kRopeMaxDim = 128;   // widest head: the limit of the attention kernels too

// =================================================================================================
// Row (b, i) of q or k is `heads` vectors of d elements.  With a norm, each becomes y = x rsqrt(mean x^2 + eps) gain, or
// (x - mean) rsqrt(var + eps) gain + offset.  Then pair p of the rotated part, (x_a, x_b), is turned by t = n_p f_p, n_p the row's
// position on the axis of p:  x_a' = A (x_a cos t - x_b sin t),  x_b' = A (x_b cos t + x_a sin t).
//
// The angle: positions are whole numbers, so whole turns may be dropped from the frequency and from the product.  f / 2 pi is held as a
// fraction of a turn in 64 bits, the product with the position is taken modulo one turn in whole numbers, and its upper 32 bits are the
// phase: exact to 2^-32 turn plus position * 2^-64, however far the position is (an fp32 product at position 10^6 is off by 0.06 rad).
// v_sin_f32 / v_cos_f32 take turns; over one turn they are off by at most 1.3e-7 (rms 3.5e-8, measured at 2^20 phases), less than
// an fp32 angle's own rounding, so fp32 tensors use them as well.
//
// A workgroup takes a few rows with all heads of q and k.  It asks for its elements, forms the sines and cosines of its rows once, in LDS, and the heads
// read them from there.  A head is shared out over a power of two of lanes, each with two accesses of VN elements (up to 16 bytes each): the two sides of VN
// pairs where the pairs lie half the rotated part apart, VN pairs in a row where they are neighbours; the part that is not rotated lies behind.  The norm's
// sums go over those lanes.  Bound by memory: every element is read once and written once; a lane writes where it has read, so q_out may be q.
// us: rotation of 16384 rows of 20 heads of 64, bf16, 84 MB 15.1 to 18.4 from run to run (5.6 to 4.6 TB/s), 10006 of 10 heads of 80, fp32, 64 MB 11.8 (5.4); norm and rotation of 18432 rows of
// 20 heads of 32, bf16, 47 MB 11.4 (4.2).  With the angles in every group of lanes and the gains in registers 15.3, 12.3 and 14.4; two, three or six heads in flight and
// occupancies of six and eight wavefronts: level or slower.
// =================================================================================================
struct RopeSide {
  const void* src; void* dst;
  const float *gain, *offset;
  int heads, ld, ldo;
};
struct RopeParams {
  RopeSide q, k;
  const unsigned long long* table;
  const int* positions;
  long long sample_positions;    // positions of a sample, 0: shared
  unsigned rows, l;
  FastDiv div_l, div_heads, div_pairs;
  int d, pairs, axis_end[AD_ROPE_MAX_AXES];   // last pair of an axis + 1
  int heads, block_rows;         // of q and k together; rows of a workgroup
  int units, log_lanes;          // lanes' shares of a head, lanes of a head
  float eps, amplitude, inv_d;
};

template <typename T, int VN> struct alignas(VN * sizeof(T)) Access { T v[VN]; };

enum { ROPE_NO_NORM = -1 };

// sum over the 2^log_lanes neighbouring lanes of a head
__device__ __forceinline__ float head_sum(float v, int log_lanes) {
  if (log_lanes > 0) v += dpp_f<0xB1>(v);
  if (log_lanes > 1) v += dpp_f<0x4E>(v);
  if (log_lanes > 2) v += dpp_f<0x141>(v);
  if (log_lanes > 3) v += dpp_f<0x140>(v);
  if (log_lanes > 4) v += __shfl_xor(v, 16, 64);
  if (log_lanes > 5) v += __shfl_xor(v, 32, 64);
  return v;
}

template <typename T, int VN, int LAYOUT, int NORM>
__global__ __launch_bounds__(256) void k_rope(RopeParams p) {
  typedef Access<T, VN> V;
  typedef Access<float, VN> F;
  extern __shared__ __attribute__((aligned(16))) float lds[];    // cosines [row][pair], sines [row][pair], then gain (and offset) of q and of k
  const int tid = threadIdx.x;
  const int unit = tid & ((1 << p.log_lanes) - 1), group = tid >> p.log_lanes, groups = 256 >> p.log_lanes;
  const unsigned row0 = blockIdx.x * (unsigned)p.block_rows;
  const int rows = min((unsigned)p.block_rows, p.rows - row0), items = rows * p.heads;

  // where this lane's two accesses lie in a head
  const int turning = p.pairs / VN;              // lanes with rotated pairs
  const bool turns = unit < turning;
  int at_a, at_b;
  if (turns) {
    at_a = LAYOUT == AD_ROPE_HALF ? unit * VN : 2 * unit * VN;
    at_b = at_a + (LAYOUT == AD_ROPE_HALF ? p.pairs : VN);
  } else {
    at_a = 2 * p.pairs + 2 * (unit - turning) * VN;
    at_b = at_a + VN;
  }
  const bool has_a = at_a < p.d, has_b = at_b < p.d;

  constexpr int UN = 4;                          // heads in flight
  V a[UN], b[UN];
  auto split = [&](int item, int& r, int& h) {
    r = (int)fast_div((unsigned)item, p.div_heads);
    h = item - r * p.heads;
  };
  auto fetch = [&](int first) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int item = first + u * groups;
#pragma unroll
      for (int e = 0; e < VN; ++e) { a[u].v[e] = from_f<T>(0.f); b[u].v[e] = from_f<T>(0.f); }
      if (item >= items) continue;
      int r, h;
      split(item, r, h);
      const bool is_k = h >= p.q.heads;
      const T* const src = (const T*)(is_k ? p.k.src : p.q.src) + (size_t)(row0 + r) * (is_k ? p.k.ld : p.q.ld) + (size_t)(is_k ? h - p.q.heads : h) * p.d;
      if (has_a) a[u] = *(const V*)(src + at_a);
      if (has_b) b[u] = *(const V*)(src + at_b);
    }
  };
  fetch(group);

  float* const cosines = lds;
  float* const sines = lds + p.block_rows * p.pairs;
  float* const gains = sines + p.block_rows * p.pairs;
  for (int at = tid; at < rows * p.pairs; at += 256) {
    const int r = (int)fast_div((unsigned)at, p.div_pairs), pair = at - r * p.pairs;
    const unsigned row = row0 + r, sample = fast_div(row, p.div_l);
    const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]);
    const int n = p.positions[(size_t)sample * p.sample_positions + (size_t)axis * p.l + (row - sample * p.l)];
    const unsigned long long f = p.table[pair];
    const unsigned f_lo = (unsigned)f, f_hi = (unsigned)(f >> 32);
    const unsigned phase = (unsigned)n * f_hi + __umulhi((unsigned)n, f_lo) - (n < 0 ? f_lo : 0u);     // bits 32 .. 63 of n * f
    const float turn = (float)(int)phase * 0x1p-32f;
    cosines[at] = __builtin_amdgcn_cosf(turn) * p.amplitude;
    sines[at] = __builtin_amdgcn_sinf(turn) * p.amplitude;
  }
  if constexpr (NORM != ROPE_NO_NORM) {
    constexpr int KINDS = NORM == AD_NORM_LAYER ? 4 : 2;
    for (int at = tid; at < KINDS * p.d; at += 256) {
      const int kind = at / p.d, e = at - kind * p.d;            // gain of q, gain of k, offset of q, offset of k
      const float* const from = kind == 0 ? p.q.gain : kind == 1 ? p.k.gain : kind == 2 ? p.q.offset : p.k.offset;
      gains[at] = from ? from[e] : (kind < 2 ? 1.f : 0.f);
    }
  }
  __syncthreads();

  for (int first = group; first < items; first += UN * groups) {
    if (first > group) fetch(first);
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int item = first + u * groups;
      if (item >= items) break;
      int row, h;
      split(item, row, h);
      const bool is_k = h >= p.q.heads;
      float x[VN], y[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) { x[e] = to_f(a[u].v[e]); y[e] = to_f(b[u].v[e]); }
      if constexpr (NORM != ROPE_NO_NORM) {
        if constexpr (NORM == AD_NORM_LAYER) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < VN; ++e) sum += x[e] + y[e];
          const float mean = head_sum(sum, p.log_lanes) * p.inv_d;
#pragma unroll
          for (int e = 0; e < VN; ++e) {
            x[e] = has_a ? x[e] - mean : 0.f;
            y[e] = has_b ? y[e] - mean : 0.f;
          }
        }
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < VN; ++e) sq = fmaf(x[e], x[e], fmaf(y[e], y[e], sq));
        const float r = rsqrtf(head_sum(sq, p.log_lanes) * p.inv_d + p.eps);
        const float* const gain = gains + (is_k ? p.d : 0);
        F ga, gb, oa{}, ob{};
        if (has_a) ga = *(const F*)(gain + at_a);
        if (has_b) gb = *(const F*)(gain + at_b);
        if constexpr (NORM == AD_NORM_LAYER) {
          if (has_a) oa = *(const F*)(gain + 2 * p.d + at_a);
          if (has_b) ob = *(const F*)(gain + 2 * p.d + at_b);
        }
#pragma unroll
        for (int e = 0; e < VN; ++e) {
          x[e] = NORM == AD_NORM_LAYER ? fmaf(x[e] * r, ga.v[e], oa.v[e]) : x[e] * r * ga.v[e];
          y[e] = NORM == AD_NORM_LAYER ? fmaf(y[e] * r, gb.v[e], ob.v[e]) : y[e] * r * gb.v[e];
        }
      }
      if (turns) {
        const F co = *(const F*)(cosines + row * p.pairs + unit * VN), si = *(const F*)(sines + row * p.pairs + unit * VN);
        if constexpr (LAYOUT == AD_ROPE_HALF || VN == 1) {
#pragma unroll
          for (int e = 0; e < VN; ++e) {
            const float xe = x[e], ye = y[e];
            x[e] = fmaf(xe, co.v[e], -(ye * si.v[e]));
            y[e] = fmaf(ye, co.v[e], xe * si.v[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < VN; e += 2) {
            const float x0 = x[e], x1 = x[e + 1], y0 = y[e], y1 = y[e + 1];
            x[e] = fmaf(x0, co.v[e / 2], -(x1 * si.v[e / 2]));
            x[e + 1] = fmaf(x1, co.v[e / 2], x0 * si.v[e / 2]);
            y[e] = fmaf(y0, co.v[(VN + e) / 2], -(y1 * si.v[(VN + e) / 2]));
            y[e + 1] = fmaf(y1, co.v[(VN + e) / 2], y0 * si.v[(VN + e) / 2]);
          }
        }
      }
      V wa, wb;
#pragma unroll
      for (int e = 0; e < VN; ++e) { wa.v[e] = from_f<T>(x[e]); wb.v[e] = from_f<T>(y[e]); }
      T* const dst = (T*)(is_k ? p.k.dst : p.q.dst) + (size_t)(row0 + row) * (is_k ? p.k.ldo : p.q.ldo) + (size_t)(is_k ? h - p.q.heads : h) * p.d;
      if (has_a) *(V*)(dst + at_a) = wa;
      if (has_b) *(V*)(dst + at_b) = wb;
    }
  }
}

static ad_status check_rope(const ad_rope_cfg* c, const char* who) {
  if (!c) AD_FAIL(AD_ERR_INVALID, "%s: null configuration", who);
  if (c->layout != AD_ROPE_HALF && c->layout != AD_ROPE_INTERLEAVED) AD_FAIL(AD_ERR_INVALID, "%s: bad layout", who);
  if (c->n_axes < 1 || c->n_axes > AD_ROPE_MAX_AXES) AD_FAIL(AD_ERR_INVALID, "%s: 1..%d axes", who, AD_ROPE_MAX_AXES);
  int sum = 0;
  for (int a = 0; a < c->n_axes; ++a) {
    if (c->axis_dims[a] < 2 || c->axis_dims[a] % 2 || c->axis_dims[a] > kRopeMaxDim) AD_FAIL(AD_ERR_INVALID, "%s: an axis turns an even number of elements, 2..%d", who, kRopeMaxDim);
    sum += c->axis_dims[a];
  }
  if (sum > kRopeMaxDim) AD_FAIL(AD_ERR_INVALID, "%s: the axes turn %d elements, at most %d", who, sum, kRopeMaxDim);
  if (!(c->base > 1.0) || !std::isfinite(c->base)) AD_FAIL(AD_ERR_INVALID, "%s: base must be above 1", who);
  if (!(c->amplitude >= 0.0) || !std::isfinite(c->amplitude)) AD_FAIL(AD_ERR_INVALID, "%s: bad amplitude", who);
  if (c->scaling < AD_ROPE_PLAIN || c->scaling > AD_ROPE_PARTS) AD_FAIL(AD_ERR_INVALID, "%s: bad scaling", who);
  if (c->scaling != AD_ROPE_PLAIN && (!(c->factor >= 1.0) || !std::isfinite(c->factor))) AD_FAIL(AD_ERR_INVALID, "%s: the scaling's factor must be at least 1", who);
  if (c->scaling == AD_ROPE_PARTS && (!(c->original_len > 0.0) || !std::isfinite(c->original_len) || !(c->slow_turns >= 0.0) || !(c->fast_turns > c->slow_turns) || !std::isfinite(c->fast_turns)))
    AD_FAIL(AD_ERR_INVALID, "%s: scaling by parts needs the original length and 0 <= slow_turns < fast_turns", who);
  return AD_OK;
}

static double rope_amplitude(const ad_rope_cfg& c) {
  if (c.amplitude > 0.0) return c.amplitude;
  return c.scaling == AD_ROPE_PARTS ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
}

// turns a position, modulo one, as a fraction of 2^64
static unsigned long long turn_fraction(double radians) {
  long double t = (long double)radians / 6.283185307179586476925286766559L;
  t -= floorl(t);
  const long double scaled = roundl(ldexpl(t, 64));
  return scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
}

static ad_status launch_rope(const char* name, int dtype, int norm, const ad_rope_cfg* cfg, const void* table, const int* positions, int per_sample, const void* q,
                             const void* k, const float* q_gain, const float* k_gain, const float* q_offset, const float* k_offset, float eps, int batch,
                             int l, int heads, int kv_heads, int d, int ldq, int ldk, void* q_out, void* k_out, int ldq_out, int ldk_out, hipStream_t s) {
  if (dtype != AD_BF16 && dtype != AD_F32) AD_FAIL(AD_ERR_INVALID, "%s: bad dtype", name);
  if (!q || !q_out || (kv_heads > 0 && (!k || !k_out))) AD_FAIL(AD_ERR_INVALID, "%s: null pointer", name);
  if (batch < 1 || l < 1 || heads < 1 || kv_heads < 0 || d < 1 || d > kRopeMaxDim || (long long)batch * l > 0x7fffffffLL)
    AD_FAIL(AD_ERR_INVALID, "%s: bad shape (head_dim 1..%d)", name, kRopeMaxDim);
  if (((long long)heads + kv_heads) * d > 0x7fff0000LL) AD_FAIL(AD_ERR_INVALID, "%s: too many heads", name);
  if (ldq < heads * d || ldq_out < heads * d || (kv_heads > 0 && (ldk < kv_heads * d || ldk_out < kv_heads * d))) AD_FAIL(AD_ERR_INVALID, "%s: bad leading dimension", name);
  if ((q == q_out && ldq != ldq_out) || (kv_heads > 0 && k == k_out && ldk != ldk_out)) AD_FAIL(AD_ERR_INVALID, "%s: in place, both leading dimensions are the same", name);
  if (kv_heads > 0 && q_out == k_out) AD_FAIL(AD_ERR_INVALID, "%s: q_out and k_out are the same", name);
  const size_t es = esize(dtype);
  uintptr_t all = (uintptr_t)q | (uintptr_t)q_out | (kv_heads > 0 ? (uintptr_t)k | (uintptr_t)k_out : 0);
  if (all % es) AD_FAIL(AD_ERR_INVALID, "%s: a tensor is not aligned to its type", name);
  RopeParams p{};
  int pairs = 0;
  if (cfg) {
    const ad_status st = check_rope(cfg, name);
    if (st != AD_OK) return st;
    if (!table || !positions) AD_FAIL(AD_ERR_INVALID, "%s: null table or positions", name);
    if ((uintptr_t)table % 8 || (uintptr_t)positions % 4) AD_FAIL(AD_ERR_INVALID, "%s: table or positions not aligned to their type", name);
    for (int a = 0; a < AD_ROPE_MAX_AXES; ++a) {
      if (a < cfg->n_axes) pairs += cfg->axis_dims[a] / 2;
      p.axis_end[a] = pairs;
    }
    if (2 * pairs > d) AD_FAIL(AD_ERR_INVALID, "%s: the axes turn %d elements of a head of %d", name, 2 * pairs, d);
    p.amplitude = (float)rope_amplitude(*cfg);
  }
  if (norm != ROPE_NO_NORM) {
    if (norm != AD_NORM_RMS && norm != AD_NORM_LAYER) AD_FAIL(AD_ERR_INVALID, "%s: bad norm", name);
    if (!(eps > 0.f) || !std::isfinite(eps)) AD_FAIL(AD_ERR_INVALID, "%s: eps must be above 0", name);
    if (norm == AD_NORM_RMS && (q_offset || k_offset)) AD_FAIL(AD_ERR_INVALID, "%s: an RMS norm has no offset", name);
    if (((uintptr_t)q_gain | (uintptr_t)k_gain | (uintptr_t)q_offset | (uintptr_t)k_offset) % 4) AD_FAIL(AD_ERR_INVALID, "%s: gain or offset not aligned to its type", name);
  }
  // the widest access that pairs, heads, rows and addresses allow
  int vn = 16 / (int)es;
  const int lds = ldq | ldq_out | (kv_heads > 0 ? ldk | ldk_out : 0);
  while (vn > 1 && (pairs % vn || d % vn || lds % vn || all % (vn * es))) vn >>= 1;
  p.units = pairs / vn + (d - 2 * pairs + 2 * vn - 1) / (2 * vn);
  while ((1 << p.log_lanes) < p.units) ++p.log_lanes;
  p.rows = (unsigned)((long long)batch * l);
  p.l = (unsigned)l;
  p.div_l = make_fastdiv(p.l);
  p.d = d; p.pairs = pairs;
  p.table = (const unsigned long long*)table;
  p.positions = positions;
  p.sample_positions = cfg && per_sample ? (long long)cfg->n_axes * l : 0;
  p.eps = eps; p.inv_d = 1.f / (float)d;
  p.q = RopeSide{q, q_out, q_gain, q_offset, heads, ldq, ldq_out};
  p.k = RopeSide{k, k_out, k_gain, k_offset, kv_heads, ldk, ldk_out};
  p.heads = heads + kv_heads;
  p.div_heads = make_fastdiv((unsigned)p.heads);
  p.div_pairs = make_fastdiv((unsigned)std::max(pairs, 1));
  // rows of a workgroup: what its lanes hold in flight at once, as far as the sines and cosines stay below 16 KiB; where that leaves CUs idle, fewer
  const int in_flight = 4 * (256 >> p.log_lanes);
  int block_rows = std::max(1, in_flight / p.heads);
  if (pairs > 0) block_rows = std::min(block_rows, std::max(1, 2048 / pairs));
  p.block_rows = (int)std::min<long long>(block_rows, std::max(1u, p.rows / 512));
  const size_t lds_bytes = (size_t)(2 * p.block_rows * pairs + (norm == ROPE_NO_NORM ? 0 : 4 * d)) * 4;
  const double elements = (double)p.rows * (heads + kv_heads) * d;
  ProfLaunch pl(norm == ROPE_NO_NORM ? "rope" : "qk_norm_rope", 0, 2.0 * es * elements, s);
  const dim3 grid((p.rows + p.block_rows - 1) / p.block_rows);
  const int layout = cfg ? cfg->layout : AD_ROPE_HALF;
#define AD_ROPE_RUN(T_, VN_, LAYOUT_, NORM_) hipLaunchKernelGGL((k_rope<T_, VN_, LAYOUT_, NORM_>), grid, dim3(256), lds_bytes, s, p)
#define AD_ROPE_NORM(T_, VN_, LAYOUT_)                                                \
  if (norm == ROPE_NO_NORM) AD_ROPE_RUN(T_, VN_, LAYOUT_, ROPE_NO_NORM);              \
  else if (norm == AD_NORM_RMS) AD_ROPE_RUN(T_, VN_, LAYOUT_, AD_NORM_RMS);           \
  else AD_ROPE_RUN(T_, VN_, LAYOUT_, AD_NORM_LAYER)
#define AD_ROPE_LAYOUT(T_, VN_)                                                       \
  if (layout == AD_ROPE_HALF) { AD_ROPE_NORM(T_, VN_, AD_ROPE_HALF); }                \
  else { AD_ROPE_NORM(T_, VN_, AD_ROPE_INTERLEAVED); }
  if (dtype == AD_BF16) {
    if (vn == 8) { AD_ROPE_LAYOUT(bf16, 8) }
    else if (vn == 4) { AD_ROPE_LAYOUT(bf16, 4) }
    else if (vn == 2) { AD_ROPE_LAYOUT(bf16, 2) }
    else { AD_ROPE_LAYOUT(bf16, 1) }
  } else {
    if (vn == 4) { AD_ROPE_LAYOUT(float, 4) }
    else if (vn == 2) { AD_ROPE_LAYOUT(float, 2) }
    else { AD_ROPE_LAYOUT(float, 1) }
  }
#undef AD_ROPE_LAYOUT
#undef AD_ROPE_NORM
#undef AD_ROPE_RUN
  AD_HIP(hipGetLastError());
  return AD_OK;
}

}  // namespace ad

using namespace ad;

extern "C" {

ad_status ad_rope_table(const ad_rope_cfg* cfg, void* out, size_t* bytes) {
  const ad_status st = check_rope(cfg, "rope table");
  if (st != AD_OK) return st;
  int pairs = 0;
  for (int a = 0; a < cfg->n_axes; ++a) pairs += cfg->axis_dims[a] / 2;
  if (bytes) *bytes = (size_t)pairs * 8;
  else if (!out) AD_FAIL(AD_ERR_INVALID, "rope table: null pointer");
  if (!out) return AD_OK;
  char* to = (char*)out;
  for (int a = 0; a < cfg->n_axes; ++a) {
    const int dim = cfg->axis_dims[a];
    double base = cfg->base;
    if (cfg->scaling == AD_ROPE_BASE && dim > 2) base *= std::pow(cfg->factor, (double)dim / (dim - 2));
    for (int i = 0; i < dim / 2; ++i) {
      double f = std::pow(base, -2.0 * i / dim);
      if (cfg->scaling == AD_ROPE_LINEAR) f /= cfg->factor;
      if (cfg->scaling == AD_ROPE_PARTS) {
        const double turns = cfg->original_len * f / 6.283185307179586476925286766559;
        const double keep = std::min(1.0, std::max(0.0, (turns - cfg->slow_turns) / (cfg->fast_turns - cfg->slow_turns)));
        f = f / cfg->factor * (1.0 - keep) + f * keep;
      }
      const unsigned long long t = turn_fraction(f);
      std::memcpy(to, &t, 8);
      to += 8;
    }
  }
  return AD_OK;
}

ad_status ad_rope_forward(int dtype, const ad_rope_cfg* cfg, const void* table, const int* positions, int per_sample, const void* q, const void* k,
                          int batch, int l, int heads, int kv_heads, int head_dim, int ldq, int ldk, void* q_out, void* k_out, int ldq_out,
                          int ldk_out, ad_stream stream) {
  if (!cfg) AD_FAIL(AD_ERR_INVALID, "rope: null configuration");
  return launch_rope("rope", dtype, ROPE_NO_NORM, cfg, table, positions, per_sample, q, k, nullptr, nullptr, nullptr, nullptr, 0.f, batch, l, heads, kv_heads,
                     head_dim, ldq, ldk, q_out, k_out, ldq_out, ldk_out, (hipStream_t)stream);
}

ad_status ad_qk_norm_rope_forward(int dtype, int norm, const ad_rope_cfg* cfg, const void* table, const int* positions, int per_sample, const void* q, const void* k,
                                  const float* q_gain, const float* k_gain, const float* q_offset, const float* k_offset, float eps, int batch, int l,
                                  int heads, int kv_heads, int head_dim, int ldq, int ldk, void* q_out, void* k_out, int ldq_out, int ldk_out,
                                  ad_stream stream) {
  if (norm != AD_NORM_RMS && norm != AD_NORM_LAYER) AD_FAIL(AD_ERR_INVALID, "qk norm: bad norm");
  return launch_rope("qk norm", dtype, norm, cfg, table, positions, per_sample, q, k, q_gain, k_gain, q_offset, k_offset, eps, batch, l, heads, kv_heads,
                     head_dim, ldq, ldk, q_out, k_out, ldq_out, ldk_out, (hipStream_t)stream);
}

}  // extern "C"
