// Differential attention for gfx950:
//   out = (softmax(q1 k1^T / sqrt d) - lambda softmax(q2 k2^T / sqrt d)) v, then an RMS norm over each head (arXiv 2410.05258).
// q1 | q2 and k1 | k2 are the two halves of a head of 2 d columns, v is 2 d wide.  Query heads that share a key head are rows of the same
// tile (row r of a key head: query r / group, head r % group of the group), so a single token still fills its tile as far as the heads allow.
#include "ad_device.h"
#include "ad_kernels.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

namespace ad {

constexpr float kLog2e = 1.44269504088896341f;
// The exponential's reference need not be the running maximum: any value near it gives the same quotient.  It is the exact maximum of the first block
// of keys that a row sees, and is raised (and what has been summed rescaled) when a block's sum of weights reaches 2^24, so the steady state computes no
// maximum.  A row sees a prefix of its keys, so where it sees any of a share, it sees the first.
constexpr float kDiffBig = 16777216.f;
constexpr int kDiffMaxSplits = 64;   // shares of the keys: a lane each when they are joined

struct DiffParams {
  const void *q, *k, *v; void* out;
  const int* key_lens;
  const float *lambda, *gain;
  float* partial;                 // sums of the key shares, see diff_record()
  int l, lk, kv_heads, group, d;  // group: query heads to a key head
  int ldq, ldk, ldv, ldo;
  int causal, rows, tiles, splits, split_keys;   // rows: l * group; a workgroup takes split_keys keys
  float scale_log2, eps, out_scale;
  FastDiv div_group, div_tiles, div_splits, div_kv;
};

// Sums of a share of the keys for one row: O1 [2d], O2 [2d] (unnormalised, relative to the references), m1, l1, m2, l2
__device__ __forceinline__ size_t diff_record(const DiffParams& p, unsigned bh, unsigned row, unsigned split) {
  return (((size_t)bh * p.rows + row) * p.splits + split) * (size_t)(4 * p.d + 4);
}

template <typename T> struct Quad;
template <> struct Quad<float> { typedef f32x4 type; };
template <> struct Quad<bf16> { typedef bf16x4 type; };
__device__ __forceinline__ float group_max(float v) {     // over the four lanes 16 apart that hold a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// What a row's weights make of its sums: f1 = 1 / l1, f2 = lambda / l2; a row that sees no key has l = 0 and stays zero
__device__ __forceinline__ float inverse_or_zero(float l) { return l == 0.f ? 0.f : 1.f / l; }

// =================================================================================================
// fp32: 16 rows a workgroup, four wavefronts share the keys out in blocks of 16.  Scores are computed transposed (a lane owns a row), so the
// probabilities are the B operand of the product with v as they stand.  Column 4 m + e of a 64-wide run of v is row m of the e-th of four
// accumulator tiles: a lane's 16-byte load feeds four tiles.  An fp32 MFMA takes 32 cycles for 2 KFLOP, so operands come straight from the
// caches into registers, those of the next block while this one is multiplied.
// =================================================================================================
template <int DT>
__global__ __launch_bounds__(256, DT <= 4 ? 2 : 1) void k_diff_f32(DiffParams p) {
  constexpr int NW = 4, VT = (2 * DT + 3) / 4, PITCH = 64 * VT + 4;
  extern __shared__ __attribute__((aligned(16))) float part[];       // [wave][row][PITCH]: one map's sums; behind the columns m and l
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned vid = xcd_remap(blockIdx.x, gridDim.x);
  const unsigned bt = fast_div(vid, p.div_splits), split = vid - bt * p.splits;
  const unsigned bh = fast_div(bt, p.div_tiles), tile = bt - bh * p.tiles;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int d = p.d, w = 2 * d;
  const int len = p.key_lens ? min(max(p.key_lens[b], 0), p.lk) : p.lk;
  const int row = tile * 16 + r16;
  const bool live = row < p.rows;
  const int i = live ? (int)fast_div((unsigned)row, p.div_group) : 0, hg = live ? row - i * p.group : 0;
  // keys that this lane's row sees: 0 .. limit - 1; the workgroup's are those of its last row
  auto limit_of = [&](int query) { return p.causal ? min(max(query + (len - p.l + 1), 0), len) : len; };
  const int limit = live ? limit_of(i) : len, limit_first = limit_of((int)fast_div(tile * 16u, p.div_group));
  const int last = min((int)tile * 16 + 15, p.rows - 1);
  const int from = split * p.split_keys, to = min(from + p.split_keys, limit_of((int)fast_div((unsigned)last, p.div_group)));

  const float* const qrow = (const float*)p.q + ((size_t)b * p.l + i) * p.ldq + (size_t)(hk * p.group + hg) * w;
  const float* const kbase = (const float*)p.k + (size_t)b * p.lk * p.ldk + (size_t)hk * w;
  const float* const vbase = (const float*)p.v + (size_t)b * p.lk * p.ldv + (size_t)hk * w;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 qf[2][DT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < DT; ++c) qf[m][c] = live && 16 * c + 4 * g < d ? *(const f32x4*)(qrow + m * d + 16 * c + 4 * g) : zero;

  f32x4 o[2][VT][4];
  float top[2] = {-INFINITY, -INFINITY}, neg[2] = {__builtin_nanf(""), __builtin_nanf("")}, sum[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][t][e] = zero;

  // what the end needs is asked for now
  const int my_row = tid >> 4, c0 = 4 * (tid & 15);
  const int out_row = tile * 16 + my_row, out_rowc = min(out_row, p.rows - 1);
  const int query = fast_div((unsigned)out_rowc, p.div_group), head = hk * p.group + out_rowc - query * p.group;
  const float lam = p.lambda[head];
  f32x4 gain[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) gain[t][e] = p.gain && 64 * t + c0 < w ? p.gain[64 * t + c0 + e] : 1.f;

  f32x4 kf[2][DT], vf[VT][4];                      // of a block: k [map][chunk of row r16], v [run of 64 columns][key 4 g + r]
  // No load is left out, so that the loop can wait for just the ones it needs: columns behind the head read its first ones (q is zero there, and what such
  // columns of v give is dropped), keys behind the last read the last (their weight is zero)
  int col_k[DT], col_v[VT];
#pragma unroll
  for (int c = 0; c < DT; ++c) col_k[c] = 16 * c + 4 * g < d ? 16 * c + 4 * g : 0;
#pragma unroll
  for (int t = 0; t < VT; ++t) col_v[t] = 64 * t + 4 * r16 < w ? 64 * t + 4 * r16 : 0;
  auto fetch_k = [&](int key0) __attribute__((always_inline)) {
    const float* const krow = kbase + (size_t)min(key0 + r16, len - 1) * p.ldk;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int c = 0; c < DT; ++c) kf[m][c] = *(const f32x4*)(krow + m * d + col_k[c]);
  };
  auto fetch_v = [&](int key0) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float* const vrow = vbase + (size_t)min(key0 + 4 * g + r, len - 1) * p.ldv;
#pragma unroll
      for (int t = 0; t < VT; ++t) vf[t][r] = *(const f32x4*)(vrow + col_v[t]);
    }
  };
  if (from + 16 * wave < to) { fetch_k(from + 16 * wave); fetch_v(from + 16 * wave); }
  for (int key0 = from + 16 * wave; key0 < to; key0 += 16 * NW) {
    const int next = key0 + 16 * NW;
    f32x4 s[2] = {zero, zero}, s_odd[2] = {zero, zero};   // four chains in turn: a product waits for the one in front of it in its chain
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          f32x4& to_sum = e & 1 ? s_odd[m] : s[m];
          to_sum = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[m][c][e], qf[m][c][e], to_sum, 0, 0, 0);
        }
    s[0] += s_odd[0];
    s[1] += s_odd[1];
    fetch_k(min(next, to - 1));
    f32x4 pr[2];
    float add[2];
    auto weigh = [&](int m) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[m][r] = __builtin_amdgcn_exp2f(fmaf(s[m][r], p.scale_log2, neg[m]));
      add[m] = (pr[m][0] + pr[m][1]) + (pr[m][2] + pr[m][3]);
    };
    if (key0 + 16 > limit_first) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (key0 + 4 * g + r >= limit) s[m][r] = -INFINITY;
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      weigh(m);
      // without a reference the weights are NaN; only rows that ask for a higher one (any of their four lanes) move
      const bool redo = !(add[m] < kDiffBig);
      if (__builtin_amdgcn_ballot_w64(redo) != 0) {
        const bool move = group_max(redo ? 1.f : 0.f) != 0.f;
        const float most = group_max(fmaxf(fmaxf(s[m][0], s[m][1]), fmaxf(s[m][2], s[m][3]))) * p.scale_log2;
        const float up = move ? fmaxf(top[m], most) : top[m];
        const float keep = !move || top[m] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[m] - up);
        top[m] = up;
        neg[m] = up == -INFINITY ? 0.f : -up;
        sum[m] *= keep;
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[m][t][e] *= keep;
        weigh(m);
        if (up == -INFINITY) neg[m] = __builtin_nanf("");
      }
      sum[m] += add[m];                          // of this lane's keys; the four groups are added at the end
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int m = 0; m < 2; ++m) o[m][t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[t][r][e], pr[m][r], o[m][t][e], 0, 0, 0);
    fetch_v(min(next, to - 1));
  }

  // the wavefronts' sums meet in LDS, a map at a time; 16 threads take a row, columns 4 c .. 4 c + 3 of every run of 64
  f32x4 acc[2][VT];
  float tops[2], sums[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    sum[m] += __shfl_xor(sum[m], 16, 64);
    sum[m] += __shfl_xor(sum[m], 32, 64);
    float* const mine = part + (wave * 16 + r16) * PITCH;
    if (m) __syncthreads();
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) *(f32x4*)(mine + 64 * t + 16 * g + 4 * r) = f32x4{o[m][t][0][r], o[m][t][1][r], o[m][t][2][r], o[m][t][3][r]};
    if (g == 0) { mine[64 * VT] = top[m]; mine[64 * VT + 1] = sum[m]; }
    __syncthreads();
    float most = -INFINITY;
#pragma unroll
    for (int x = 0; x < NW; ++x) most = fmaxf(most, part[(x * 16 + my_row) * PITCH + 64 * VT]);
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[m][t] = zero;
    float den = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float* const from_wave = part + (x * 16 + my_row) * PITCH;
      const float f = most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(from_wave[64 * VT] - most);
      den += f * from_wave[64 * VT + 1];
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[m][t] += f * *(const f32x4*)(from_wave + 64 * t + c0);
    }
    tops[m] = most; sums[m] = den;
  }
  if (out_row >= p.rows) return;
  if (p.splits > 1) {
    float* const rec = p.partial + diff_record(p, bh, out_row, split);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int t = 0; t < VT; ++t)
        if (64 * t + c0 < w) *(f32x4*)(rec + m * w + 64 * t + c0) = acc[m][t];
      if (c0 == 0) { rec[2 * w + 2 * m] = tops[m]; rec[2 * w + 2 * m + 1] = sums[m]; }
    }
    return;
  }
  const float f1 = inverse_or_zero(sums[0]), f2 = lam * inverse_or_zero(sums[1]);
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < VT; ++t) {
    acc[0][t] = 64 * t + c0 < w ? acc[0][t] * f1 - acc[1][t] * f2 : zero;
#pragma unroll
    for (int e = 0; e < 4; ++e) sq = fmaf(acc[0][t][e], acc[0][t][e], sq);
  }
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) sq += __shfl_xor(sq, x, 64);
  const float r = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  float* const out = (float*)p.out + ((size_t)b * p.l + query) * p.ldo + (size_t)head * w;
#pragma unroll
  for (int t = 0; t < VT; ++t) {
    const int col = 64 * t + c0;
    if (col >= w) continue;
    *(f32x4*)(out + col) = acc[0][t] * r * gain[t];
  }
}

// =================================================================================================
// bf16.  Tiles of 64 keys and their values are brought into LDS by the load unit, two of each.  A tile of k and one of v have the same shape: 64 rows of the
// head's 2 d columns (k1 | k2), on a pitch of 128, 256 or 512 bytes; columns behind 2 d and keys behind the sample's length read as zeros.  Scores are
// computed transposed (S^T = K Q^T, a lane owns a row), so the probabilities are the B operand of O^T += V^T P^T as they stand; V^T fragments are read from
// the row-major tile by the transposing LDS read, four keys of a column at a time.
//
// A wavefront owns 32 rows and one map, WR x 2 of them share the tiles; the second map's sums go to the first's wavefront through LDS at the end.  (Both maps
// in a wavefront read every fragment of v for two products, but the sums of both, 2 x 2 d a row, leave no registers to overlap anything with: 2304 x 2304, 5 heads
// of 2 x 64, two samples 66 us against 53.)  WB = 2, few rows: half of the wavefronts take every other tile half.
//
// A step of 32 keys is one straight line of MFMAs, the scores of the next block and the products of the block before, with the exponentials of this
// block between them; the order is pinned, left alone the exponentials gather behind the MFMAs.  So k runs a tile ahead of v, and a barrier every two steps is enough.
//
// Probabilities are rounded to bf16 for the product with v, and the row's sum is of the rounded ones (half the instructions of a sum in front of the
// rounding; the weights then add up to 1); scores, sums and references are fp32; q is not scaled in front of the product (a rounding less).  The difference of the maps
// is smaller than the maps, so those roundings would leave a result 1.53 to 1.55 times as far off as one that is only rounded at the end (relative L2, scores of
// variance 1); the first 16 of every 64 keys go into the product in two parts, the second what the rounding dropped, which share their fragments of v: 1.43 times, for 11 to 13 % of the
// time (all keys in two parts: for twice the products with v).
//
// Bound: narrow heads by vector instructions (about 60 a step beside 7 MFMAs at d = 32), wide ones by the MFMAs (19 to 22 ns each on random numbers, 17 on constants); at 9216 x 9216
// the clock falls to 1.9 GHz.  us: 2 x 9216 x 9216, 5 heads of 2 x 32 414 (790 TFLOP/s at 12 d operations a pair), 2 x 2304 x 2304, 5 of 2 x 64 56 (725; 180 workgroups on
// 256 CUs), 1511 x 6007 causal, 8 of 2 x 128 on 2 153 (637; 190 workgroups), one token x 8190 13.5.
// =================================================================================================
// f(0), f(1), .. f(N - 1) with constants: a loop of this length is not unrolled by itself, and arrays indexed in it would go to memory
template <int N, typename F> __device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (N > 0) {
    unrolled<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}
constexpr int diff_pitch(int nc) { return nc <= 2 ? 128 : nc <= 4 ? 256 : 512; }

template <int NC, int WR, int WB, int OCC>
__global__ __launch_bounds__(128 * WR * WB, OCC) void k_diff_mfma(DiffParams p) {
  constexpr int PITCH = diff_pitch(NC), CPR = PITCH / 16, KEYS = 64 * WB, TILE = KEYS * PITCH, NW = 2 * WR * WB, LPT = TILE / 1024 / NW;
  static_assert(LPT >= 1, "every wavefront loads");
  extern __shared__ __attribute__((aligned(128))) char lds[];      // two tiles of k, two of v
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const bool low = half == 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), map = wave & 1, my_block = (wave >> 1) % WB, row_wave = (wave >> 1) / WB;
  const unsigned vid = xcd_remap(blockIdx.x, gridDim.x);
  const unsigned bt = fast_div(vid, p.div_splits), split = vid - bt * p.splits;
  const unsigned bh = fast_div(bt, p.div_tiles), tile = bt - bh * p.tiles;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int d = p.d, w = 2 * d;
  const int len = __builtin_amdgcn_readfirstlane(p.key_lens ? min(max(p.key_lens[b], 0), p.lk) : p.lk);
  auto limit_of = [&](int row) {
    return p.causal ? min(max((int)fast_div((unsigned)min(row, p.rows - 1), p.div_group) + (len - p.l + 1), 0), len) : len;
  };
  const int row0 = tile * (32 * WR) + 32 * row_wave, row = row0 + l32;
  const int rowc = min(row, p.rows - 1);                       // rows behind the last repeat it, and are not stored
  const int i = (int)fast_div((unsigned)rowc, p.div_group), hg = rowc - i * p.group;
  const int limit = limit_of(row), lim_first = limit_of(row0);
  const int from = split * p.split_keys, to = min(from + p.split_keys, limit_of(tile * (32 * WR) + 32 * WR - 1));
  const int ntiles = to > from ? (to - from + KEYS - 1) / KEYS : 0;

  // ---- tile loads
  const bf16* const kbase = (const bf16*)p.k + (size_t)b * p.lk * p.ldk + (size_t)hk * w;
  const bf16* const vbase = (const bf16*)p.v + (size_t)b * p.lk * p.ldv + (size_t)hk * w;
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds + wave * 1024u;
  struct Stream { const bf16* at; int left; };                 // the next tile, and the keys from its first on
  Stream next_k{kbase + (size_t)from * p.ldk, len - from}, next_v{vbase + (size_t)from * p.ldv, len - from};
  // descriptor of the next tile; behind the last one nothing lies in range
  auto next_tile = [&](Stream& n, int ld) __attribute__((always_inline)) {
    u32x4 rsrc = make_rsrc_words(n.at, n.left > 0 ? (unsigned)((min(n.left, KEYS) - 1) * ld + w) * 2u : 0u);
#pragma unroll
    for (int e = 0; e < 4; ++e) rsrc[e] = __builtin_amdgcn_readfirstlane(rsrc[e]);     // a descriptor lies in scalar registers
    n.at += (size_t)KEYS * ld;
    n.left -= KEYS;
    return rsrc;
  };
  auto piece = [&](const u32x4& rsrc, int ld, unsigned at, int x, auto swizzle) __attribute__((always_inline)) {
    const int id = (x * NW + wave) * 64 + lane, r = id / CPR, c = (id % CPR) ^ swizzle(r);
    dma_load16(rsrc, c * 8 < w ? (unsigned)(r * ld) * 2u + c * 16u : kOob, 0u, at + x * NW * 1024u);
  };
  auto piece_k = [&](const u32x4& rsrc, int slot, int x) __attribute__((always_inline)) {
    piece(rsrc, p.ldk, lds_base + slot * TILE, x, [](int r) { return PITCH == 128 ? (r >> 1) & 7 : r & 15; });
  };
  auto piece_v = [&](const u32x4& rsrc, int slot, int x) __attribute__((always_inline)) {
    piece(rsrc, p.ldv, lds_base + (2 + slot) * TILE, x, [](int r) { return PITCH == 128 ? (r << 1) & 4 : (r & 3) << 2; });
  };
  if (ntiles > 0) {
    const u32x4 rk = next_tile(next_k, p.ldk), rv = next_tile(next_v, p.ldv);
#pragma unroll
    for (int x = 0; x < LPT; ++x) piece_k(rk, 0, x);
#pragma unroll
    for (int x = 0; x < LPT; ++x) piece_v(rv, 0, x);
  }

  // what the end needs is asked for now: the gains go behind the tiles, a wavefront of the second map keeps lambda
  float* const gains = (float*)(lds + 4 * TILE);
  for (int at = tid; at < w; at += 64 * NW) gains[at] = p.gain ? p.gain[at] : 1.f;
  const int head = hk * p.group + hg;
  const float lam = p.lambda[head];

  // ---- queries: B operand of the score product
  const bf16* const qrow = (const bf16*)p.q + ((size_t)b * p.l + i) * p.ldq + (size_t)(hk * p.group + hg) * w + map * d;
  bf16x8 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) qf[c][e] = (bf16)0.f;
    if (16 * c + 8 * half < d) qf[c] = *(const bf16x8*)(qrow + 16 * c + 8 * half);
  }
  f32x16 o[NC], s[2];
  bf16x8 pb[2][2], dropped;                                    // weights; what the rounding of a tile's first 16 dropped
  float m_ref = -INFINITY, neg = __builtin_nanf(""), l_run = 0.f;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) { pb[1][0][e] = (bf16)0.f; pb[1][1][e] = (bf16)0.f; }

  // fragments.  K: row l32 of block j, 16-byte chunk map * d / 8 + 2 c + half at its swizzled place
  const int k_swz = PITCH == 128 ? (l32 >> 1) & 7 : l32 & 15, k_chunk = map * (d >> 3) + half;
  unsigned k_at[NC];                                           // in tile 0 or 1 of k (of which the last step read)
#pragma unroll
  for (int c = 0; c < NC; ++c) k_at[c] = (my_block * 64 + l32) * PITCH + (((k_chunk + 2 * c) ^ k_swz) << 4);
  auto k_frag = [&](int j, int c) __attribute__((always_inline)) { return *(const bf16x8*)(lds + k_at[c] + j * 32 * PITCH); };
  // V^T, n: tile of 32 columns n / 2, keys 16 (n % 2) .. of the block.  The 16 lanes of a group read four keys' 16 columns; lane x of a group addresses
  // key x / 4, columns 4 (x % 4)
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const int x16 = lane & 15, v_row = 4 * half + (x16 >> 2), v_chunk = 2 * ((lane >> 4) & 1) + ((x16 & 3) >> 1);
  const int v_swz = PITCH == 128 ? (v_row << 1) & 4 : (v_row & 3) << 2;
  constexpr int VA = NC < 4 ? NC : 4;                          // tiles 4 .. 7 lie 256 bytes behind tiles 0 .. 3
  unsigned v_at[VA];
#pragma unroll
  for (int t = 0; t < VA; ++t) v_at[t] = 2 * TILE + (my_block * 64 + v_row) * PITCH + 8 * (x16 & 1) + (((4 * t + v_chunk) ^ v_swz) << 4);
  auto v_frag = [&](int j, int n) __attribute__((always_inline)) {
    const char* const at = lds + v_at[(n >> 1) % 4] + (n >> 3) * 256 + (32 * j + 16 * (n & 1)) * PITCH;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
    const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * PITCH));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const bf16x2 ones = {(bf16)1.f, (bf16)1.f};
  // weights from registers r and r + 1 of the scores; returns the row's sum with them
  auto weigh = [&](int x, int r, float sum) __attribute__((always_inline)) {
    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[x][r], p.scale_log2, neg)), e1 = __builtin_amdgcn_exp2f(fmaf(s[x][r + 1], p.scale_log2, neg));
    const bf16x2 e = {(bf16)e0, (bf16)e1};
    pb[x][r >> 3][r & 7] = e[0];
    pb[x][r >> 3][(r & 7) + 1] = e[1];
    if (x == 0 && r < 8) {
      dropped[r] = (bf16)(e0 - (float)e[0]);
      dropped[r + 1] = (bf16)(e1 - (float)e[1]);
    }
    return __builtin_amdgcn_fdot2_f32_bf16(e, ones, sum, false);
  };
  // A step, in one straight line: the scores of the next block, the products of the block before with its values, and between those MFMAs the weights of
  // this block, x its place in its tile, and what else goes beside MFMA g.  Fragments are asked for AHEAD MFMAs early.
  constexpr int NM = 3 * NC;
  auto step = [&](int x, auto&& beside) __attribute__((always_inline)) {
    constexpr int AHEAD = 3;
    bf16x8 fr[AHEAD + 1];
    auto fetch = [&](int g) { fr[g % (AHEAD + 1)] = g < NC ? k_frag(1 - x, g) : v_frag(1 - x, g - NC); };
#pragma unroll
    for (int g = 0; g < AHEAD; ++g) fetch(g);
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) s[1 - x][r] = 0.f;
    unrolled<NM>([&](auto g_) __attribute__((always_inline)) {
      constexpr int g = decltype(g_)::value;
#pragma unroll
      for (int e = (8 * g + NM - 1) / NM; e < (8 * (g + 1) + NM - 1) / NM; ++e) sum[e & 1] = weigh(x, 2 * e, sum[e & 1]);
      if constexpr (g + AHEAD < NM) fetch(g + AHEAD);
      const bf16x8& f = fr[g % (AHEAD + 1)];
      if constexpr (g < NC) s[1 - x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[g], s[1 - x], 0, 0, 0);
      else o[(g - NC) >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pb[1 - x][(g - NC) & 1], o[(g - NC) >> 1], 0, 0, 0);
      if constexpr (g >= NC && (g - NC) % 2 == 0)
        if (x == 1) o[(g - NC) >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, dropped, o[(g - NC) >> 1], 0, 0, 0);
      beside(g_);
      __builtin_amdgcn_sched_barrier(0);
    });
    return sum[0] + sum[1];
  };
  // whether some row does not see all of block x of tile t
  auto masked = [&](int t, int x) { return from + KEYS * t + 64 * my_block + 32 * x + 32 > lim_first; };
  auto mask = [&](int t, int x) __attribute__((always_inline)) {
    if (masked(t, x)) {
      const int kb = from + KEYS * t + 64 * my_block + 32 * x + 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (kb + 8 * (r >> 2) + (r & 3) >= limit) s[x][r] = -INFINITY;
    }
  };
  // takes a block's sum of weights in, or raises the reference first.  Without a reference the weights are NaN.  Only rows that ask for it (either half)
  // move: what a row gives does not depend on the rows beside it
  auto settle = [&](int x, float sum) __attribute__((always_inline)) {
    const bool redo = !(sum < kDiffBig);
    if (__builtin_amdgcn_ballot_w64(redo) != 0) {
      const float mine = redo ? 1.f : 0.f;
      const bool move = mine + other_half(mine, low) != 0.f;
      float a = s[x][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) a = fmaxf(a, s[x][r]);
      a = fmaxf(a, other_half(a, low)) * p.scale_log2;
      const float up = move ? fmaxf(m_ref, a) : m_ref;
      const float keep = !move || m_ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_ref - up);
      m_ref = up;
      neg = up == -INFINITY ? 0.f : -up;
      l_run *= keep;
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= keep;
      sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; r += 2) sum = weigh(x, r, sum);
      if (up == -INFINITY) neg = __builtin_nanf("");
    }
    l_run += sum;
  };

  if (ntiles > 0) {
    // in front of the first block the weights are zero; what they are multiplied with must not be NaN
    for (int at = tid * 16; at < TILE; at += 16 * 64 * NW) *(f32x4*)(lds + 3 * TILE + at) = f32x4{0.f, 0.f, 0.f, 0.f};
    wait_vmcnt<0>();
    __syncthreads();
    {
      const u32x4 rk = next_tile(next_k, p.ldk);
#pragma unroll
      for (int x = 0; x < LPT; ++x) piece_k(rk, 1, x);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(0, c), qf[c], s[0], 0, 0, 0);
#pragma unroll
    for (int t = 0; t < VA; ++t) v_at[t] ^= TILE;
#pragma unroll 1
    for (int t = 0; t < ntiles; ++t) {
      mask(t, 0);
      settle(0, step(0, [](auto) {}));                                   // k: tile t, v: tile t - 1
#pragma unroll
      for (int c = 0; c < NC; ++c) k_at[c] ^= TILE;
#pragma unroll
      for (int c = 0; c < VA; ++c) v_at[c] ^= TILE;
      // tile t + 1 of k and tile t of v have landed, and everybody is done with tile t of k and tile t - 1 of v
      wait_vmcnt<0>();
      __syncthreads();
      const u32x4 rk = next_tile(next_k, p.ldk), rv = next_tile(next_v, p.ldv);
      mask(t, 1);
      // k: tile t + 1 (behind the last tile: zeros, not used), v: tile t.  The loads of k's tile t + 2 and v's t + 1 are spread over the step: all at once they
      // fill the load unit's queue, and the wavefront waits
      settle(1, step(1, [&](auto g_) __attribute__((always_inline)) {
        constexpr int g = decltype(g_)::value, N = 2 * LPT;
#pragma unroll
        for (int x = N * g / NM; x < N * (g + 1) / NM; ++x) {
          if (x < LPT) piece_k(rk, t & 1, x);
          else piece_v(rv, (t + 1) & 1, x - LPT);
        }
      }));
    }
#pragma unroll
    for (int n = 0; n < 2 * NC; ++n) o[n >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(1, n), pb[1][n & 1], o[n >> 1], 0, 0, 0);
  }

  wait_vmcnt<0>();                                             // the last tiles' loads write LDS too
  l_run += other_half(l_run, low);
  // sums change hands in LDS, four registers of all lanes at a time
  auto quad = [&](int t, int q4) { return f32x4{o[t][4 * q4], o[t][4 * q4 + 1], o[t][4 * q4 + 2], o[t][4 * q4 + 3]}; };
  if constexpr (WB > 1) {
    // the other blocks' wavefronts hand theirs to the first's
    constexpr int HAND = (4 * NC + 1) * 64;                    // quads
    static_assert((WB - 1) * 2 * WR * HAND * 16 <= 4 * TILE, "the sums");
    f32x4* const mine = (f32x4*)lds + (row_wave * 2 + map) * (WB - 1) * HAND + lane;
    __syncthreads();
    if (my_block > 0) {
      f32x4* const at = mine + (my_block - 1) * HAND;
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) at[(4 * t + q4) * 64] = quad(t, q4);
      at[4 * NC * 64] = f32x4{m_ref, l_run, 0.f, 0.f};
    }
    __syncthreads();
    if (my_block == 0) {
#pragma unroll 1
      for (int g = 0; g < WB - 1; ++g) {
        const f32x4* const at = mine + g * HAND;
        const f32x4 ml = at[4 * NC * 64];
        const float up = fmaxf(m_ref, ml[0]), ref = up == -INFINITY ? 0.f : up;
        const float f0 = __builtin_amdgcn_exp2f(m_ref - ref), f1 = __builtin_amdgcn_exp2f(ml[0] - ref);
        m_ref = up;
        l_run = l_run * f0 + ml[1] * f1;
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const f32x4 x = at[(4 * t + q4) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][4 * q4 + e] = o[t][4 * q4 + e] * f0 + x[e] * f1;
          }
      }
    }
  }
  if (p.splits > 1) {
    if (my_block == 0 && row < p.rows) {
      float* const rec = p.partial + diff_record(p, bh, row, split);
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int col = 32 * t + 8 * q4 + 4 * half;
          if (col < w) *(f32x4*)(rec + map * w + col) = quad(t, q4);
        }
      if (low) { rec[2 * w + 2 * map] = m_ref; rec[2 * w + 2 * map + 1] = l_run; }
    }
    return;
  }
  // the second map's wavefront hands lambda o2 / l2 to the first's
  static_assert(WR * 16 * NC * 64 * 4 <= 4 * TILE, "a map's results");
  f32x4* const at = (f32x4*)lds + row_wave * (4 * NC * 64) + lane;
  __syncthreads();
  if (map == 1 && my_block == 0) {
    const float f2 = lam * inverse_or_zero(l_run);
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) at[(4 * t + q4) * 64] = quad(t, q4) * f2;
  }
  __syncthreads();
  if (map == 1 || my_block > 0) return;
  const float f1 = inverse_or_zero(l_run);
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 x = quad(t, q4) * f1 - at[(4 * t + q4) * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[t][4 * q4 + e] = x[e];
        sq = fmaf(x[e], x[e], sq);                             // columns behind 2 d are zero
      }
    }
  sq += other_half(sq, low);
  const float r0 = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  if (row >= p.rows) return;
  bf16* const out = (bf16*)p.out + ((size_t)b * p.l + i) * p.ldo + (size_t)head * w;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int col = 32 * t + 8 * q4 + 4 * half;
      if (col >= w) continue;
      const f32x4 g4 = *(const f32x4*)(gains + col);
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[t][4 * q4 + e] * r0 * g4[e]);
      *(bf16x4*)(out + col) = v;
    }
}

// =================================================================================================
// bf16, up to 96 keys and heads of 2 x 64 (image tokens against a text): all keys and values of a head lie in LDS, a wavefront takes 32 rows and holds the
// scores of both maps in registers.  So the weights of both are known before the product with v, their difference is rounded once, and one product
// does for both maps (8 d operations a pair instead of 12 d).  Bound by the chain load - scores - softmax - product - store and its vector instructions (about
// 650 for 32 rows of 77 keys, both maps; masks only in blocks where a row does not see all: 982 with them everywhere, 15.6 us).
// 2 x 9216 x 77, 5 heads of 2 x 32 (24 MB): 12.4 us, the kernel above 14.9; 2 x 36864 x 77 35 us, 2.7 TB/s.
// =================================================================================================
template <int NC, int NB>
__global__ __launch_bounds__(256, NC <= 2 ? 3 : 2) void k_diff_short(DiffParams p) {
  constexpr int PITCH = diff_pitch(NC), CPR = PITCH / 16, TILE = NB * 32 * PITCH, LPT = TILE / 4096;
  extern __shared__ __attribute__((aligned(128))) char lds[];      // k, v
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const bool low = half == 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned vid = xcd_remap(blockIdx.x, gridDim.x);
  const unsigned bh = fast_div(vid, p.div_tiles), tile = vid - bh * p.tiles;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int d = p.d, w = 2 * d;
  const int len = __builtin_amdgcn_readfirstlane(p.key_lens ? min(max(p.key_lens[b], 0), p.lk) : p.lk);
  const int row = tile * 128 + wave * 32 + l32, rowc = min(row, p.rows - 1);
  const int i = (int)fast_div((unsigned)rowc, p.div_group), head = hk * p.group + rowc - i * p.group;
  auto limit_of = [&](int query) { return p.causal ? min(max(query + (len - p.l + 1), 0), len) : len; };
  const int limit = limit_of(i), lim_first = limit_of((int)fast_div((unsigned)min((int)tile * 128 + wave * 32, p.rows - 1), p.div_group));

  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds + wave * 1024u;
  auto load = [&](const void* base, int ld, unsigned at, auto swizzle) __attribute__((always_inline)) {
    // no key: nothing lies in range
    u32x4 rsrc = make_rsrc_words((const bf16*)base + (size_t)b * p.lk * ld + (size_t)hk * w, len > 0 ? (unsigned)((len - 1) * ld + w) * 2u : 0u);
#pragma unroll
    for (int e = 0; e < 4; ++e) rsrc[e] = __builtin_amdgcn_readfirstlane(rsrc[e]);
#pragma unroll
    for (int x = 0; x < LPT; ++x) {
      const int id = (x * 4 + wave) * 64 + lane, r = id / CPR, c = (id % CPR) ^ swizzle(r);
      dma_load16(rsrc, c * 8 < w && r < len ? (unsigned)(r * ld) * 2u + c * 16u : kOob, 0u, at + x * 4096u);
    }
  };
  load(p.k, p.ldk, lds_base, [](int r) { return PITCH == 128 ? (r >> 1) & 7 : r & 15; });
  load(p.v, p.ldv, lds_base + TILE, [](int r) { return PITCH == 128 ? (r << 1) & 4 : (r & 3) << 2; });
  const bf16* const qrow = (const bf16*)p.q + ((size_t)b * p.l + i) * p.ldq + (size_t)head * w;
  bf16x8 qf[2][NC];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[m][c][e] = (bf16)0.f;
      if (16 * c + 8 * half < d) qf[m][c] = *(const bf16x8*)(qrow + m * d + 16 * c + 8 * half);
    }
  const float lam = p.lambda[head];
  float* const gains = (float*)(lds + 2 * TILE);
  if (tid < w) gains[tid] = p.gain ? p.gain[tid] : 1.f;
  wait_vmcnt<0>();
  __syncthreads();

  f32x16 s[2][NB];
  const int k_swz = PITCH == 128 ? (l32 >> 1) & 7 : l32 & 15;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[m][j][r] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 f = *(const bf16x8*)(lds + (32 * j + l32) * PITCH + (((m * (d >> 3) + 2 * c + half) ^ k_swz) << 4));
        s[m][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[m][c], s[m][j], 0, 0, 0);
      }
    }
  // weights of a map: exponentials relative to the row's maximum, and what they are multiplied with
  float factor[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (32 * j + 32 > lim_first) {
        const int seen = limit - 32 * j - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) >= seen) s[m][j][r] = -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) most = fmaxf(most, s[m][j][r]);
    }
    most = fmaxf(most, other_half(most, low)) * p.scale_log2;
    const float neg = most == -INFINITY ? 0.f : -most;
    f32x4 sums = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[m][j][r] = __builtin_amdgcn_exp2f(fmaf(s[m][j][r], p.scale_log2, neg));
        sums[r & 3] += s[m][j][r];
      }
    const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    factor[m] = inverse_or_zero(sum + other_half(sum, low));
  }
  factor[1] *= lam;

  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const int x16 = lane & 15, v_row = 4 * half + (x16 >> 2), v_chunk = 2 * ((lane >> 4) & 1) + ((x16 & 3) >> 1);
  const int v_swz = PITCH == 128 ? (v_row << 1) & 4 : (v_row & 3) << 2;
  const char* const v_at = lds + TILE + v_row * PITCH + 8 * (x16 & 1);
  f32x16 o[NC];
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      bf16x8 pb;
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[e] = (bf16)fmaf(s[0][j][8 * s2 + e], factor[0], -(s[1][j][8 * s2 + e] * factor[1]));
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        const char* const at = v_at + (32 * j + 16 * s2) * PITCH + (((4 * t + v_chunk) ^ v_swz) << 4);
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * PITCH));
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7)), pb, o[t], 0, 0, 0);
      }
    }
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) sq = fmaf(o[t][r], o[t][r], sq);      // columns behind 2 d are zero
  sq += other_half(sq, low);
  const float r0 = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  if (row >= p.rows) return;
  bf16* const out = (bf16*)p.out + ((size_t)b * p.l + i) * p.ldo + (size_t)head * w;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int col = 32 * t + 8 * q4 + 4 * half;
      if (col >= w) continue;
      const f32x4 g4 = *(const f32x4*)(gains + col);
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[t][4 * q4 + e] * r0 * g4[e]);
      *(bf16x4*)(out + col) = v;
    }
}

// Joins the shares of the keys, in their order.  A workgroup a row: the shares' references and sums give one factor each, then a thread has four
// columns of a map (d threads) and every 256 / d-th share, and the shares' groups meet in LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_diff_join(DiffParams p) {
  __shared__ float factor[2][kDiffMaxSplits];
  __shared__ f32x4 meet[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned bh = blockIdx.x / (unsigned)p.rows, row = blockIdx.x - bh * p.rows;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int d = p.d, w = 2 * d, n = p.splits;
  const unsigned query = fast_div(row, p.div_group), head = hk * p.group + row - query * p.group;
  const float* const recs = p.partial + diff_record(p, bh, row, 0);
  const size_t pitch = 4 * d + 4;
  // quad `quad` of a record's 4 d sums, shares first, first + groups, ...; what is read first does not need the factors
  const int groups = 256 / d, quad = tid % d, first = tid / d;
  const bool on = first < groups;
  constexpr int UN = 16;                        // in flight: all 64 shares of a head of 2 x 64 (one token x 8190, 32 rows: 12.8 us, with four in flight 13.7)
  f32x4 x[UN];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (on && s0 + u * groups < n) x[u] = *(const f32x4*)(recs + (size_t)(s0 + u * groups) * pitch + 4 * quad);
  };
  fetch(first);
  if (wave < 2) {                                              // a wavefront a map; lane s: share s
    const bool mine = lane < n;
    const float m = mine ? recs[lane * pitch + 2 * w + 2 * wave] : -INFINITY, l = mine ? recs[lane * pitch + 2 * w + 2 * wave + 1] : 0.f;
    float most = m;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s, 64));
    const float f = most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - most);
    float inv = inverse_or_zero(wave_sum(f * l));
    if (wave == 1) inv *= -p.lambda[head];
    if (mine) factor[wave][lane] = f * inv;
  }
  __syncthreads();
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const float* const f = factor[quad >= d / 2];
  for (int s0 = first; on && s0 < n; s0 += UN * groups) {
    if (s0 > first) fetch(s0);
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (s0 + u * groups < n) acc += f[s0 + u * groups] * x[u];
  }
  meet[tid] = acc;
  __syncthreads();
  if (wave > 0) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const bool mine = lane < d / 2;                              // columns 4 lane .. 4 lane + 3 of the head
  if (mine)
    for (int g = 0; g < groups; ++g) o += meet[g * d + lane] + meet[g * d + d / 2 + lane];
  const float sq = wave_sum(o[0] * o[0] + o[1] * o[1] + o[2] * o[2] + o[3] * o[3]);
  const float r = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  if (!mine) return;
  typename Quad<T>::type res;
#pragma unroll
  for (int e = 0; e < 4; ++e) res[e] = from_f<T>(o[e] * r * (p.gain ? p.gain[4 * lane + e] : 1.f));
  *(typename Quad<T>::type*)((T*)p.out + ((size_t)b * p.l + query) * p.ldo + (size_t)head * w + 4 * lane) = res;
}

// How a call is cut up: rows a workgroup takes, and over how many workgroups the keys of a row are shared out.
// Rows, bf16: the largest tile that gives 150 workgroups.  A larger tile reads keys and values less often, and its wavefronts hide each other's waits; too few
// leave CUs idle.  us at 128 / 64 / 32 rows: 2304 x 2304, 5 heads of 2 x 64, two samples 54 (180 workgroups) / 58 / 86, one sample 52 (90) / 41 / 57;
// 1024 x 1024, 5 heads of 2 x 64 29 (40) / 23 (80) / 19; 3000 x 3000, 8 heads of 2 x 128 on 2 129 (188) / 168 / 248, 4 heads on 4 at 1511 70 (48) / 49 / 49.
// 257 to 384 workgroups of 128 rows give some CUs two and most one, where 64 rows even out: 280 of 2 x 32 / 2 x 64 105 -> 88 / 175 -> 154, 320 of 2 x 32 / 64 / 128 122 -> 104 /
// 204 -> 182 / 417 -> 337; not 500 (206 / 224, 337 / 358), 720 (425 / 456) or 180 (44 / 47).
// Keys: shared out where the tiles leave the chip idle, at least 128 each.  us with 1 / 2 / 4 / 8 / .. shares: 64 tiles of 8192 keys 79 / 50 / 33 / 40 / 53; 16 tiles
// 79 / 47 / 29 / 21 / 19 / 28; 80 tiles of 2048 keys 26 / 24 / 30; 160 tiles of 1024 keys 19 / 33: the sums' way through memory costs more than it brings.
struct DiffPlan { bool keys_in_lds; int rows_a_tile, tiles, splits; };
static DiffPlan diff_plan(int dtype, long long bh, int rows, int lk, int d) {
  DiffPlan a{};
  a.keys_in_lds = dtype == AD_BF16 && lk <= 96 && d <= 64;
  const long long large = bh * ((rows + 127) / 128);
  a.rows_a_tile = dtype == AD_F32 ? 16 : a.keys_in_lds ? 128 : large >= 150 && (large <= 256 || large > 384) ? 128 : bh * ((rows + 63) / 64) >= 150 ? 64 : 32;
  a.tiles = (rows + a.rows_a_tile - 1) / a.rows_a_tile;
  const long long want = 256 / (bh * a.tiles), most = a.keys_in_lds ? 1 : (lk + 127) / 128;
  a.splits = (int)std::max(1LL, std::min(std::min(want, most), (long long)kDiffMaxSplits));
  return a;
}
static bool diff_shape_ok(int batch, int l, int lk, int heads, int kv_heads, int d) {
  return batch >= 1 && l >= 1 && lk >= 1 && lk <= 0x7fff0000 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 1 && d <= 128 &&
         (long long)l * (heads / kv_heads) <= 0x7fffff00LL && (long long)batch * kv_heads * ((long long)l * (heads / kv_heads) / 16 + 1) <= 0x1ffffffLL;
}
static size_t diff_partial_bytes(long long bh, long long rows, int splits, int d) {
  return splits > 1 ? (size_t)(bh * rows * splits) * (4 * (size_t)d + 4) * sizeof(float) : 0;
}

// lds_bytes: beyond 64 KiB a kernel has to be told, once on every device (attr_set: a bit for each of the first 64)
template <typename K>
static ad_status launch_diff(K kern, int threads, int lds_bytes, std::atomic<unsigned long long>& attr_set, unsigned blocks, const DiffParams& p, hipStream_t s) {
  if (lds_bytes > 65536) {
    int device = 0;
    AD_HIP(hipGetDevice(&device));
    const unsigned long long bit = device < 64 ? 1ull << device : 0;
    if (!(attr_set & bit)) {
      AD_HIP(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024));
      attr_set |= bit;
    }
  }
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(threads), lds_bytes, s, p);
  AD_HIP(hipGetLastError());
  return AD_OK;
}

template <int DT>
static ad_status run_diff_f32(const DiffParams& p, unsigned blocks, hipStream_t s) {
  static std::atomic<unsigned long long> attr_set{0};
  return launch_diff(k_diff_f32<DT>, 256, 4 * 16 * (64 * ((2 * DT + 3) / 4) + 4) * 4, attr_set, blocks, p, s);
}

template <int NC, int WR, int WB, int OCC>
static ad_status run_diff_waves(const DiffParams& p, unsigned blocks, hipStream_t s) {
  static std::atomic<unsigned long long> attr_set{0};
  return launch_diff(k_diff_mfma<NC, WR, WB, OCC>, 128 * WR * WB, 4 * 64 * WB * diff_pitch(NC) + 8 * p.d, attr_set, blocks, p, s);
}
// OCC: wavefronts per SIMD that the register budget is set for; heads wider than 96 have a CU's LDS for one workgroup
template <int NC>
static ad_status run_diff_mfma(const DiffParams& p, const DiffPlan& plan, unsigned blocks, hipStream_t s) {
  constexpr int OCC = NC <= 2 ? 4 : 2, OCC_FEW = NC > 6 ? 1 : NC <= 2 ? 3 : 2;
  if (plan.rows_a_tile == 128) return run_diff_waves<NC, 4, 1, OCC>(p, blocks, s);
  if (plan.rows_a_tile == 64) return run_diff_waves<NC, 2, 1, OCC_FEW>(p, blocks, s);
  return run_diff_waves<NC, 1, NC <= 4 ? 2 : 1, OCC_FEW>(p, blocks, s);
}

template <int NC, int NB>
static ad_status run_diff_blocks(const DiffParams& p, unsigned blocks, hipStream_t s) {
  static std::atomic<unsigned long long> attr_set{0};
  return launch_diff(k_diff_short<NC, NB>, 256, 2 * NB * 32 * diff_pitch(NC) + 8 * p.d, attr_set, blocks, p, s);
}
template <int NC>
static ad_status run_diff_short(const DiffParams& p, unsigned blocks, hipStream_t s) {
  if (p.lk <= 32) return run_diff_blocks<NC, 1>(p, blocks, s);
  if (p.lk <= 64) return run_diff_blocks<NC, 2>(p, blocks, s);
  return run_diff_blocks<NC, 3>(p, blocks, s);
}

static ad_status run_diff(int dtype, DiffParams p, const DiffPlan& plan, int batch, hipStream_t s) {
  p.tiles = plan.tiles;
  p.splits = plan.splits;
  const int step = dtype == AD_BF16 ? 128 : 16;
  p.split_keys = ((p.lk + p.splits - 1) / p.splits + step - 1) / step * step;
  p.div_tiles = make_fastdiv((unsigned)p.tiles);
  p.div_splits = make_fastdiv((unsigned)p.splits);
  const unsigned blocks = (unsigned)(batch * p.kv_heads) * (unsigned)p.tiles * (unsigned)p.splits;
  const int chunks = (p.d + 15) / 16;
  ad_status st;
  if (plan.keys_in_lds) {
    if (chunks <= 2) st = run_diff_short<2>(p, blocks, s);
    else if (chunks == 3) st = run_diff_short<3>(p, blocks, s);
    else st = run_diff_short<4>(p, blocks, s);
  } else if (dtype == AD_BF16) {
    if (chunks <= 2) st = run_diff_mfma<2>(p, plan, blocks, s);
    else if (chunks == 3) st = run_diff_mfma<3>(p, plan, blocks, s);
    else if (chunks == 4) st = run_diff_mfma<4>(p, plan, blocks, s);
    else if (chunks == 5) st = run_diff_mfma<5>(p, plan, blocks, s);
    else if (chunks == 6) st = run_diff_mfma<6>(p, plan, blocks, s);
    else st = run_diff_mfma<8>(p, plan, blocks, s);
  } else {
    if (chunks <= 1) st = run_diff_f32<1>(p, blocks, s);
    else if (chunks == 2) st = run_diff_f32<2>(p, blocks, s);
    else if (chunks <= 4) st = run_diff_f32<4>(p, blocks, s);
    else st = run_diff_f32<8>(p, blocks, s);
  }
  if (st != AD_OK || p.splits <= 1) return st;
  const unsigned total = (unsigned)(batch * p.kv_heads) * (unsigned)p.rows;
  if (dtype == AD_BF16) hipLaunchKernelGGL((k_diff_join<bf16>), dim3(total), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((k_diff_join<float>), dim3(total), dim3(256), 0, s, p);
  AD_HIP(hipGetLastError());
  return AD_OK;
}

}  // namespace ad

using namespace ad;

extern "C" {

size_t ad_diff_attention_workspace_bytes(int dtype, int batch, int l, int lk, int heads, int kv_heads, int head_dim) {
  if ((dtype != AD_BF16 && dtype != AD_F32) || !diff_shape_ok(batch, l, lk, heads, kv_heads, head_dim)) return 0;
  const long long rows = (long long)l * (heads / kv_heads), bh = (long long)batch * kv_heads;
  return diff_partial_bytes(bh, rows, diff_plan(dtype, bh, (int)rows, lk, head_dim).splits, head_dim);
}

ad_status ad_diff_attention_forward(int dtype, const void* q, const void* k, const void* v, int batch, int l, int lk, int heads, int kv_heads,
                                    int head_dim, int ldq, int ldk, int ldv, int ldo, const int* key_lens, int causal, const float* lambda,
                                    const float* norm_gain, float norm_eps, float out_scale, void* out, void* workspace, size_t workspace_bytes,
                                    ad_stream stream) {
  if (dtype != AD_BF16 && dtype != AD_F32) AD_FAIL(AD_ERR_INVALID, "differential attention: bad dtype");
  if (!q || !k || !v || !lambda || !out) AD_FAIL(AD_ERR_INVALID, "differential attention: null pointer");
  if (!diff_shape_ok(batch, l, lk, heads, kv_heads, head_dim)) AD_FAIL(AD_ERR_INVALID, "differential attention: bad shape");
  const int vn = 16 / (int)esize(dtype);
  if (head_dim % vn) AD_FAIL(AD_ERR_INVALID, "differential attention: head_dim must be a multiple of %d", vn);
  const long long w = 2LL * head_dim;
  if (ldq < heads * w || ldk < kv_heads * w || ldv < kv_heads * w || ldo < heads * w) AD_FAIL(AD_ERR_INVALID, "differential attention: bad leading dimension");
  // the tile loads address up to 128 keys through 32-bit byte offsets from the first of them
  if (dtype == AD_BF16 && (ldk > (1 << 23) - 256 || ldv > (1 << 23) - 256)) AD_FAIL(AD_ERR_INVALID, "differential attention: rows of keys or values too far apart");
  if ((ldq | ldk | ldv | ldo) % vn || (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15))
    AD_FAIL(AD_ERR_INVALID, "differential attention: tensors and rows must be aligned to 16 bytes");
  if (((uintptr_t)key_lens | (uintptr_t)lambda | (uintptr_t)norm_gain) % 4 || (uintptr_t)workspace % 16) AD_FAIL(AD_ERR_INVALID, "differential attention: misaligned argument");
  if (norm_gain && (!(norm_eps > 0.f) || !std::isfinite(norm_eps))) AD_FAIL(AD_ERR_INVALID, "differential attention: eps must be above 0");
  if (!std::isfinite(out_scale)) AD_FAIL(AD_ERR_INVALID, "differential attention: bad out_scale");
  DiffParams p{};
  p.q = q; p.k = k; p.v = v; p.out = out;
  p.key_lens = key_lens; p.lambda = lambda; p.gain = norm_gain;
  p.partial = (float*)workspace;
  p.l = l; p.lk = lk; p.kv_heads = kv_heads; p.group = heads / kv_heads; p.d = head_dim;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
  p.causal = causal != 0; p.rows = l * p.group;
  p.scale_log2 = kLog2e / sqrtf((float)head_dim); p.eps = norm_eps; p.out_scale = out_scale;
  p.div_group = make_fastdiv((unsigned)p.group);
  p.div_kv = make_fastdiv((unsigned)kv_heads);
  const long long bh = (long long)batch * kv_heads;
  DiffPlan plan = diff_plan(dtype, bh, p.rows, lk, head_dim);
  if (plan.splits > 1 && (!workspace || workspace_bytes < diff_partial_bytes(bh, p.rows, plan.splits, head_dim))) plan.splits = 1;
  ProfLaunch pl(dtype == AD_BF16 ? "diff_attn_bf16" : "diff_attn_f32", 12.0 * batch * heads * head_dim * l * lk,
                2.0 * esize(dtype) * batch * head_dim * (2.0 * l * heads + 2.0 * lk * kv_heads), (hipStream_t)stream, batch * l, lk, (int)(heads * w));
  return run_diff(dtype, p, plan, batch, (hipStream_t)stream);
}

ad_status ad_diff_lambda(const float* q1, const float* k1, const float* q2, const float* k2, int n, float init, float* lambda) {
  if (!q1 || !k1 || !q2 || !k2 || !lambda || n < 1) AD_FAIL(AD_ERR_INVALID, "differential lambda: bad argument");
  double a = 0.0, b = 0.0;
  for (int i = 0; i < n; ++i) { a += (double)q1[i] * k1[i]; b += (double)q2[i] * k2[i]; }
  *lambda = (float)(std::exp(a) - std::exp(b) + (double)init);
  return AD_OK;
}

}  // extern "C"
