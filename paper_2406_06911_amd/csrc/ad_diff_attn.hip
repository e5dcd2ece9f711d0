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
template <typename T> __device__ __forceinline__ f32x4 load_quad(const T* at) {
  const typename Quad<T>::type raw = *(const typename Quad<T>::type*)at;
  return f32x4{to_f(raw[0]), to_f(raw[1]), to_f(raw[2]), to_f(raw[3])};
}
__device__ __forceinline__ float group_max(float v) {     // over the four lanes 16 apart that hold a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// What a row's weights make of its sums: f1 = 1 / l1, f2 = lambda / l2; a row that sees no key has l = 0 and stays zero
__device__ __forceinline__ float inverse_or_zero(float l) { return l == 0.f ? 0.f : 1.f / l; }

// =================================================================================================
// Any head width up to 128, on fp32 MFMA: 16 rows a workgroup, eight wavefronts share the keys out in blocks of 16.  Scores are computed
// transposed (a lane owns a row), so the probabilities are the B operand of the product with v as they stand.  Column 4 m + e of a 64-wide
// run of v is row m of the e-th of four accumulator tiles: a lane's 16-byte load feeds four tiles.
// =================================================================================================
template <typename T, int DT>
__global__ __launch_bounds__(512) void k_diff_generic(DiffParams p) {
  constexpr int NW = 8, VT = (2 * DT + 3) / 4, PITCH = 64 * VT + 4;
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
  auto limit_of = [&](int query) { return p.causal ? min(max(query + len - p.l + 1, 0), len) : len; };
  const int limit = live ? limit_of(i) : 0;
  const int last = min((int)tile * 16 + 15, p.rows - 1);
  const int from = split * p.split_keys, to = min(from + p.split_keys, limit_of((int)fast_div((unsigned)last, p.div_group)));

  const T* const qrow = (const T*)p.q + ((size_t)b * p.l + i) * p.ldq + (size_t)(hk * p.group + hg) * w;
  const T* const kbase = (const T*)p.k + (size_t)b * p.lk * p.ldk + (size_t)hk * w;
  const T* const vbase = (const T*)p.v + (size_t)b * p.lk * p.ldv + (size_t)hk * w;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 qf[2][DT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < DT; ++c) qf[m][c] = live && 16 * c + 4 * g < d ? load_quad(qrow + m * d + 16 * c + 4 * g) : zero;

  f32x4 o[2][VT][4];
  float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][t][e] = zero;

  for (int key0 = from + 16 * wave; key0 < to; key0 += 16 * NW) {
    const T* const krow = kbase + (size_t)min(key0 + r16, len - 1) * p.ldk;
    f32x4 s[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      s[m] = zero;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        const f32x4 kf = 16 * c + 4 * g < d ? load_quad(krow + m * d + 16 * c + 4 * g) : zero;
        Mma16<float>::run(kf, qf[m][c], s[m]);
      }
    }
    f32x4 vf[VT][4];                             // [run of 64 columns][key 4 g + r]
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = key0 + 4 * g + r;
      const T* const vrow = vbase + (size_t)min(key, len - 1) * p.ldv;
#pragma unroll
      for (int t = 0; t < VT; ++t) vf[t][r] = key < len && 64 * t + 4 * r16 < w ? load_quad(vrow + 64 * t + 4 * r16) : zero;
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float most = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[m][r] = key0 + 4 * g + r < limit ? s[m][r] * p.scale_log2 : -INFINITY;
        most = fmaxf(most, s[m][r]);
      }
      const float up = fmaxf(top[m], group_max(most));
      const float keep = up == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[m] - up), ref = up == -INFINITY ? 0.f : up;
      top[m] = up;
      float add = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) { s[m][r] = __builtin_amdgcn_exp2f(s[m][r] - ref); add += s[m][r]; }
      sum[m] = sum[m] * keep + add;              // of this lane's keys; the four groups are added at the end
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[m][t][e] *= keep;
#pragma unroll
          for (int r = 0; r < 4; ++r) o[m][t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[t][r][e], s[m][r], o[m][t][e], 0, 0, 0);
        }
    }
  }

  // the wavefronts' sums meet in LDS, a map at a time; 32 threads take a row, columns c, c + 32, ...
  const int my_row = tid >> 5, c0 = tid & 31;
  constexpr int CN = 2 * VT;
  float acc[2][CN], tops[2], sums[2];
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
    for (int c = 0; c < CN; ++c) acc[m][c] = 0.f;
    float den = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float* const from_wave = part + (x * 16 + my_row) * PITCH;
      const float f = most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(from_wave[64 * VT] - most);
      den += f * from_wave[64 * VT + 1];
#pragma unroll
      for (int c = 0; c < CN; ++c) acc[m][c] += f * from_wave[c0 + 32 * c];
    }
    tops[m] = most; sums[m] = den;
  }
  const int out_row = tile * 16 + my_row;
  if (out_row >= p.rows) return;
  if (p.splits > 1) {
    float* const rec = p.partial + diff_record(p, bh, out_row, split);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int c = 0; c < CN; ++c)
        if (c0 + 32 * c < w) rec[m * w + c0 + 32 * c] = acc[m][c];
      if (c0 == 0) { rec[2 * w + 2 * m] = tops[m]; rec[2 * w + 2 * m + 1] = sums[m]; }
    }
    return;
  }
  const int query = fast_div((unsigned)out_row, p.div_group), head = hk * p.group + out_row - query * p.group;
  const float f1 = inverse_or_zero(sums[0]), f2 = p.lambda[head] * inverse_or_zero(sums[1]);
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < CN; ++c) {
    acc[0][c] = c0 + 32 * c < w ? acc[0][c] * f1 - acc[1][c] * f2 : 0.f;
    sq = fmaf(acc[0][c], acc[0][c], sq);
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) sq += __shfl_xor(sq, x, 64);
  const float r = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  T* const out = (T*)p.out + ((size_t)b * p.l + query) * p.ldo + (size_t)head * w;
#pragma unroll
  for (int c = 0; c < CN; ++c) {
    const int col = c0 + 32 * c;
    if (col < w) out[col] = from_f<T>(acc[0][c] * r * (p.gain ? p.gain[col] : 1.f));
  }
}

// =================================================================================================
// bf16.  Tiles of 64 keys and their values are brought into LDS by the load unit, two stages.  A tile of k and one of v have the same shape: 64 rows of the
// head's 2 d columns (k1 | k2), on a pitch of 128, 256 or 512 bytes; columns behind 2 d and keys behind the sample's length read as zeros.  Scores are
// computed transposed (S^T = K Q^T, a lane owns a row), so the probabilities are the B operand of O^T += V^T P^T as they stand; V^T fragments are read from
// the row-major tile by the transposing LDS read, four keys of a column at a time.
//
// The exponential's reference need not be the running maximum: any value near it gives the same quotient.  It is the exact maximum of the first 32 keys
// that a row sees, and is raised (and what has been summed rescaled) when a block's sum of weights reaches 2^24, so the steady state computes no
// maximum.  A row sees a prefix of its keys, so where it sees any of a share, it sees the first.
//
// A wavefront owns 32 rows and both maps: a fragment of v serves two products.  FEW: for few rows, a workgroup takes 32 rows, and its four wavefronts take a
// map and every other block of 32 keys each; their sums meet in LDS.
//
// Probabilities are rounded to bf16 for the product with v, scores, sums and references are fp32; q is not scaled in front of the product (a rounding less).
// =================================================================================================
constexpr int diff_pitch(int nc) { return nc <= 2 ? 128 : nc <= 4 ? 256 : 512; }
constexpr float kDiffBig = 16777216.f;

template <int NC, bool FEW>
__global__ __launch_bounds__(256, NC <= 2 ? 3 : NC <= 4 ? 2 : 1) void k_diff_mfma(DiffParams p) {
  constexpr int PITCH = diff_pitch(NC), CPR = PITCH / 16, TILE = 64 * PITCH, STAGE = 2 * TILE, LPT = TILE / 4096;
  constexpr int MAPS = FEW ? 1 : 2, ROWS = FEW ? 32 : 128;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const bool low = half == 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int map0 = FEW ? wave & 1 : 0, my_block = wave >> 1;
  const unsigned vid = xcd_remap(blockIdx.x, gridDim.x);
  const unsigned bt = fast_div(vid, p.div_splits), split = vid - bt * p.splits;
  const unsigned bh = fast_div(bt, p.div_tiles), tile = bt - bh * p.tiles;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int d = p.d, w = 2 * d, d8 = d >> 3;
  const int len = __builtin_amdgcn_readfirstlane(p.key_lens ? min(max(p.key_lens[b], 0), p.lk) : p.lk);
  auto limit_of = [&](int row) {
    return p.causal ? min(max((int)fast_div((unsigned)min(row, p.rows - 1), p.div_group) + len - p.l + 1, 0), len) : len;
  };
  const int row0 = tile * ROWS + (FEW ? 0 : wave * 32), row = row0 + l32;
  const int rowc = min(row, p.rows - 1);                       // rows behind the last repeat it, and are not stored
  const int i = (int)fast_div((unsigned)rowc, p.div_group), hg = rowc - i * p.group;
  const int limit = limit_of(row), lim_first = limit_of(row0), lim_last = limit_of(row0 + 31);
  const int from = split * p.split_keys, to = min(from + p.split_keys, limit_of(tile * ROWS + ROWS - 1));
  const int ntiles = to > from ? (to - from + 63) >> 6 : 0;

  // ---- tile loads
  const bf16* const kbase = (const bf16*)p.k + (size_t)b * p.lk * p.ldk + (size_t)hk * w;
  const bf16* const vbase = (const bf16*)p.v + (size_t)b * p.lk * p.ldv + (size_t)hk * w;
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds;
  auto issue = [&](int t, int stage) {
    const int key0 = from + 64 * t, n = min(64, len - key0);
    const u32x4 rk = make_rsrc_words(kbase + (size_t)key0 * p.ldk, (unsigned)((n - 1) * p.ldk + w) * 2u);
    const u32x4 rv = make_rsrc_words(vbase + (size_t)key0 * p.ldv, (unsigned)((n - 1) * p.ldv + w) * 2u);
    const unsigned at = lds_base + stage * STAGE + wave * 1024u;
#pragma unroll
    for (int x = 0; x < LPT; ++x) {
      const int id = (x * 4 + wave) * 64 + lane, r = id / CPR, pos = id % CPR;
      const int ck = pos ^ (PITCH == 128 ? (r >> 1) & 7 : r & 15), cv = pos ^ (PITCH == 128 ? (r << 1) & 4 : (r & 3) << 2);
      dma_load16(rk, ck * 8 < w ? (unsigned)(r * p.ldk) * 2u + ck * 16u : kOob, 0u, at + x * 4096u);
      dma_load16(rv, cv * 8 < w ? (unsigned)(r * p.ldv) * 2u + cv * 16u : kOob, 0u, at + TILE + x * 4096u);
    }
  };
  if (ntiles > 0) issue(0, 0);

  // ---- queries: B operand of the score product
  const bf16* const qrow = (const bf16*)p.q + ((size_t)b * p.l + i) * p.ldq + (size_t)(hk * p.group + hg) * w;
  bf16x8 qf[MAPS][NC];
#pragma unroll
  for (int m = 0; m < MAPS; ++m)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[m][c][e] = (bf16)0.f;
      if (16 * c + 8 * half < d) qf[m][c] = *(const bf16x8*)(qrow + (map0 + m) * d + 16 * c + 8 * half);
    }
  f32x16 o[MAPS][NC];
  float m_ref[MAPS], neg[MAPS], l_run[MAPS];
#pragma unroll
  for (int m = 0; m < MAPS; ++m) {
    m_ref[m] = -INFINITY; neg[m] = 0.f; l_run[m] = 0.f;
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[m][t][r] = 0.f;
  }
  // fragment offsets in a tile: K row l32, 16-byte chunk map * d / 8 + 2 c + half at its swizzled place
  const int k_swz = PITCH == 128 ? (l32 >> 1) & 7 : l32 & 15;
  // V: the 16 lanes of a group read four keys' 16 columns; lane x of a group addresses key x / 4, columns 4 (x % 4)
  const int x16 = lane & 15, v_row = 4 * half + (x16 >> 2), v_chunk = 2 * ((lane >> 4) & 1) + ((x16 & 3) >> 1);
  const int v_swz = PITCH == 128 ? (v_row << 1) & 4 : (v_row & 3) << 2;
  const int v_base = v_row * PITCH + 8 * (x16 & 1);

  auto block = [&](const char* Ks, int j, int kb, bool masked) {
    const char* Vs = Ks + TILE;
    f32x16 s[MAPS];
#pragma unroll
    for (int m = 0; m < MAPS; ++m) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[m][r] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 kf = *(const bf16x8*)(Ks + (j * 32 + l32) * PITCH + ((((map0 + m) * d8 + 2 * c + half) ^ k_swz) << 4));
        s[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[m][c], s[m], 0, 0, 0);
      }
    }
    if (masked) {
#pragma unroll
      for (int m = 0; m < MAPS; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kb + 8 * (r >> 2) + 4 * half + (r & 3) >= limit) s[m][r] = -INFINITY;
    }
    bf16x8 pb[MAPS][2];
    auto probs = [&](int m) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[m][r], p.scale_log2, neg[m]));
        sum += e;
        pb[m][r >> 3][r & 7] = (bf16)e;
      }
      return sum;
    };
    float sum[MAPS];
    bool redo[MAPS], any = false;
#pragma unroll
    for (int m = 0; m < MAPS; ++m) {
      sum[m] = probs(m);
      redo[m] = !(sum[m] < kDiffBig) || m_ref[m] == -INFINITY;
      any |= redo[m];
    }
    if (__builtin_amdgcn_ballot_w64(any) != 0) {
#pragma unroll
      for (int m = 0; m < MAPS; ++m) {
        // only rows that asked for it (either half) move: what a row gives does not depend on the rows beside it
        const float mine = redo[m] ? 1.f : 0.f;
        const bool move = mine + other_half(mine, low) != 0.f;
        float a = s[m][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) a = fmaxf(a, s[m][r]);
        a = fmaxf(a, other_half(a, low)) * p.scale_log2;
        const float up = move ? fmaxf(m_ref[m], a) : m_ref[m];
        const float keep = !move || m_ref[m] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_ref[m] - up);
        m_ref[m] = up;
        neg[m] = up == -INFINITY ? 0.f : -up;
        l_run[m] *= keep;
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[m][t][r] *= keep;
        sum[m] = probs(m);
      }
    }
#pragma unroll
    for (int m = 0; m < MAPS; ++m) l_run[m] += sum[m];
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const char* at = Vs + (j * 32 + 16 * s2) * PITCH + v_base + (((4 * t + v_chunk) ^ v_swz) << 4);
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * PITCH));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int m = 0; m < MAPS; ++m) o[m][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[m][s2], o[m][t], 0, 0, 0);
      }
  };

  for (int t = 0; t < ntiles; ++t) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < ntiles) issue(t + 1, (t + 1) & 1);
    const char* const Ks = lds + (t & 1) * STAGE;
#pragma unroll 1
    for (int j = FEW ? my_block : 0; j < (FEW ? my_block + 1 : 2); ++j) {
      const int kb = from + 64 * t + 32 * j;
      if (kb < lim_last) block(Ks, j, kb, kb + 32 > lim_first);
    }
  }

  float l_tot[MAPS];
#pragma unroll
  for (int m = 0; m < MAPS; ++m) l_tot[m] = l_run[m] + other_half(l_run[m], low);
  float* const hand = (float*)lds;
  constexpr int HAND = (16 * NC + 2) * 64;                     // a wavefront's sums, a register of all lanes at a time
  if constexpr (FEW) {
    // the second block's wavefronts hand theirs to the first's
    __syncthreads();
    float* const at = hand + map0 * HAND + lane;
    if (my_block == 1) {
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) at[(16 * t + r) * 64] = o[0][t][r];
      at[16 * NC * 64] = m_ref[0];
      at[(16 * NC + 1) * 64] = l_tot[0];
    }
    __syncthreads();
    if (my_block == 0) {
      const float other = at[16 * NC * 64], up = fmaxf(m_ref[0], other), ref = up == -INFINITY ? 0.f : up;
      const float f0 = __builtin_amdgcn_exp2f(m_ref[0] - ref), f1 = __builtin_amdgcn_exp2f(other - ref);
      m_ref[0] = up;
      l_tot[0] = l_tot[0] * f0 + at[(16 * NC + 1) * 64] * f1;
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[0][t][r] = o[0][t][r] * f0 + at[(16 * t + r) * 64] * f1;
    }
  }
  if (p.splits > 1) {
    if ((!FEW || my_block == 0) && row < p.rows) {
      float* const rec = p.partial + diff_record(p, bh, row, split);
#pragma unroll
      for (int m = 0; m < MAPS; ++m) {
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int col = 32 * t + 8 * q4 + 4 * half;
            if (col < w) *(f32x4*)(rec + (map0 + m) * w + col) = f32x4{o[m][t][4 * q4], o[m][t][4 * q4 + 1], o[m][t][4 * q4 + 2], o[m][t][4 * q4 + 3]};
          }
        if (low) { rec[2 * w + 2 * (map0 + m)] = m_ref[m]; rec[2 * w + 2 * (map0 + m) + 1] = l_tot[m]; }
      }
    }
    return;
  }
  const int head = hk * p.group + hg;
  const float lam = p.lambda[head];
  f32x16 res[NC];
  if constexpr (FEW) {
    // the second map's wavefront hands lambda o2 / l2 to the first's
    __syncthreads();
    if (wave == 1) {
      const float f2 = lam * inverse_or_zero(l_tot[0]);
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) hand[(16 * t + r) * 64 + lane] = o[0][t][r] * f2;
    }
    __syncthreads();
    if (wave > 0) return;
    const float f1 = inverse_or_zero(l_tot[0]);
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) res[t][r] = o[0][t][r] * f1 - hand[(16 * t + r) * 64 + lane];
  } else {
    const float f1 = inverse_or_zero(l_tot[0]), f2 = lam * inverse_or_zero(l_tot[MAPS - 1]);
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) res[t][r] = o[0][t][r] * f1 - o[MAPS - 1][t][r] * f2;
  }
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < NC; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) sq = fmaf(res[t][r], res[t][r], sq);     // columns behind 2 d are zero
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
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(res[t][4 * q4 + e] * r0 * (p.gain ? p.gain[col + e] : 1.f));
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
  constexpr int UN = 4;
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

// How a call is cut up: rows a workgroup takes, and over how many workgroups the keys of a row are shared out where the rows leave the chip idle (at
// least 256 keys each)
struct DiffPlan { bool few; int rows_a_tile, tiles, splits; };
static DiffPlan diff_plan(int dtype, long long bh, int rows, int lk) {
  DiffPlan a{};
  a.few = dtype == AD_BF16 && bh * ((rows + 127) / 128) <= 256;
  a.rows_a_tile = dtype == AD_F32 ? 16 : a.few ? 32 : 128;
  a.tiles = (rows + a.rows_a_tile - 1) / a.rows_a_tile;
  const long long tiles = bh * a.tiles, want = (512 + tiles - 1) / tiles, most = (lk + 255) / 256;
  a.splits = (int)std::max(1LL, std::min(std::min(want, most), (long long)kDiffMaxSplits));
  return a;
}
static bool diff_shape_ok(int batch, int l, int lk, int heads, int kv_heads, int d) {
  return batch >= 1 && l >= 1 && lk >= 1 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 1 && d <= 128 &&
         (long long)l * (heads / kv_heads) <= 0x7fffff00LL && (long long)batch * kv_heads * ((long long)l * (heads / kv_heads) / 16 + 1) <= 0x1ffffffLL;
}
static size_t diff_partial_bytes(long long bh, long long rows, int splits, int d) {
  return splits > 1 ? (size_t)(bh * rows * splits) * (4 * (size_t)d + 4) * sizeof(float) : 0;
}

template <typename K>
static ad_status launch_diff(K kern, int threads, int lds_bytes, std::atomic<bool>& attr_set, unsigned blocks, const DiffParams& p, hipStream_t s) {
  if (lds_bytes > 65536 && !attr_set) {
    AD_HIP(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes));
    attr_set = true;
  }
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(threads), lds_bytes, s, p);
  AD_HIP(hipGetLastError());
  return AD_OK;
}

template <int DT>
static ad_status run_diff_generic(const DiffParams& p, unsigned blocks, hipStream_t s) {
  static std::atomic<bool> attr_set{false};
  return launch_diff(k_diff_generic<float, DT>, 512, 8 * 16 * (64 * ((2 * DT + 3) / 4) + 4) * 4, attr_set, blocks, p, s);
}

template <int NC>
static ad_status run_diff_mfma(const DiffParams& p, bool few, unsigned blocks, hipStream_t s) {
  constexpr int lds_bytes = 2 * 2 * 64 * diff_pitch(NC);
  static_assert(2 * (16 * NC + 2) * 64 * 4 <= lds_bytes, "the sums of two wavefronts");
  static std::atomic<bool> set_few{false}, set_many{false};
  return few ? launch_diff(k_diff_mfma<NC, true>, 256, lds_bytes, set_few, blocks, p, s) : launch_diff(k_diff_mfma<NC, false>, 256, lds_bytes, set_many, blocks, p, s);
}

static ad_status run_diff(int dtype, DiffParams p, const DiffPlan& plan, int batch, hipStream_t s) {
  p.tiles = plan.tiles;
  p.splits = plan.splits;
  const int step = dtype == AD_BF16 ? 64 : 16;
  p.split_keys = ((p.lk + p.splits - 1) / p.splits + step - 1) / step * step;
  p.div_tiles = make_fastdiv((unsigned)p.tiles);
  p.div_splits = make_fastdiv((unsigned)p.splits);
  const unsigned blocks = (unsigned)(batch * p.kv_heads) * (unsigned)p.tiles * (unsigned)p.splits;
  const int chunks = (p.d + 15) / 16;
  ad_status st;
  if (dtype == AD_BF16) {
    if (chunks <= 2) st = run_diff_mfma<2>(p, plan.few, blocks, s);
    else if (chunks == 3) st = run_diff_mfma<3>(p, plan.few, blocks, s);
    else if (chunks == 4) st = run_diff_mfma<4>(p, plan.few, blocks, s);
    else if (chunks == 5) st = run_diff_mfma<5>(p, plan.few, blocks, s);
    else if (chunks == 6) st = run_diff_mfma<6>(p, plan.few, blocks, s);
    else st = run_diff_mfma<8>(p, plan.few, blocks, s);
  } else {
    if (chunks <= 1) st = run_diff_generic<1>(p, blocks, s);
    else if (chunks == 2) st = run_diff_generic<2>(p, blocks, s);
    else if (chunks <= 4) st = run_diff_generic<4>(p, blocks, s);
    else st = run_diff_generic<8>(p, blocks, s);
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
  return diff_partial_bytes(bh, rows, diff_plan(dtype, bh, (int)rows, lk).splits, head_dim);
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
  // the tile loads address 64 keys through 32-bit byte offsets from the first of them
  if (dtype == AD_BF16 && (ldk >= (1 << 24) || ldv >= (1 << 24))) AD_FAIL(AD_ERR_INVALID, "differential attention: rows of keys or values too far apart");
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
  DiffPlan plan = diff_plan(dtype, bh, p.rows, lk);
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
