// Differential attention for gfx950:
//   out = (softmax(q1 k1^T / sqrt d) - lambda softmax(q2 k2^T / sqrt d)) v, then an RMS norm over each head (arXiv 2410.05258).
// q1 | q2 and k1 | k2 are the two halves of a head of 2 d columns, v is 2 d wide.  Query heads that share a key head are rows of the same
// tile (row r of a key head: query r / group, head r % group of the group), so a single token still fills its tile as far as the heads allow.
#include "ad_device.h"
#include "ad_kernels.h"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace ad {

constexpr float kLog2e = 1.44269504088896341f;

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

// Joins the shares of the keys, in their order: a wavefront a row, lane j has columns j, j + 64, ...
template <typename T>
__global__ __launch_bounds__(256) void k_diff_join(DiffParams p, unsigned total) {
  const unsigned at = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (at >= total) return;
  const unsigned bh = at / p.rows, row = at - bh * p.rows;
  const unsigned b = fast_div(bh, p.div_kv), hk = bh - b * p.kv_heads;
  const int w = 2 * p.d;
  constexpr int CN = 4;
  float acc[2][CN], den[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float most = -INFINITY;
    for (int x = 0; x < p.splits; ++x) most = fmaxf(most, p.partial[diff_record(p, bh, row, x) + 2 * w + 2 * m]);
    den[m] = 0.f;
#pragma unroll
    for (int c = 0; c < CN; ++c) acc[m][c] = 0.f;
    for (int x = 0; x < p.splits; ++x) {
      const float* const rec = p.partial + diff_record(p, bh, row, x);
      const float f = most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rec[2 * w + 2 * m] - most);
      den[m] += f * rec[2 * w + 2 * m + 1];
#pragma unroll
      for (int c = 0; c < CN; ++c)
        if (lane + 64 * c < w) acc[m][c] += f * rec[m * w + lane + 64 * c];
    }
  }
  const unsigned query = fast_div(row, p.div_group), head = hk * p.group + row - query * p.group;
  const float f1 = inverse_or_zero(den[0]), f2 = p.lambda[head] * inverse_or_zero(den[1]);
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < CN; ++c) {
    acc[0][c] = acc[0][c] * f1 - acc[1][c] * f2;
    sq = fmaf(acc[0][c], acc[0][c], sq);
  }
  sq = wave_sum(sq);
  const float r = p.gain ? p.out_scale * rsqrtf(sq / (float)w + p.eps) : p.out_scale;
  T* const out = (T*)p.out + ((size_t)b * p.l + query) * p.ldo + (size_t)head * w;
#pragma unroll
  for (int c = 0; c < CN; ++c) {
    const int col = lane + 64 * c;
    if (col < w) out[col] = from_f<T>(acc[0][c] * r * (p.gain ? p.gain[col] : 1.f));
  }
}

// Where the tiles leave the chip idle the keys are shared out over workgroups, at least 256 keys each
static int diff_splits(long long tiles, int lk) {
  const long long want = (512 + tiles - 1) / tiles, most = (lk + 255) / 256;
  return (int)std::max(1LL, std::min(std::min(want, most), 64LL));
}
static bool diff_shape_ok(int batch, int l, int lk, int heads, int kv_heads, int d) {
  return batch >= 1 && l >= 1 && lk >= 1 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 1 && d <= 128 &&
         (long long)l * (heads / kv_heads) <= 0x7fffff00LL && (long long)batch * kv_heads * ((long long)l * (heads / kv_heads) / 16 + 1) <= 0x1ffffffLL;
}
static size_t diff_partial_bytes(long long bh, long long rows, int splits, int d) {
  return splits > 1 ? (size_t)(bh * rows * splits) * (4 * (size_t)d + 4) * sizeof(float) : 0;
}

template <typename T>
static ad_status run_diff(DiffParams p, int batch, int splits, hipStream_t s) {
  p.tiles = (p.rows + 15) / 16;
  p.splits = splits;
  p.split_keys = ((p.lk + splits - 1) / splits + 15) / 16 * 16;
  p.div_tiles = make_fastdiv((unsigned)p.tiles);
  p.div_splits = make_fastdiv((unsigned)splits);
  const dim3 grid((unsigned)(batch * p.kv_heads) * (unsigned)p.tiles * (unsigned)splits);
#define AD_DIFF(DT_)                                                                                                                   \
  do {                                                                                                                                 \
    constexpr int lds_bytes = 8 * 16 * (64 * ((2 * DT_ + 3) / 4) + 4) * 4;                                                             \
    static std::atomic<bool> attr_set{false};                                                                                          \
    if (lds_bytes > 65536 && !attr_set) {                                                                                              \
      AD_HIP(hipFuncSetAttribute((const void*)k_diff_generic<T, DT_>, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes));         \
      attr_set = true;                                                                                                                 \
    }                                                                                                                                  \
    hipLaunchKernelGGL((k_diff_generic<T, DT_>), grid, dim3(512), lds_bytes, s, p);                                                    \
  } while (0)
  if (p.d <= 16) AD_DIFF(1);
  else if (p.d <= 32) AD_DIFF(2);
  else if (p.d <= 64) AD_DIFF(4);
  else AD_DIFF(8);
#undef AD_DIFF
  AD_HIP(hipGetLastError());
  if (splits > 1) {
    const unsigned total = (unsigned)(batch * p.kv_heads) * (unsigned)p.rows;
    hipLaunchKernelGGL((k_diff_join<T>), dim3((total + 3) / 4), dim3(256), 0, s, p, total);
    AD_HIP(hipGetLastError());
  }
  return AD_OK;
}

}  // namespace ad

using namespace ad;

extern "C" {

size_t ad_diff_attention_workspace_bytes(int dtype, int batch, int l, int lk, int heads, int kv_heads, int head_dim) {
  if ((dtype != AD_BF16 && dtype != AD_F32) || !diff_shape_ok(batch, l, lk, heads, kv_heads, head_dim)) return 0;
  const long long rows = (long long)l * (heads / kv_heads), bh = (long long)batch * kv_heads;
  return diff_partial_bytes(bh, rows, diff_splits(bh * ((rows + 15) / 16), lk), head_dim);
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
  int splits = diff_splits(bh * ((p.rows + 15) / 16), lk);
  if (splits > 1 && (!workspace || workspace_bytes < diff_partial_bytes(bh, p.rows, splits, head_dim))) splits = 1;
  ProfLaunch pl(dtype == AD_BF16 ? "diff_attn_bf16" : "diff_attn_f32", 12.0 * batch * heads * head_dim * l * lk,
                2.0 * esize(dtype) * batch * head_dim * (2.0 * l * heads + 2.0 * lk * kv_heads), (hipStream_t)stream, batch * l, lk, (int)(heads * w));
  return dtype == AD_BF16 ? run_diff<bf16>(p, batch, splits, (hipStream_t)stream) : run_diff<float>(p, batch, splits, (hipStream_t)stream);
}

ad_status ad_diff_lambda(const float* q1, const float* k1, const float* q2, const float* k2, int n, float init, float* lambda) {
  if (!q1 || !k1 || !q2 || !k2 || !lambda || n < 1) AD_FAIL(AD_ERR_INVALID, "differential lambda: bad argument");
  double a = 0.0, b = 0.0;
  for (int i = 0; i < n; ++i) { a += (double)q1[i] * k1[i]; b += (double)q2[i] * k2[i]; }
  *lambda = (float)(std::exp(a) - std::exp(b) + (double)init);
  return AD_OK;
}

}  // extern "C"
