// Attention inside the documents of a packed batch.  Query i of a document with len_q
// queries and len_k keys stands at place p = len_k - len_q + i among the keys; it sees key
// j < len_k if the call is not causal or j < max(p + 1, prefix):
//   s_j = cap tanh(scale q.k_j / cap)          (cap > 0; else scale q.k_j)
//         - slope |p - j|                      (or slope times the distance of two voxels)
//   out = sum_j softmax(s)_j v_j               (zeros where no key is seen)
//
// One pass over the keys: the running maximum and sum of a row's exponentials stay in
// float32 registers beside the unnormalised output, which is rescaled when the maximum
// grows.  Scores are computed transposed, S^T = K Q^T: a lane then holds scores of one query
// only, and its exponentials are, as they lie, the second operand of out^T = V^T P^T.
// P is rounded to the rows' type for that product, which is what the matrix unit multiplies at full
// rate; sums of P are not.  The rounding is at most that of the result once more (bfloat16: 0.0019
// to 0.0023 of the result in place of 0.0014 to 0.0017, float16 0.00024 in place of 0.00021, from 8-bit pages 0.00032 in
// place of 0.00022; float32 even).  What it leaves off as a second operand, twice the products with V, would give that
// back, and takes: chunks of 1024 over pages 577 -> 739 us, over 8-bit pages 681 -> 905, 512 of float16 113 -> 141,
// single tokens 157 -> 158 and 103 -> 106.
#include "attention_device.h"

namespace spc {
namespace {
using namespace attn;

// Whether a row of the packed queries is a query that a document gives output: rows of no document
// and queries behind max_q have no partial results, and their output stays as it is.  The
// last document that starts at or before the row is the only one that can hold it.
__device__ __forceinline__ bool has_output(const AttnArgs& a, int64_t row) {
  int lo = 0;
  for (int n = a.n_docs; n > 1;) {
    const int half = n / 2;
    if (a.q_start[lo + half] <= row) lo += half, n -= half;
    else n = half;
  }
  const int64_t first = std::max(a.q_start[lo], 0);
  return row >= first && row < a.q_start[lo + 1] && row - first < a.max_q;
}

// Joins the results of up to FEW key ranges: a group of G lanes per row and head, four columns a
// lane; all maxima and sums are read together, then all outputs (11,003 rows of 8 heads of 32, three
// ranges: 34 us with a wave per row and head, 11 so).
constexpr int kFewRanges = 8;
template <typename T, int G>
__global__ __launch_bounds__(256) void k_attn_join_few(AttnArgs a) {
  const int64_t rows = a.n_q * a.heads;
  const int64_t at = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
  const int x = 4 * (threadIdx.x % G);
  if (at >= rows || x >= a.d) return;
  f32x2 ml[kFewRanges];
  float top = a.floor;
#pragma unroll
  for (int s = 0; s < kFewRanges; ++s) {
    ml[s] = s < a.splits ? a.part_ml[(int64_t)s * rows + at] : f32x2{a.floor, 0.0f};
    top = fmaxf(top, ml[s][0]);
  }
  if (!has_output(a, at / a.heads)) return;
  f32x4 p[kFewRanges];
#pragma unroll
  for (int s = 0; s < kFewRanges; ++s) {
    p[s] = f32x4{0, 0, 0, 0};  // a range without keys has written no output
    if (ml[s][1] != 0.0f) p[s] = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)s * rows + at) * a.d + x);
  }
  float sum = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < kFewRanges; ++s) {
    if (ml[s][1] == 0.0f) continue;
    const float by = __builtin_amdgcn_exp2f((ml[s][0] - top) * a.exp_by);
    sum = fmaf(ml[s][1], by, sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fmaf(p[s][j], by, v[j]);
  }
  const float inv = 1.0f / sum;
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = sum == 0.0f ? 0.0f : v[i] * inv;
  store4(static_cast<T*>(a.out) + at / a.heads * a.out_row + at % a.heads * a.out_head + x, r);
}

// Joins the results of any number of key ranges: a wave per row and head.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int64_t rows = a.n_q * a.heads;
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int lane = threadIdx.x % kWave;
  if (at >= rows || !has_output(a, at / a.heads)) return;
  // the ranges' maxima and sums, one a lane
  float top = a.floor, sum = 0.0f;
  for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, a.part_ml[(int64_t)s * rows + at][0]);
#pragma unroll
  for (int i = 1; i < kWave; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
  // their outputs: a group of lanes a range, four columns a lane
  const int wide = (a.d + 3) / 4 <= 8 ? 8 : (a.d + 3) / 4 <= 16 ? 16 : (a.d + 3) / 4 <= 32 ? 32 : 64;
  const int x = 4 * (lane % wide), groups = kWave / wide;
  f32x4 v = {0, 0, 0, 0};
  for (int s0 = 0; s0 < a.splits; s0 += kWave) {
    const int s = s0 + lane;
    float by = -1.0f;  // less than any weight: nothing to add (a weight of 0 still makes NaN of a NaN)
    if (s < a.splits) {
      const f32x2 ml = a.part_ml[(int64_t)s * rows + at];
      if (ml[1] != 0.0f) {  // a range without keys has written nothing else
        by = __builtin_amdgcn_exp2f((ml[0] - top) * a.exp_by);
        sum = fmaf(ml[1], by, sum);
      }
    }
    const int here = std::min(a.splits - s0, kWave);
    for (int i0 = 0; i0 < here; i0 += 4 * groups) {  // all lanes take part in the exchange
      f32x4 p[4];
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * groups + lane / wide;
        const float from = __shfl(by, i);
        w[u] = i < here ? from : -1.0f;
        p[u] = f32x4{0, 0, 0, 0};
        if (w[u] >= 0.0f && x < a.d)
          p[u] = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)(s0 + i) * rows + at) * a.d + x);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(p[u][j], w[u], v[j]);
    }
  }
#pragma unroll
  for (int i = 1; i < kWave; i *= 2) sum += __shfl_xor(sum, i);
  for (int i = wide; i < kWave; i *= 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], i);
  if (lane >= wide || x >= a.d) return;
  const float inv = 1.0f / sum;
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = sum == 0.0f ? 0.0f : v[i] * inv;
  store4(static_cast<T*>(a.out) + at / a.heads * a.out_row + at % a.heads * a.out_head + x, r);
}

template <typename T>
void join_t(const AttnArgs& a, hipStream_t s) {
  const int64_t rows = a.n_q * a.heads;
#define SPC_J(G) \
  hipLaunchKernelGGL((k_attn_join_few<T, G>), dim3((unsigned)((rows + 256 / G - 1) / (256 / G))), dim3(256), 0, s, a)
  if (a.splits > kFewRanges) hipLaunchKernelGGL((k_attn_join<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
  else if (a.d <= 32) SPC_J(8);
  else if (a.d <= 64) SPC_J(16);
  else if (a.d <= 128) SPC_J(32);
  else SPC_J(64);
#undef SPC_J
}

}  // namespace

// Key ranges of the many-query form: the number with the shortest estimated time.  A CU takes
// `tile` us for 64 keys of 128 queries where it has one such workgroup, and `together` of that
// for each where others cover its waits.  A launch lasts as long as its longest workgroup, or as all of
// them on 256 CUs and a part of the longest behind them; joining costs a launch and the
// partial outputs' way to memory and back, more than eight of them twice that.  (us, by 1, 2, 3, 4, 6, 8
// ranges: 4096 queries of 8 heads of 128, causal, bfloat16 88, 77, 62, 73, 72, 78; 1024 of 32
// heads of 64 20, 26, 26, 25, 28, 32; 1024 of 8 heads of 128 in float32 141, 80, 64, 49, 45, 55; voxels of two
// frames, 11,003 of 8 heads of 32, 199, 170, 159, 164, 164, 165.)
int tile_splits(int64_t groups, int64_t rows, int max_q, int max_k, int d, bool f32, bool causal) {
  const float tile = f32 ? 0.066f * d : 0.5f + 0.006f * d, together = f32 ? 0.95f : 0.65f;
  const float seen = causal ? std::max(0.5f, 1.0f - 0.5f * max_q / max_k) : 1.0f;
  const int tiles = (max_k + 63) / 64;
  const float all = groups * (tiles * seen) * tile * together / 256;
  const float join = rows * d * 8.0f * seen / 4e6f;  // of one range
  int best = 1;
  float least = INFINITY;
  for (int n = 1; n <= 32 && n <= tiles; ++n) {
    const float longest = (tiles + n - 1) / n * tile;
    const float us = std::max(longest, all + 0.7f * longest) + (n > 1 ? 5.0f + join * n * (n > kFewRanges ? 2 : 1) : 0.0f);
    if (us < least) least = us, best = n;
  }
  return best;
}

AttnPlan attention_plan(int64_t n_q, int n_docs, int max_q, int max_k, int heads, int kv_heads, int d, int dtype,
                        bool causal, bool paged) {
  AttnPlan p = {};
  const int group = heads / kv_heads;
  p.cols = (int64_t)max_q * group <= 64 ? max_q * group : 0;
  p.rows = p.cols > 0;
  // the grid's second dimension holds key heads and columns, the third the documents
  if (p.rows && (n_docs > 65535 || (int64_t)kv_heads * ((p.cols + 15) / 16) > 65535)) p.rows = false;
  // tiles of a head's queries; over pages of all queries of a key head: a document with fewer than 128 has few rows
  // in them (7 x 33 queries of 1501 keys, 12 heads of 80 on 4, float32: 86 us, so 36 with slots without gaps)
  const int64_t tile_rows = paged ? n_q * group : n_q, units = paged ? kv_heads : heads;
  p.slots = tile_rows / kQueryTile + n_docs;
  // as many for each document as the longest takes, where that is no more: none are empty if all are as long
  const int64_t most = ((int64_t)max_q * group + kQueryTile - 1) / kQueryTile;
  if (paged && most * n_docs <= p.slots) p.slots = most * n_docs, p.doc_slots = (int)most;
  int64_t splits, step;
  if (p.rows) {
    // Ranges of equal length until a launch has about 3072 workgroups (48 caches of up to 8192
    // keys, 8 key heads: 209 us with one range, 168 to 160 with 5 to 16, 178 with 22), of 256 keys at least, and
    // of 128 while there are no more than eight (one token, 32 heads of 128: 1024 keys 10.4 us by
    // four ranges, 9.2 by eight; 2048 by 16 even; 300 keys 6.7 by one, 7.7 by two).
    const int64_t work = std::max<int64_t>((int64_t)n_docs * kv_heads, 1);
    const int most = max_k < 512 ? 1 : std::max(max_k / 256, std::min(kFewRanges, max_k / 128));
    // Over pages about 1536, which begin with a chain of loads more (one token for each of 48 documents of up to
    // 2048 keys, 32 heads of 128 on 8: 8 bits 50 us with 3072, 44 so, the rows' type 69 and 62; of 8
    // documents of 16,384 75 and 67, 120 and 110; of 48 up to 8192 145 and 143, 226 and 229).
    splits = std::min<int64_t>(((paged ? 1536 : 3072) + work - 1) / work, most);
    step = 128;
  } else {
    const int64_t tiles = p.doc_slots ? p.slots : tile_rows / kQueryTile + std::min<int64_t>(n_docs, n_q);
    splits = tile_splits(tiles * units, n_q * heads, max_q, max_k, d, dtype == 0, causal);
    step = 64;
  }
  p.chunk = (int)std::max<int64_t>(step, (((int64_t)max_k + splits - 1) / splits + step - 1) / step * step);
  p.splits = std::max(1, (max_k + p.chunk - 1) / p.chunk);
  return p;
}

hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  // a row and head is joined by a wave at most
  if (a.splits > 1 && !fits_launch(a.n_q * a.heads, kWave)) return hipErrorInvalidConfiguration;
  {
    ProfScope ps(KN_ATTENTION, s);
    const hipError_t e = a.k_scale ? launch_attention_pages8(a, p, dtype, s)
                         : a.paged ? launch_attention_pages(a, p, dtype, s)
                         : p.rows  ? launch_attention_rows(a, p, dtype, s)
                                   : launch_attention_tile(a, p, dtype, s);
    if (e != hipSuccess) return e;
  }
  if (a.splits <= 1) return hipSuccess;
  ProfScope ps(KN_ATTENTION_JOIN, s);
  if (dtype == 0) join_t<float>(a, s);
  else if (dtype == 1) join_t<_Float16>(a, s);
  else join_t<__bf16>(a, s);
  return hipGetLastError();
}

}  // namespace spc
