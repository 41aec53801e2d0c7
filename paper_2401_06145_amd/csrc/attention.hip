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
// P is rounded to the rows' type for that product (sums of P are not).
#include "attention_device.h"

namespace spc {
namespace {
using namespace attn;

// Joins the results of the key ranges: a wave per row and head.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int64_t rows = a.n_q * a.heads;
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int lane = threadIdx.x % kWave;
  if (at >= rows) return;
  float top = a.floor;
  for (int s = 0; s < a.splits; ++s) {
    const f32x2 ml = a.part_ml[(int64_t)s * rows + at];
    top = fmaxf(top, ml[0]);
  }
  float sum = 0.0f;
  f32x4 v = {0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
    const f32x2 ml = a.part_ml[(int64_t)s * rows + at];
    if (ml[1] == 0.0f) continue;
    const float by = __builtin_amdgcn_exp2f((ml[0] - top) * a.exp_by);
    sum = fmaf(ml[1], by, sum);
    if (4 * lane < a.d) {
      const f32x4 p = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)s * rows + at) * a.d + 4 * lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = fmaf(p[i], by, v[i]);
    }
  }
  if (4 * lane >= a.d) return;
  const float inv = 1.0f / sum;
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = sum == 0.0f ? 0.0f : v[i] * inv;
  store4(static_cast<T*>(a.out) + at / a.heads * a.out_row + at % a.heads * a.out_head + 4 * lane, r);
}

template <typename T>
void join_t(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_attn_join<T>), dim3((unsigned)((a.n_q * a.heads + 3) / 4)), dim3(256), 0, s, a);
}

}  // namespace

AttnPlan attention_plan(int64_t n_q, int n_docs, int max_q, int max_k, int heads, int kv_heads) {
  AttnPlan p = {};
  const int group = heads / kv_heads;
  p.cols = (int64_t)max_q * group <= 64 ? max_q * group : 0;
  p.rows = p.cols > 0;
  // the grid's third dimension holds the documents, or the key ranges
  if (p.rows && n_docs > 65535) p.rows = false;
  p.slots = n_q / kQueryTile + n_docs;
  const int64_t work = p.rows ? (int64_t)n_docs * kv_heads : (n_q / kQueryTile + std::min<int64_t>(n_docs, n_q)) * heads;
  // key ranges until a launch has about four workgroups per CU, of at least 128 keys
  int splits = 1;
  while (splits < 64 && work * splits < 1024 && max_k / (2 * splits) >= 128) splits *= 2;
  p.chunk = std::max(128, (int)(((int64_t)max_k + splits - 1) / splits + 127) / 128 * 128);
  p.splits = std::max(1, (max_k + p.chunk - 1) / p.chunk);
  return p;
}

hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  {
    ProfScope ps(KN_ATTENTION, s);
    const hipError_t e = p.rows ? launch_attention_rows(a, p, dtype, s) : launch_attention_tile(a, p, dtype, s);
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
