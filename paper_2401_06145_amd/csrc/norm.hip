// Root-mean-square norm of rows with the residual's addition before it, the result in the
// rows' type or in 8 bits with a scale for each 128 columns:
//   s = x + residual,  y = s / sqrt(mean(s^2) + eps) * gamma
//   8 bits: scale = max(max|y| / 448, 2^-126) of each 128 columns, q = e4m3(y / scale)
//
// A row is read once and stays in registers, in float32, between the sum of squares and
// the output; the norm is that of the unrounded sum.  What bounds it is memory: 16-bit
// rows with a residual move 7 bytes an element (x, residual, sum, q).  65,536 x 4096 in
// bfloat16, 1.89 GB: 305 us, 6.2 TB/s (stores through the caches cost 3 %); 11,003 x 256
// in float16 5.7 us; one token of 1024 2.2 us, of which starting the kernel is most.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;  // of a workgroup, unless a row takes more
constexpr int threads_of(int lanes) { return lanes > kThreads ? lanes : kThreads; }

struct NormArgs {
  const void* x;
  const void* res;
  const void* gamma;
  void* sum;
  void* y;
  float* scales;
  int64_t ld_x, ld_res, ld_sum, ld_y, ld_scales;
  int64_t n;
  int c;
  float eps;
};

// 1 / sqrt(m), the remainders of the root and of the quotient included.
__device__ __forceinline__ float inverse_root(float m) {
  const float s = sqrtf(m), inv = 1.0f / s;
  const float off = fmaf(-0.5f * fmaf(-s, s, m) * inv, inv, fmaf(-s, inv, 1.0f));
  return m > 0.0f && m < INFINITY ? fmaf(inv, off, inv) : inv;
}
// An output.  One that becomes 8 bits keeps the first product's remainder, and its quotient by
// the scale the quotient's: a value that a rounding carries over the middle between two e4m3
// numbers is off by a whole step.  (6567 rows of 960 in bfloat16: 567 such values, so 546; of four
// plain float32 operations 649.)  An infinite output has none.
template <bool Q8>
__device__ __forceinline__ float output(float v, float inv, float gamma) {
  const float p = v * inv, y = p * gamma;
  return Q8 && fabsf(y) < INFINITY ? fmaf(p, gamma, fmaf(v, inv, -p) * gamma) : y;
}
__device__ __forceinline__ float quotient(float y, float scale, float by) {
  const float q = y * by;
  return fmaf(fmaf(-q, scale, y), by, q);
}

// G lanes per row (a power of two up to 1024), CH chunks of 8 columns per lane.
// Chunk i of a lane is columns 8 (i G + lane): 16 neighbouring lanes hold one scale block.
template <typename T, bool Q8, int G, int CH>
__global__ __launch_bounds__(threads_of(G)) void k_rms_norm(NormArgs a) {
  constexpr int kRows = threads_of(G) / G;
  const int lane = threadIdx.x % G;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  const bool mine = row < a.n;  // a wave's other rows may still be there: no return before the shuffles
  const T* x = static_cast<const T*>(a.x) + (mine ? row : 0) * a.ld_x;
  const T* res = a.res ? static_cast<const T*>(a.res) + (mine ? row : 0) * a.ld_res : nullptr;
  float v[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int col = 8 * (i * G + lane);
    if (mine && col < a.c) {
      load8(x + col, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
  if (res) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = 8 * (i * G + lane);
      if (mine && col < a.c) {
        float r[8];
        load8(res + col, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += r[j];
        if (a.sum) store8_past(static_cast<T*>(a.sum) + row * a.ld_sum + col, v[i]);
      }
    }
  }
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(v[i][j], v[i][j], sq);
#pragma unroll
  for (int m = 1; m < (G < kWave ? G : kWave); m *= 2) sq += __shfl_xor(sq, m);
  if constexpr (G > kWave) {
    __shared__ float part[kRows][G / kWave];
    if (threadIdx.x % kWave == 0) part[threadIdx.x / G][lane / kWave] = sq;
    __syncthreads();
    sq = 0.0f;
#pragma unroll
    for (int w = 0; w < G / kWave; ++w) sq += part[threadIdx.x / G][w];
  }
  const float inv = inverse_root(sq / (float)a.c + a.eps);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int col = 8 * (i * G + lane);
    const bool in = mine && col < a.c;
    float w[8];
    if (in) {
      load8(static_cast<const T*>(a.gamma) + col, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = output<Q8>(v[i][j], inv, w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 0.0f;
    }
    if constexpr (Q8) {
      float top = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(w[j]));
#pragma unroll
      for (int m = 1; m < kScaleBlock / 8; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
      const float scale = block_scale(top), by = 1.0f / scale;
      if (in) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = quotient(w[j], scale, by);
        const u32x2 q = {pack_e4m3(w[0], w[1], w[2], w[3]), pack_e4m3(w[4], w[5], w[6], w[7])};
        __builtin_nontemporal_store(q, reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.y) + row * a.ld_y + col));
        if (lane % (kScaleBlock / 8) == 0) a.scales[row * a.ld_scales + col / kScaleBlock] = scale;
      }
    } else if (in) {
      store8_past(static_cast<T*>(a.y) + row * a.ld_y + col, w);
    }
  }
}

// Any width, stride and alignment: G lanes per row, element by element; the row is read again
// (from cache) for its output.
template <typename T, bool Q8, int G>
__global__ __launch_bounds__(kThreads) void k_rms_norm_any(NormArgs a) {
  const int lane = threadIdx.x % G;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int cols = row < a.n ? a.c : 0;  // a wave's other rows may still be there
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* res = a.res ? static_cast<const T*>(a.res) + row * a.ld_res : nullptr;
  const T* gamma = static_cast<const T*>(a.gamma);
  const auto at = [&](int col) { return (float)x[col] + (res ? (float)res[col] : 0.0f); };
  float sq = 0.0f;
  for (int col = lane; col < cols; col += G) {
    const float s = at(col);
    sq = fmaf(s, s, sq);
  }
#pragma unroll
  for (int m = 1; m < (G < kWave ? G : kWave); m *= 2) sq += __shfl_xor(sq, m);
  if constexpr (G > kWave) {
    __shared__ float part[G / kWave];
    if (lane % kWave == 0) part[lane / kWave] = sq;
    __syncthreads();
    sq = 0.0f;
#pragma unroll
    for (int w = 0; w < G / kWave; ++w) sq += part[w];
  }
  const float inv = inverse_root(sq / (float)a.c + a.eps);
  // The sum may be stored over x or the residual: each element is read before it is written,
  // and again by no other lane
  const auto out = [&](int col) {
    const float s = at(col);
    if (res && a.sum) static_cast<T*>(a.sum)[row * a.ld_sum + col] = (T)s;
    return output<Q8>(s, inv, (float)gamma[col]);
  };
  if constexpr (Q8) {
    // a wave takes a scale block at a time, two columns a lane
    for (int b = lane / kWave; b * kScaleBlock < cols; b += G / kWave) {
      const int col = b * kScaleBlock + 2 * (lane % kWave);
      float w[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (col + j < cols) w[j] = out(col + j);
      float top = fmaxf(fabsf(w[0]), fabsf(w[1]));
#pragma unroll
      for (int m = 1; m < kWave; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
      const float scale = block_scale(top), by = 1.0f / scale;
      const uint32_t q = pack_e4m3(quotient(w[0], scale, by), quotient(w[1], scale, by), 0.0f, 0.0f);
      uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.ld_y;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (col + j < cols) y[col + j] = (uint8_t)(q >> (8 * j));
      if (lane % kWave == 0) a.scales[row * a.ld_scales + b] = scale;
    }
  } else {
    for (int col = lane; col < cols; col += G) static_cast<T*>(a.y)[row * a.ld_y + col] = (T)out(col);
  }
}

// Rows from `first` on, up to `most` of them.
template <typename T, bool Q8>
NormArgs part_of(const NormArgs& a, int64_t first, int64_t most) {
  NormArgs p = a;
  const auto at = [first](const void* from, int64_t ld, int64_t e) {
    return from ? const_cast<char*>(static_cast<const char*>(from)) + first * ld * e : nullptr;
  };
  p.x = at(a.x, a.ld_x, sizeof(T));
  p.res = at(a.res, a.ld_res, sizeof(T));
  p.sum = at(a.sum, a.ld_sum, sizeof(T));
  p.y = at(a.y, a.ld_y, Q8 ? 1 : sizeof(T));
  p.scales = a.scales ? a.scales + first * a.ld_scales : nullptr;
  p.n = std::min(a.n - first, most);
  return p;
}

template <typename T, bool Q8>
void norm_t(const NormArgs& a, bool wide, hipStream_t s) {
  const int chunks = (a.c + 7) / 8;
  // more rows than one launch takes (2^31 work items, half of what it may have) go in parts
  const auto launch = [&](auto kernel, int threads, int rows) {
    const int64_t most = (int64_t)(0x7fffffff / threads) * rows;
    for (int64_t first = 0; first < a.n; first += most) {
      const NormArgs p = part_of<T, Q8>(a, first, most);
      hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n + rows - 1) / rows)), dim3(threads), 0, s, p);
    }
  };
  if (!wide || chunks > 2048) {
#define SPC_N(G) launch(k_rms_norm_any<T, Q8, G>, kThreads, kThreads / G)
    // float16 with residual, by 16, 64 and 256 lanes a row: 24,914 x 4 5.4, 6.9, 13.4 us;
    // 20,000 x 129 8.8, 11.2, 19.2; 11,000 x 515 31.7, 17.9, 20.2; 11,000 x 1001 62.8, 34.0, 27.7
    if (!Q8 && a.c <= 192) SPC_N(16);
    else if (a.c <= 640) SPC_N(64);
    else SPC_N(256);
#undef SPC_N
    return;
  }
#define SPC_N(G, CH) launch(k_rms_norm<T, Q8, G, CH>, threads_of(G), threads_of(G) / G)
  // One or two chunks a lane, so that a row's loads all fly at once and many rows fit a
  // CU: with a row of 4096 to a wave of 8 chunks a lane, 2000 rows in bfloat16 took 14.2 us
  // against 10.9 by a workgroup, 65,536 rows 339 against 303, 64 rows 8.9 against 3.8.
  // 512 lanes of one chunk are no better there (310); 8192 columns by 256 lanes of four
  // chunks 161.6 (16,384 rows) against 155.6, 16,384 columns by 256 of eight 175 (8192
  // rows) against 154; 1000 columns in float32 by a wave 7.4 (4099 rows) against 6.5.
  if (chunks <= 16) SPC_N(16, 1);
  else if (chunks <= 32) SPC_N(32, 1);
  else if (chunks <= 64) SPC_N(64, 1);
  else if (chunks <= 128) SPC_N(128, 1);
  else if (chunks <= 256) SPC_N(256, 1);
  else if (chunks <= 512) SPC_N(256, 2);
  else if (chunks <= 1024) SPC_N(512, 2);
  else SPC_N(1024, 2);
#undef SPC_N
}

}  // namespace

hipError_t launch_rms_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* gamma, void* sum,
                           int64_t ld_sum, void* y, int64_t ld_y, float* scales, int64_t ld_scales, int64_t n, int c,
                           int dtype, bool bits8, float eps, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  if (n > 0x7fffffff) return hipErrorInvalidValue;
  ProfScope ps(KN_RMS_NORM, s);
  const int64_t e = dtype == 0 ? 4 : 2;
  const auto fits = [](const void* p, int64_t ld, int64_t elem, int64_t by) {
    return !p || (reinterpret_cast<uintptr_t>(p) % by == 0 && ld * elem % by == 0);
  };
  // whole 16-byte accesses, where every row of every array allows them
  const bool wide = c % 8 == 0 && fits(x, ld_x, e, 16) && fits(res, ld_res, e, 16) && fits(gamma, 0, e, 16) &&
                    fits(sum, ld_sum, e, 16) && (bits8 ? fits(y, ld_y, 1, 8) : fits(y, ld_y, e, 16));
  const NormArgs a = {x, res, gamma, sum, y, scales, ld_x, ld_res, ld_sum, ld_y, ld_scales, n, c, eps};
#define SPC_N(T) (bits8 ? norm_t<T, true>(a, wide, s) : norm_t<T, false>(a, wide, s))
  if (dtype == 0) SPC_N(float);
  else if (dtype == 1) SPC_N(_Float16);
  else SPC_N(__bf16);
#undef SPC_N
  return hipGetLastError();
}

}  // namespace spc
