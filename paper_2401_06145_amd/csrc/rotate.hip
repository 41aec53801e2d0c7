// Queries and keys before attention: the root-mean-square norm of each head, and the rotation of
// pairs of its columns by the row's position.
//   y = x / sqrt(mean(x^2) + eps) gamma            (or y = x)
//   pair j, of columns (j, j + rot / 2) or (2 j, 2 j + 1), turns by the angle p f_j:
//     (a, b) -> gain (a cos - b sin, a sin + b cos);   columns from rot on stay y
//
// A workgroup takes a few rows: first the cosines and sines of their pairs, into LDS, once for all
// heads; then a group of lanes takes a head, and a lane both columns of its pairs, so that a head is
// read once and nothing is exchanged but the sum of squares.  Angles are products of float64,
// of which whole turns are taken off before they become float32: at place 10^6 a float32 angle would
// be off by 0.06.  What bounds it is memory: 65,536 rows of 40 heads of 128 in bfloat16, 1.34 GB,
// 266 us (5.0 TB/s, what a large copy reaches; float32 as well, 20,000 rows 167 us, but 411 with pairs side by side,
// whose stores of eight columns fill half lines each); for one row the host's call (5.4 us, the kernel 3.5 under the profiler).
#include <algorithm>
#include <type_traits>

#include "rotate.h"

namespace spc {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 16;  // of a workgroup

template <typename T, int W>
struct Cols {
  typedef T Vec __attribute__((ext_vector_type(W)));
};
template <typename T>
struct Cols<T, 1> {
  typedef T Vec;
};
template <typename T, int W>
__device__ __forceinline__ void widen(const typename Cols<T, W>::Vec& c, float* v) {
  if constexpr (W == 1) {
    v[0] = (float)c;
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = (float)c[j];
  }
}
template <typename T, int W>
__device__ __forceinline__ void store_cols(T* p, const float* v) {
  if constexpr (W == 8) {
    store8_past(p, v);
  } else if constexpr (W == 4 && sizeof(T) == 2) {
    __builtin_nontemporal_store(u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])}, reinterpret_cast<u32x2*>(p));
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) p[j] = (T)v[j];
  }
}

// N cosines or sines from LDS, in accesses as wide as their place allows.
template <int N>
__device__ __forceinline__ void read_n(const float* p, float* v) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 x = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * i + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const f32x2 x = *reinterpret_cast<const f32x2*>(p);
    v[0] = x[0], v[1] = x[1];
  } else {
    v[0] = p[0];
  }
}

// A lane's part of a head: two runs of W columns, from ca and from cb on (-1: none).  Pairs lie across
// the two, or, interleaved with W > 1, inside each.
struct Part {
  int ca, cb;
  bool turned;  // (across) whether the two are pairs
};
template <int W, bool INTER>
__device__ __forceinline__ Part part_of(int i, int d, int rot) {
  const int half = rot / 2;
  if constexpr (INTER && W > 1) {
    const int c = 2 * W * i;
    return Part{c < d ? c : -1, c + W < d ? c + W : -1, false};
  }
  if (i < half / W) return INTER ? Part{2 * i, 2 * i + 1, true} : Part{W * i, half + W * i, true};
  const int c = rot + 2 * W * (i - half / W);
  return Part{c < d ? c : -1, c + W < d ? c + W : -1, false};
}

// Cosines and sines of the pairs of a workgroup's rows, [rows][rot / 2] each.
__device__ __forceinline__ void turns_of(const RotateArgs& a, int64_t row0, int rows, float* cosines, float* sines) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int r = i / half, j = i - r * half;
    const int32_t p = a.voxels ? a.pos[4 * (row0 + r) + 1 + j % 3] : a.pos[row0 + r];
    const double turns = p * (a.freq[j] * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cosines[i] = a.gain * c;
    sines[i] = a.gain * s;
  }
}

// G lanes a head, I parts of two runs of W columns a lane.
template <typename T, int W, int I, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate(RotateArgs a, int g) {
  typedef typename Cols<T, W>::Vec Vec;
  __shared__ __align__(16) float cosines[kMostRows * kMostRotated / 2], sines[kMostRows * kMostRotated / 2];
  const int half = a.rot / 2, heads = a.heads[0] + a.heads[1];
  const int64_t row0 = (int64_t)blockIdx.x * a.per;
  const int rows = (int)std::min<int64_t>(a.per, a.n - row0);
  const int head0 = blockIdx.y * a.share, mine = std::min(a.share, heads - head0);
  const int tasks = rows * mine, groups = kThreads / g, lane = threadIdx.x % g;
  Part part[I];
#pragma unroll
  for (int i = 0; i < I; ++i) part[i] = part_of<W, INTER>(lane + g * i, a.d, a.rot);

  struct Where {
    int64_t row;
    int which, head;
  };
  const auto where = [&](int t) {
    const int r = t / mine, h = head0 + t - r * mine;
    return Where{row0 + r, h >= a.heads[0], h >= a.heads[0] ? h - a.heads[0] : h};
  };
  Vec ahead[I][2];
  const auto fetch = [&](int t) {
    const Where w = where(t);
    const T* p = static_cast<const T*>(a.x[w.which]) + w.row * a.x_row[w.which] + (int64_t)w.head * a.x_head[w.which];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      ahead[i][0] = ahead[i][1] = Vec{};
      if (part[i].ca >= 0) ahead[i][0] = *reinterpret_cast<const Vec*>(p + part[i].ca);
      if (part[i].cb >= 0) ahead[i][1] = *reinterpret_cast<const Vec*>(p + part[i].cb);
    }
  };
  int t = threadIdx.x / g;
  if (t < tasks) fetch(t);

  turns_of(a, row0, rows, cosines, sines);
  __syncthreads();

  for (; t < tasks; t += groups) {
    const Where w = where(t);
    float v[I][2][W];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) widen<T, W>(ahead[i][k], v[i][k]);
    if (t + groups < tasks) fetch(t + groups);
    if (a.gamma[w.which]) {
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < W; ++j) sq = fmaf(v[i][k][j], v[i][k][j], sq);
      for (int m = 1; m < g; m *= 2) sq += __shfl_xor(sq, m);
      const float inv = 1.0f / sqrtf(sq / (float)a.d + a.eps);
      const T* gamma = static_cast<const T*>(a.gamma[w.which]);
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int c = k ? part[i].cb : part[i].ca;
          float by[W] = {};
          if (c >= 0) widen<T, W>(*reinterpret_cast<const Vec*>(gamma + c), by);
#pragma unroll
          for (int j = 0; j < W; ++j) v[i][k][j] *= inv * by[j];
        }
    }
    const float* cs = cosines + (w.row - row0) * half;
    const float* sn = sines + (w.row - row0) * half;
    T* const out = static_cast<T*>(a.y[w.which]) + w.row * a.y_row[w.which] + (int64_t)w.head * a.y_head[w.which];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      if constexpr (INTER && W > 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int c = k ? part[i].cb : part[i].ca;
          if (c >= 0 && c < a.rot) {
            float co[W / 2], si[W / 2];
            read_n<W / 2>(cs + c / 2, co);
            read_n<W / 2>(sn + c / 2, si);
#pragma unroll
            for (int j = 0; j < W / 2; ++j) {
              const float x = v[i][k][2 * j], y = v[i][k][2 * j + 1];
              v[i][k][2 * j] = x * co[j] - y * si[j];
              v[i][k][2 * j + 1] = x * si[j] + y * co[j];
            }
          }
        }
      } else if (part[i].turned) {
        const int j0 = INTER ? part[i].ca / 2 : part[i].ca;
        float co[W], si[W];
        read_n<W>(cs + j0, co);
        read_n<W>(sn + j0, si);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float x = v[i][0][j], y = v[i][1][j];
          v[i][0][j] = x * co[j] - y * si[j];
          v[i][1][j] = x * si[j] + y * co[j];
        }
      }
      if (part[i].ca >= 0) store_cols<T, W>(out + part[i].ca, v[i][0]);
      if (part[i].cb >= 0) store_cols<T, W>(out + part[i].cb, v[i][1]);
    }
  }
}

// Heads whose pairs or addresses fit no wide access (an odd width, an odd number of pairs): rows of
// heads that follow each other come through LDS in 16-byte pieces, and go back so; a lane has single pairs of
// a head, as above with W = 1.  From 2^23 elements on (41,323 rows of 20 heads of 33, 32 turned, bfloat16: element by
// element from memory 151 us, 109 so).  Six widths and types, 20 to 256 columns, of 8 to 24 heads, staged against not:
// 2^21 elements 0.99 to 1.84, 2^22 0.83 to 1.31, 2^23 0.74 to 1.13, 2^24 0.70 to 1.15, 2^25 0.67 to 1.01.  (The slow ends
// are 100 of 128 columns turned and 7 heads of 33 with pairs side by side.)  Bound by the vector unit and LDS, a few instructions an element.
constexpr int kStage = 4096;  // elements
template <typename T, int I, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate_staged(RotateArgs a, int g, int tile_rows) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float cosines[kMostRows * kMostRotated / 2], sines[kMostRows * kMostRotated / 2];
  __shared__ __align__(16) T stage[kStage + 16];
  const int half = a.rot / 2, heads = a.heads[0] + a.heads[1];
  const int64_t row0 = (int64_t)blockIdx.x * a.per;
  const int rows = (int)std::min<int64_t>(a.per, a.n - row0);
  const int groups = kThreads / g, lane = threadIdx.x % g;
  Part part[I];
#pragma unroll
  for (int i = 0; i < I; ++i) part[i] = part_of<1, INTER>(lane + g * i, a.d, a.rot);
  turns_of(a, row0, rows, cosines, sines);

  for (int r0 = 0; r0 < rows; r0 += tile_rows)
    for (int h0 = 0; h0 < heads; h0 += a.share) {
      const int nr = std::min(tile_rows, rows - r0), nh = std::min(a.share, heads - h0);
      // of the tile's heads, those of the queries and of the keys; each begins at 16 bytes
      const int of[2] = {std::max(0, std::min(nh, a.heads[0] - h0)), nh - std::max(0, std::min(nh, a.heads[0] - h0))};
      const int off = (of[0] * a.d + 7) / 8 * 8, pitch = off + (of[1] * a.d + 7) / 8 * 8;
      const auto copy = [&](auto out) {
        constexpr bool OUT = decltype(out)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int n = of[k] * a.d, first = k ? std::max(0, h0 - a.heads[0]) : h0;
          if (n == 0) continue;
          const int64_t ld = OUT ? a.y_row[k] : a.x_row[k];
          T* const base = (OUT ? static_cast<T*>(a.y[k]) : const_cast<T*>(static_cast<const T*>(a.x[k]))) + (row0 + r0) * ld + (int64_t)first * a.d;
          T* const here = stage + (k ? off : 0);
          const bool wide = reinterpret_cast<uintptr_t>(base) % 16 == 0 && ld * (int64_t)sizeof(T) % 16 == 0;
          const int pieces = wide ? n / V : 0, rest = n - pieces * V;
          for (int i = threadIdx.x; i < nr * pieces; i += kThreads) {
            const int r = i / pieces, c = (i - r * pieces) * V;
            u32x4 *const l = reinterpret_cast<u32x4*>(here + r * pitch + c), *const m = reinterpret_cast<u32x4*>(base + r * ld + c);
            if (OUT) *m = *l;
            else *l = *m;
          }
          for (int i = threadIdx.x; i < nr * rest; i += kThreads) {
            const int r = i / rest, c = pieces * V + i - r * rest;
            if (OUT) base[r * ld + c] = here[r * pitch + c];
            else here[r * pitch + c] = base[r * ld + c];
          }
        }
      };
      copy(std::false_type());
      __syncthreads();
      for (int t = threadIdx.x / g; t < nr * nh; t += groups) {
        const int r = t / nh, h = t - r * nh, k = h >= of[0];
        T* const x = stage + r * pitch + (k ? off + (h - of[0]) * a.d : h * a.d);
        float v[I][2];
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
          v[i][0] = part[i].ca >= 0 ? (float)x[part[i].ca] : 0.0f;
          v[i][1] = part[i].cb >= 0 ? (float)x[part[i].cb] : 0.0f;
          sq = fmaf(v[i][0], v[i][0], fmaf(v[i][1], v[i][1], sq));
        }
        if (a.gamma[k]) {
          for (int m = 1; m < g; m *= 2) sq += __shfl_xor(sq, m);
          const float inv = 1.0f / sqrtf(sq / (float)a.d + a.eps);
          const T* gamma = static_cast<const T*>(a.gamma[k]);
#pragma unroll
          for (int i = 0; i < I; ++i) {
            if (part[i].ca >= 0) v[i][0] *= inv * (float)gamma[part[i].ca];
            if (part[i].cb >= 0) v[i][1] *= inv * (float)gamma[part[i].cb];
          }
        }
#pragma unroll
        for (int i = 0; i < I; ++i) {
          if (part[i].turned) {
            const int j = (r0 + r) * half + (INTER ? part[i].ca / 2 : part[i].ca);
            const float p = v[i][0], q = v[i][1], co = cosines[j], si = sines[j];
            v[i][0] = p * co - q * si;
            v[i][1] = p * si + q * co;
          }
          if (part[i].ca >= 0) x[part[i].ca] = (T)v[i][0];
          if (part[i].cb >= 0) x[part[i].cb] = (T)v[i][1];
        }
      }
      __syncthreads();
      copy(std::true_type());
      __syncthreads();
    }
}

template <typename T, bool INTER>
hipError_t rotate_t(RotateArgs a, hipStream_t s) {
  // the widest runs of columns that pairs and all addresses allow
  const auto fits = [&](int w) {
    if (a.d % w != 0 || (INTER ? a.rot : a.rot / 2) % w != 0) return false;
    const int64_t by = std::min<int64_t>(16, w * sizeof(T));
    for (int k = 0; k < 2; ++k) {
      for (const void* p : {a.x[k], static_cast<const void*>(a.y[k]), a.gamma[k]})
        if (reinterpret_cast<uintptr_t>(p) % by != 0) return false;
      for (int64_t ld : {a.x_row[k], a.x_head[k], a.y_row[k], a.y_head[k]})
        if (ld * (int64_t)sizeof(T) % by != 0) return false;
    }
    return true;
  };
  const int w = fits(8) ? 8 : fits(4) ? 4 : 1;
  // parts of a head: its pairs, and what is left of its columns by two runs
  const int parts = INTER && w > 1 ? (a.d + 2 * w - 1) / (2 * w) : a.rot / 2 / w + (a.d - a.rot + 2 * w - 1) / (2 * w);
  int g = 1;
  while (g < parts && g < kWave) g *= 2;
  const int groups = kThreads / g, heads = a.heads[0] + a.heads[1];
  a.per = (int)std::min<int64_t>({std::max(1, 4 * groups / heads), std::max<int64_t>(1, a.n / 1024), kMostRows});
  a.share = heads;
  // few rows: a workgroup for as many heads as it has groups
  if (a.n < 1024) a.share = std::min(heads, groups);
  bool follow = true;  // heads of every row
  for (int k = 0; k < 2; ++k) follow = follow && (a.heads[k] <= 1 || (a.x_head[k] == a.d && a.y_head[k] == a.d));
  if (w == 1 && follow && a.n * heads * a.d >= 1 << 23) {
    a.share = std::min(heads, kStage / a.d / 8 * 8);
    const int tile_rows = a.share < heads ? 1 : std::max(1, std::min(kMostRows, kStage / (heads * a.d + 16)));
    a.per = (int)std::min<int64_t>({std::max(4, tile_rows), std::max<int64_t>(1, a.n / 1024), kMostRows});
    const int64_t wgs = (a.n + a.per - 1) / a.per;
    if (!fits_launch(wgs, kThreads)) return hipErrorInvalidConfiguration;
    if (parts <= kWave) hipLaunchKernelGGL((k_rotate_staged<T, 1, INTER>), dim3((unsigned)wgs), dim3(kThreads), 0, s, a, g, tile_rows);
    else hipLaunchKernelGGL((k_rotate_staged<T, 2, INTER>), dim3((unsigned)wgs), dim3(kThreads), 0, s, a, g, tile_rows);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((a.n + a.per - 1) / a.per), (unsigned)((heads + a.share - 1) / a.share));
  if (!fits_launch((a.n + a.per - 1) / a.per, kThreads) || grid.y > 65535) return hipErrorInvalidConfiguration;
  if (w == 8) hipLaunchKernelGGL((k_rotate<T, 8, 1, INTER>), grid, dim3(kThreads), 0, s, a, g);
  else if (w == 4) hipLaunchKernelGGL((k_rotate<T, 4, 1, INTER>), grid, dim3(kThreads), 0, s, a, g);
  else if (parts <= kWave) hipLaunchKernelGGL((k_rotate<T, 1, 1, INTER>), grid, dim3(kThreads), 0, s, a, g);
  else hipLaunchKernelGGL((k_rotate<T, 1, 2, INTER>), grid, dim3(kThreads), 0, s, a, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int dtype, bool interleaved, hipStream_t s) {
  ProfScope ps(KN_ROTATE, s);
#define SPC_R(T) (interleaved ? rotate_t<T, true>(a, s) : rotate_t<T, false>(a, s))
  if (dtype == 0) return SPC_R(float);
  if (dtype == 1) return SPC_R(_Float16);
  return SPC_R(__bf16);
#undef SPC_R
}

}  // namespace spc
