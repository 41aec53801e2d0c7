// Tokens' keys and values into the pages of their documents, and back:
//   write  token i of document t, of len_t with the new_t ones of the call, has the place
//          p = len_t - new_t + i; its row of each head goes to page table[t][p / page], row p % page
//   read   row i of document t comes from place i
// Pages hold the rows' type, or e4m3 and scale = max(max|x| / 448, 2^-126) of a row of a head.
//
// A group of lanes takes a row of one head, eight columns a lane, so that the largest magnitude is
// found in registers and a row is read once.  What bounds it is memory (45,384 rows, 8 heads of 128, bfloat16
// to 8 bits 52 us, 5.4 TB/s; back 60 us, 4.7; the rows' type 73 and 65; 48,969 rows from 8 bits to float32 123 us, 4.1,
// as its stores of eight columns fill half lines each); for a few tokens the
// chain of loads to a row's page (first rows, length, table), which the rows' own loads fly beside.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace spc {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 64;     // of a workgroup
constexpr int kStaged = 1024;     // documents whose first rows are looked through in LDS

struct CacheArgs {
  PageArgs pages;
  HeadRows rows[2];  // keys, values
  const int32_t* start;
  const int32_t* len;
  int64_t n;
  int per;  // rows of a workgroup
};

// Eight elements as they lie in memory.
template <typename T>
struct Chunk {
  u32x4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void widen(const Chunk<T>& c, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(float, (uint32_t)c.w[i / 4][i % 4]);
    else if (i % 2 == 0) unpack2<T>(c.w[0][i / 2], &v[i], &v[i + 1]);
  }
}
template <typename T>
__device__ __forceinline__ void store_past(T* p, const Chunk<T>& c) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) __builtin_nontemporal_store(c.w[i], reinterpret_cast<u32x4*>(p) + i);
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
  }
}

// The document of a row: the last one that starts at or before it (-1: none does).
template <typename Start>
__device__ __forceinline__ int document_of(Start start, int docs, int64_t row) {
  int lo = 0, n = docs;
  while (n > 0) {
    const int half = n / 2;
    if (start(lo + half) <= row) lo += half + 1, n -= half + 1;
    else n = half;
  }
  return lo - 1;
}

// A quotient with its remainder: a value that a rounding carries over the middle between two
// e4m3 numbers is off by a whole step.
__device__ __forceinline__ float quotient(float y, float scale, float by) {
  const float q = y * by;
  return fmaf(fmaf(-q, scale, y), by, q);
}

// U rows of a head (twice as many where they are 8 bits to read) are on their way to each group of lanes while it works on U others.
template <typename T, bool BITS8, bool READ, int G>
__global__ __launch_bounds__(kThreads) void k_cache(CacheArgs a) {
  constexpr int kGroups = kThreads / G, U = READ && BITS8 ? 4 : 2;
  const PageArgs& pg = a.pages;
  __shared__ int32_t first[kStaged], length[READ ? 1 : kStaged];
  __shared__ int64_t row_of[kMostRows];  // of the pages, for head 0
  constexpr int64_t kNone = -1, kNobody = -2;  // no page (zeros are read, nothing is written), no document
  const int64_t row0 = (int64_t)blockIdx.x * a.per;
  const int rows = (int)std::min<int64_t>(a.per, a.n - row0), units = 2 * pg.kv_heads;
  const int lane = threadIdx.x % G, x = 8 * lane;
  const bool in = x < pg.d;

  // A group's rows of heads: unit u (keys' heads, then values') of row r, kGroups apart.
  struct Task {
    int r, u;
  };
  const int step_r = kGroups / units, step_u = kGroups % units;
  const auto advance = [&](Task t) {
    t.r += step_r, t.u += step_u;
    if (t.u >= units) t.u -= units, ++t.r;
    return t;
  };
  Task at[U];
  at[0] = Task{(int)(threadIdx.x / G) / units, (int)(threadIdx.x / G) % units};
#pragma unroll
  for (int i = 1; i < U; ++i) at[i] = advance(at[i - 1]);
  const auto outside = [&](Task t) {
    const bool values = t.u >= pg.kv_heads;
    const HeadRows& h = a.rows[values];
    return static_cast<T*>(h.p) + (row0 + t.r) * h.row + (int64_t)(t.u - (values ? pg.kv_heads : 0)) * h.head + x;
  };
  // What a task reads: elements or bytes, and (read, 8 bits) their scale.
  typedef std::conditional_t<BITS8 && READ, u32x2, Chunk<T>> Raw;
  struct Got {
    Raw raw;
    float scale;
  };
  const auto inside = [&](Task t, int64_t* row) {
    const bool values = t.u >= pg.kv_heads;
    const int64_t of = row_of[t.r];
    *row = of < 0 ? of : of + ((int64_t)(t.u - (values ? pg.kv_heads : 0)) << pg.shift);
    return static_cast<char*>(values ? pg.v : pg.k) + (*row * pg.d + x) * (BITS8 ? 1 : (int64_t)sizeof(T));
  };
  const auto fetch = [&](Task t) {
    Got g = {};
    if (t.r >= rows || !in) return g;
    if constexpr (!READ) {
      const u32x4* p = reinterpret_cast<const u32x4*>(outside(t));
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) g.raw.w[i] = p[i];
    } else {
      int64_t row;
      const char* p = inside(t, &row);
      if (row < 0) return g;
      if constexpr (BITS8) {
        g.raw = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        g.scale = (t.u >= pg.kv_heads ? pg.v_scale : pg.k_scale)[row];
      } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) g.raw.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
      }
    }
    return g;
  };
  Got next[U];
  if (!READ) {
#pragma unroll
    for (int i = 0; i < U; ++i) next[i] = fetch(at[i]);
  }

  const bool staged = pg.n_docs <= kStaged;
  if (staged) {
    for (int i = threadIdx.x; i < pg.n_docs; i += kThreads) {
      first[i] = a.start[i];
      if (!READ) length[i] = a.len[i];
    }
    __syncthreads();
  }
  if ((int)threadIdx.x < rows) {
    const int64_t row = row0 + threadIdx.x;
    const int doc = staged ? document_of([&](int i) { return first[i]; }, pg.n_docs, row)
                           : document_of([&](int i) { return a.start[i]; }, pg.n_docs, row);
    int64_t to = kNobody;
    if (doc >= 0) {
      const int64_t begin = staged ? first[doc] : a.start[doc];
      const int64_t end = staged && doc + 1 < pg.n_docs ? first[doc + 1] : a.start[doc + 1];
      const int64_t place = READ ? row - begin : (staged ? length[doc] : a.len[doc]) - end + row;
      if (row < end) {
        to = kNone;
        if (place >= 0 && place < (int64_t)pg.table_row << pg.shift)
          to = page_row(pg, pg.table[(int64_t)doc * pg.table_row + (place >> pg.shift)], (int)place, 0);
      }
    }
    row_of[threadIdx.x] = to;
  }
  __syncthreads();
  if (READ) {
#pragma unroll
    for (int i = 0; i < U; ++i) next[i] = fetch(at[i]);
  }

  while (at[0].r < rows) {
    Got got[U];
    Task t[U];
#pragma unroll
    for (int i = 0; i < U; ++i) got[i] = next[i], t[i] = at[i];
    at[0] = advance(t[U - 1]);
#pragma unroll
    for (int i = 1; i < U; ++i) at[i] = advance(at[i - 1]);
#pragma unroll
    for (int i = 0; i < U; ++i) next[i] = fetch(at[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (t[i].r >= rows) continue;  // of all lanes of the group
      if constexpr (READ) {
        if (row_of[t[i].r] == kNobody || !in) continue;
        T* const to = outside(t[i]);
        if constexpr (BITS8) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(got[i].raw[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(got[i].raw[j], true);
            v[4 * j] = lo[0] * got[i].scale, v[4 * j + 1] = lo[1] * got[i].scale;
            v[4 * j + 2] = hi[0] * got[i].scale, v[4 * j + 3] = hi[1] * got[i].scale;
          }
          store8(to, v);
        } else {
          store_past(to, got[i].raw);
        }
      } else {
        int64_t row;
        char* const kept = inside(t[i], &row);
        if (row < 0) continue;
        if constexpr (BITS8) {
          float v[8] = {};
          float top = 0.0f;
          widen<T>(got[i].raw, v);  // (zeros in lanes that have no columns)
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
#pragma unroll
          for (int m = 1; m < G; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
          const float scale = block_scale(top), by = 1.0f / scale;
          if (!in) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = quotient(v[j], scale, by);
          *reinterpret_cast<u32x2*>(kept) = u32x2{pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])};
          if (lane == 0) (t[i].u >= pg.kv_heads ? pg.v_scale : pg.k_scale)[row] = scale;
        } else if (in) {
#pragma unroll
          for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<u32x4*>(kept)[j] = got[i].raw.w[j];
        }
      }
    }
  }
}

template <typename T, bool BITS8, bool READ>
hipError_t cache_t(CacheArgs a, hipStream_t s) {
  const auto launch = [&](auto kernel, int groups) {
    // rows of a head for each group of lanes: eight of 8 bits, four of a type (45,384 rows, 8 heads of 128, bfloat16:
    // by four, eight: 8 bits written 55, 52 us, read 65, 60; the rows' type 73, 75 and 65, 68),
    // but workgroups for all CUs first
    a.per = (int)std::min<int64_t>({std::max(1, (BITS8 ? 8 : 4) * groups / (2 * a.pages.kv_heads)), std::max<int64_t>(1, a.n / 2048), kMostRows});
    const int64_t wgs = (a.n + a.per - 1) / a.per;
    if (!fits_launch(wgs, kThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
#define SPC_G(G) launch(k_cache<T, BITS8, READ, G>, kThreads / (G))
  const int lanes = a.pages.d / 8;
  if (lanes <= 1) return SPC_G(1);
  if (lanes <= 2) return SPC_G(2);
  if (lanes <= 4) return SPC_G(4);
  if (lanes <= 8) return SPC_G(8);
  if (lanes <= 16) return SPC_G(16);
  return SPC_G(32);
#undef SPC_G
}

template <typename T>
hipError_t cache_form(const CacheArgs& a, hipStream_t s) {
  if (a.pages.k_scale) return a.len ? cache_t<T, true, false>(a, s) : cache_t<T, true, true>(a, s);
  return a.len ? cache_t<T, false, false>(a, s) : cache_t<T, false, true>(a, s);
}

}  // namespace

hipError_t launch_cache(const PageArgs& pages, const HeadRows& k, const HeadRows& v, const int32_t* start, const int32_t* len,
                        int64_t n, int dtype, hipStream_t s) {
  ProfScope ps(len ? KN_CACHE_WRITE : KN_CACHE_READ, s);
  const CacheArgs a = {pages, {k, v}, start, len, n, 1};
  if (dtype == 0) return cache_form<float>(a, s);
  if (dtype == 1) return cache_form<_Float16>(a, s);
  return cache_form<__bf16>(a, s);
}

}  // namespace spc
