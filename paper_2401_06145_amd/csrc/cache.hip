// Tokens' keys and values into the pages of their documents, and back:
//   write  token i of document t, of len_t with the new_t ones of the call, has the place
//          p = len_t - new_t + i; its row of each head goes to page table[t][p / page], row p % page
//   read   row i of document t comes from place i
// Pages hold the rows' type, or e4m3 and scale = max(max|x| / 448, 2^-126) of a row of a head.
//
// A group of lanes takes a row of one head, eight columns a lane, so that the largest magnitude is
// found in registers and a row is read once.  What bounds it is memory; for a few tokens the
// chain of loads to a row's page (first rows, length, table), which the rows' own loads fly beside.
#include <algorithm>

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

template <typename T, bool BITS8, bool READ, int G>
__global__ __launch_bounds__(kThreads) void k_cache(CacheArgs a) {
  constexpr int kGroups = kThreads / G;
  const PageArgs& pg = a.pages;
  __shared__ int32_t first[kStaged];
  __shared__ int page_of[kMostRows], place_of[kMostRows];  // page -1: zeros (read), nothing (write); place -1: nobody's row
  const int64_t row0 = (int64_t)blockIdx.x * a.per;
  const int rows = (int)std::min<int64_t>(a.per, a.n - row0);
  const int tasks = rows * 2 * pg.kv_heads;
  const int lane = threadIdx.x % G, x = 8 * lane;
  const bool in = x < pg.d;
  const auto from = [&](int t) {
    const HeadRows& h = a.rows[t / pg.kv_heads % 2];
    return static_cast<T*>(h.p) + (row0 + t / (2 * pg.kv_heads)) * h.row + (int64_t)(t % pg.kv_heads) * h.head + x;
  };
  const auto fetch = [&](int t) {
    Chunk<T> c;
    const u32x4* p = reinterpret_cast<const u32x4*>(from(t));
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) c.w[i] = p[i];
    return c;
  };
  int t = threadIdx.x / G;
  Chunk<T> next = {};
  if (!READ && t < tasks && in) next = fetch(t);

  const bool staged = pg.n_docs <= kStaged;
  if (staged) {
    for (int i = threadIdx.x; i < pg.n_docs; i += kThreads) first[i] = a.start[i];
    __syncthreads();
  }
  if ((int)threadIdx.x < rows) {
    const int64_t row = row0 + threadIdx.x;
    const int doc = staged ? document_of([&](int i) { return first[i]; }, pg.n_docs, row)
                           : document_of([&](int i) { return a.start[i]; }, pg.n_docs, row);
    int page = -1, at = -1;
    if (doc >= 0) {
      const int64_t begin = a.start[doc], end = a.start[doc + 1];
      const int64_t place = READ ? row - begin : a.len[doc] - end + row;
      if (row < end) {
        at = 0;
        if (place >= 0 && place < (int64_t)pg.table_row << pg.shift) {
          at = (int)place;
          page = pg.table[(int64_t)doc * pg.table_row + (place >> pg.shift)];
        }
      }
    }
    page_of[threadIdx.x] = page;
    place_of[threadIdx.x] = at;
  }
  __syncthreads();

  for (; t < tasks; t += kGroups) {
    const Chunk<T> c = next;
    if (!READ && t + kGroups < tasks && in) next = fetch(t + kGroups);
    const int r = t / (2 * pg.kv_heads), values = t / pg.kv_heads % 2, head = t % pg.kv_heads;
    const int place = place_of[r];
    const int64_t at = place < 0 ? -1 : page_row(pg, page_of[r], place, head);
    char* const kept = static_cast<char*>(values ? pg.v : pg.k) + (at * pg.d + x) * (BITS8 ? 1 : (int64_t)sizeof(T));
    float* const scale_at = BITS8 ? (values ? pg.v_scale : pg.k_scale) + at : nullptr;
    if constexpr (READ) {
      if (place < 0 || !in) continue;
      T* const to = from(t);
      Chunk<T> got = {};
      if (at >= 0) {
        if constexpr (BITS8) {
          const u32x2 q = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(kept));
          const float scale = *scale_at;
          float v[8];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], true);
            v[4 * i] = lo[0] * scale, v[4 * i + 1] = lo[1] * scale;
            v[4 * i + 2] = hi[0] * scale, v[4 * i + 3] = hi[1] * scale;
          }
          store8_past(to, v);
          continue;
        } else {
#pragma unroll
          for (int i = 0; i < (int)sizeof(T) / 2; ++i) got.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kept) + i);
        }
      }
      store_past(to, got);
    } else {
      if (at < 0) continue;  // of all lanes of the group
      if constexpr (BITS8) {
        float v[8] = {};
        float top = 0.0f;
        if (in) widen<T>(c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
#pragma unroll
        for (int m = 1; m < G; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
        const float scale = block_scale(top), by = 1.0f / scale;
        if (!in) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = quotient(v[i], scale, by);
        *reinterpret_cast<u32x2*>(kept) = u32x2{pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])};
        if (lane == 0) *scale_at = scale;
      } else if (in) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(kept)[i] = c.w[i];
      }
    }
  }
}

template <typename T, bool BITS8, bool READ>
hipError_t cache_t(CacheArgs a, hipStream_t s) {
  const auto launch = [&](auto kernel, int groups) {
    // about four rows of a head for each group, where there are enough of them
    const int64_t fill = std::max<int64_t>(1, a.n / 1024);
    a.per = (int)std::min<int64_t>({std::max(1, 4 * groups / (2 * a.pages.kv_heads)), fill, kMostRows});
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
