// Device code that both forms of the attention share.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attention.h"
#include "rows.h"

namespace spc {
namespace attn {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

// Matrix products on 8 consecutive elements a lane.  mma32: 32 x 32 over 16; lane l holds row
// (column) l % 32 and elements 8 (l / 32) + j.  mma16: 16 x 16 over 32, row l % 16, elements
// 8 (l / 16) + j.  float32 goes as eight products, the j-th over every lane's element j.
template <typename T>
struct Mat;
template <>
struct Mat<_Float16> {
  typedef f16x8 Frag;
  __device__ static f32x16 mma32(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  __device__ static f32x4 mma16(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mat<__bf16> {
  typedef bf16x8 Frag;
  __device__ static f32x16 mma32(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  __device__ static f32x4 mma16(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mat<float> {
  typedef f32x8 Frag;
  __device__ static f32x16 mma32(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  __device__ static f32x4 mma16(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// A fragment from 8 consecutive elements in memory (16-byte aligned).
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag load_frag(const T* p) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  } else {
    return *reinterpret_cast<const typename Mat<T>::Frag*>(p);
  }
}
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag zero_frag() {
  typename Mat<T>::Frag f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = (T)0.0f;
  return f;
}
// Eight float32 values as a fragment, rounded to nearest even.
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag to_frag(const float* v) {
  if constexpr (sizeof(T) == 4) {
    return f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  } else {
    return __builtin_bit_cast(typename Mat<T>::Frag, (u32x4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]),
                                                            pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])}));
  }
}

// Whether any of the elements in 16 bytes is an infinity or not a number.
template <typename T>
__device__ __forceinline__ bool odd_values(u32x4 w) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      bad |= (w[i] & 0x7f800000u) == 0x7f800000u;
    } else {
      constexpr uint32_t e = std::is_same_v<T, __bf16> ? 0x7f80u : 0x7c00u;
      bad |= (w[i] & e) == e || (w[i] & (e << 16)) == (e << 16);
    }
  }
  return bad;
}
// 1 where an element is NaN (kind 0), +inf (1) or -inf (2); and the value that it adds.
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag odd_ones(typename Mat<T>::Frag f, int kind) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = (float)f[j];
    const bool is = kind == 0 ? v != v : v == (kind == 1 ? INFINITY : -INFINITY);
    f[j] = (T)(is ? 1.0f : 0.0f);
  }
  return f;
}
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag finite_only(typename Mat<T>::Frag f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = (float)f[j];
    f[j] = fabsf(v) < INFINITY ? f[j] : (T)0.0f;
  }
  return f;
}
__device__ __forceinline__ int odd_kind(float v) { return v != v ? 0 : v == INFINITY ? 1 : v == -INFINITY ? 2 : -1; }
__device__ __forceinline__ float odd_value(int kind) { return kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY; }

// Columns that a row takes in LDS: a power of two.  Those of 96 that no product takes are left
// out of all else (23 documents of 77 queries and 2652 keys, 24 heads of 96: 144 us as 128 columns, 126 so).
constexpr int lds_columns(int d) { return d == 96 ? 128 : d; }

// Rows of a K or V tile in LDS, in 16-byte chunks that are exchanged inside a row so that the
// lanes of one access meet different banks: K is read as one chunk of 16 (32) rows, V as 64
// (32) bytes of 4 (16) rows.
template <int ROW_BYTES>
struct Lds {
  static constexpr uint32_t CH = ROW_BYTES / 16;                         // chunks of a row
  static constexpr uint32_t R = ROW_BYTES >= 256 ? 1 : 256 / ROW_BYTES;  // rows in 256 bytes
  __device__ static uint32_t k_chunk(uint32_t row, uint32_t c) { return c ^ (row / R & (CH < 16 ? CH - 1 : 15)); }
  __device__ static uint32_t v_chunk(uint32_t row, uint32_t c) { return c ^ ((row / R & (CH < 16 ? CH / 4 - 1 : 3)) << 2); }
  __device__ static uint32_t v_chunk16(uint32_t row, uint32_t c) { return c ^ ((row / R & (CH < 16 ? CH / 2 - 1 : 7)) << 1); }
};

// Four consecutive rows' elements of one column for every lane of a group of 16: lane i gives
// the address of four columns of row i / 4, and gets column i of the four rows.
__device__ __forceinline__ i16x4 read_columns(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4*)(__attribute__((address_space(3))) const void*)p);
}

// Exponentials are taken as 2^15 and less instead of 1 and less for float16 rows: rounded for the
// product with V, those below 2^-25 of the largest would vanish from the sum of values, but
// not from the sum of exponentials (131,072 keys at 2^-25.5 beside a dominant one hold 0.3 % of a
// row).  The factor is part of both sums and leaves with their quotient.
template <typename T>
constexpr float kExpRaise = std::is_same_v<T, _Float16> ? 15.0f : 0.0f;

// A document's part of the batch.
struct Doc {
  int q0, len_q;
  int64_t k0;
  int len_k, prefix;
};
__device__ __forceinline__ Doc load_doc(const AttnArgs& a, int doc) {
  Doc d;
  d.q0 = std::max(a.q_start[doc], 0);
  d.len_q = std::min((int)std::min<int64_t>(a.q_start[doc + 1], a.n_q) - d.q0, a.max_q);
  d.k0 = std::max(a.k_start[doc], 0);
  const int64_t len = a.k_len ? a.k_len[doc] : a.k_start[doc + 1] - d.k0;
  d.len_k = (int)std::max<int64_t>(0, std::min<int64_t>(std::min<int64_t>(len, a.max_k), a.n_k - d.k0));
  d.prefix = a.prefix ? a.prefix[doc] : 0;
  return d;
}
// Number of keys that query i sees: the first ones of its document.
__device__ __forceinline__ int seen(const AttnArgs& a, const Doc& d, int i) {
  if (!a.causal) return d.len_k;
  return std::min(std::max(std::max(d.len_k - d.len_q + i + 1, d.prefix), 0), d.len_k);
}

// The largest document whose first slot is at most `slot`; slots of document t start at
// q_start[t] / tile + t, so each has room for its tiles and no running sum is needed.
__device__ __forceinline__ int find_doc(const AttnArgs& a, int slot, int tile, int* first) {
  const int lane = threadIdx.x % kWave;
  int lo = 0, n = a.n_docs;
  while (true) {
    const int step = (n + kWave - 1) / kWave, at = lane * step;
    const bool ok = at < n && a.q_start[lo + at] / tile + lo + at <= slot;
    const int c = std::max(popc64(__ballot(ok)) - 1, 0);
    lo += c * step;
    n = std::min(step, n - c * step);
    if (step == 1) break;
  }
  *first = a.q_start[lo] / tile + lo;
  return lo;
}

// Scores of one query, as the running maximum is taken of them: capped ones are in units of
// log2, the others in those of the products q.k (exp_by folds their scale into the
// exponential's).  key(i) is the document's key of product i; hidden keys get -inf.
struct Query {
  int place;           // among the keys
  float slope;         // in the scores' units
  float x, y, z;       // voxel
  int lim;             // keys seen
};

// cap tanh(u), u = scale s / cap, in units of log2.  Where every product of the wave is small
// (most are, as caps are meant for the few large ones) as s times a polynomial of u^2, whose error
// goes by the score and not by the cap (api.hip, set_cap): of degree 3 in u, 7, and 9 for float32
// rows (FINE); else as tanh(u) = 1 - 2 / (1 + e^{2u}), with its exact limits, within 1.2e-7 of
// the cap: a few of float32's steps, as such scores are at least a fifth of it.  3 or 6
// instructions instead of 3 and two transcendental ones, which take twice as long (whole
// documents, cap 50, before their maximum was kept: 855 us, 767 with degree 7, 719 to 735 with 3).
// Which one runs goes by the values: 4096 rows of 8 heads of 128 in bfloat16 take 77 us where all
// scores are within 0.11 of the cap, and 93 beyond.
template <bool FINE>
__device__ __forceinline__ float cap_factor(const AttnArgs& a, float s) {
  const float u = s * a.cap_by, z = u * u;
  const float top = FINE ? fmaf(z, a.poly[4], a.poly[3]) : a.poly[3];
  return fmaf(fmaf(fmaf(z, top, a.poly[2]), z, a.poly[1]), z, a.poly[0]);
}
__device__ __forceinline__ float cap_exactly(const AttnArgs& a, float s, float from) {
  const float e = __builtin_amdgcn_exp2f(s * a.tanh_by);
  return fmaf(-2.0f * a.cap_log2, __builtin_amdgcn_rcpf(1.0f + e), from);
}
template <int COUNT, bool FINE>
__device__ __forceinline__ void cap_scores(const AttnArgs& a, float* s) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) most = fmaxf(most, fabsf(s[i]));
  if (!FINE && !__any(most > a.low_most)) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] *= fmaf(s[i] * s[i], a.low[1], a.low[0]);
  } else if (!__any(most > a.poly_most)) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] *= cap_factor<FINE>(a, s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] = cap_exactly(a, s[i], a.cap_log2);
  }
}
// Capped scores less m, with what the caller knows of the wave's products: low, that none is beyond
// low_most, and `most`, the largest magnitude of the lane's.
template <int COUNT, bool FINE>
__device__ __forceinline__ void cap_scores_less(const AttnArgs& a, float* s, bool low, float most, float m) {
  if (!FINE && low) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] = fmaf(s[i], fmaf(s[i] * s[i], a.low[1], a.low[0]), -m);
  } else if (!__any(most > a.poly_most)) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] = fmaf(s[i], cap_factor<FINE>(a, s[i]), -m);
  } else {
    const float from = a.cap_log2 - m;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] = cap_exactly(a, s[i], from);
  }
}

// A voxel from its row (b, x, y, z), seen from `origin` (another such row): small numbers
// wherever the scene lies, exact in float32 up to 2^24 from it.
struct Voxel {
  float x, y, z;
};
__device__ __forceinline__ Voxel voxel_from(const int32_t* p, const int32_t* origin) {
  return Voxel{(float)((int64_t)p[1] - origin[1]), (float)((int64_t)p[2] - origin[2]), (float)((int64_t)p[3] - origin[3])};
}

template <int COUNT, typename Pos>
__device__ __forceinline__ void add_voxel_bias(const Query& q, float* s, Pos pos) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    const Voxel p = pos(i);
    const float dx = p.x - q.x, dy = p.y - q.y, dz = p.z - q.z;
    s[i] = fmaf(-q.slope, __builtin_amdgcn_sqrtf(fmaf(dx, dx, fmaf(dy, dy, dz * dz))), s[i]);
  }
}
// The difference of whole numbers: places from 2^24 on are not all float32 numbers, near distances are.
template <int COUNT, typename Key>
__device__ __forceinline__ void add_place_bias(const Query& q, float* s, Key key) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) s[i] = fmaf(-q.slope, fabsf((float)(q.place - key(i))), s[i]);
}
template <int COUNT, typename Key>
__device__ __forceinline__ void hide(const Query& q, float* s, Key key) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) s[i] = key(i) < q.lim ? s[i] : -INFINITY;
}

// `origin`: the row that voxels are seen from, or NULL where there are none.
__device__ __forceinline__ Query make_query(const AttnArgs& a, const Doc& d, int i, int head, const int32_t* origin) {
  Query q;
  q.lim = seen(a, d, i);
  q.place = d.len_k - d.len_q + i;
  q.slope = 0.0f;
  if (a.slopes) {  // a finite one stays finite in the scores' units: infinity times the distance 0 is not a number
    const float given = a.slopes[head], there = given * a.slope_by;
    q.slope = fabsf(given) < INFINITY ? fminf(fmaxf(there, -3e38f), 3e38f) : there;
  }
  q.x = q.y = q.z = 0.0f;
  if (origin) {
    const Voxel v = voxel_from(a.q_pos + 4 * (int64_t)(d.q0 + i), origin);
    q.x = v.x, q.y = v.y, q.z = v.z;
  }
  return q;
}

// Four consecutive values of a row of the output, or of its partial result.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  else *reinterpret_cast<u32x2*>(p) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
}

}  // namespace attn
}  // namespace spc
