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
#include <algorithm>
#include <type_traits>

#include "attention.h"
#include "rows.h"

namespace spc {
namespace {

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
__device__ __forceinline__ float odd_value(int kind) { return kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY; }

// Rows of a K or V tile in LDS, in 16-byte chunks that are exchanged inside a row so that the
// lanes of one access meet different banks: K is read as one chunk of 16 (32) rows, V as 64
// (32) bytes of 4 (16) rows.
template <int ROW_BYTES>
struct Lds {
  static constexpr int CH = ROW_BYTES / 16;                                // chunks of a row
  static constexpr int R = ROW_BYTES >= 256 ? 1 : 256 / ROW_BYTES;         // rows in 256 bytes
  __device__ static int k_chunk(int row, int c) { return c ^ (row / R & (CH < 16 ? CH - 1 : 15)); }
  __device__ static int v_chunk(int row, int c) { return c ^ ((row / R & (CH < 16 ? CH / 4 - 1 : 3)) << 2); }
  __device__ static int v_chunk16(int row, int c) { return c ^ ((row / R & (CH < 16 ? CH / 2 - 1 : 7)) << 1); }
};

// Four consecutive rows' elements of one column for every lane of a group of 16: lane i gives
// the address of four columns of row i / 4, and gets column i of the four rows.
__device__ __forceinline__ i16x4 read_columns(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4*)(__attribute__((address_space(3))) const void*)p);
}

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

// Turns 'count' products q.k of one query into the scores that the running maximum is taken
// of; key(i) is the document's key of product i.  Without cap and bias the scores stay the
// bare products (their scale is folded into the exponential's), else they are in units of
// log2.  Hidden keys get -inf.
struct Query {
  float place, slope;  // place among the keys; slope in units of log2
  float x, y, z;       // voxel
  int lim;             // keys seen
};
template <int COUNT, typename Key, typename Pos>
__device__ __forceinline__ void to_scores(const AttnArgs& a, const Query& q, float* s, bool masked, Key key, Pos pos) {
  if (a.cap > 0.0f) {
    // tanh(u) = 1 - 2 / (1 + e^{2u}): exact limits at both ends, absolute error 2^-23
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const float e = __builtin_amdgcn_exp2f(s[i] * a.tanh_by);
      s[i] = fmaf(-2.0f * a.cap_log2, __builtin_amdgcn_rcpf(1.0f + e), a.cap_log2);
    }
  } else if (a.slopes) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] *= a.scale_log2;
  }
  if (a.slopes) {
    if (a.k_pos) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i) {
        const f32x4 p = pos(i);
        const float dx = p[0] - q.x, dy = p[1] - q.y, dz = p[2] - q.z;
        s[i] = fmaf(-q.slope, __builtin_amdgcn_sqrtf(fmaf(dx, dx, fmaf(dy, dy, dz * dz))), s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; ++i) s[i] = fmaf(-q.slope, fabsf(q.place - (float)key(i)), s[i]);
    }
  }
  if (masked) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i] = key(i) < q.lim ? s[i] : -INFINITY;
  }
}

__device__ __forceinline__ Query make_query(const AttnArgs& a, const Doc& d, int i, int head) {
  Query q;
  q.lim = seen(a, d, i);
  q.place = (float)(d.len_k - d.len_q + i);
  q.slope = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  q.x = q.y = q.z = 0.0f;
  if (a.q_pos) {
    const int32_t* p = a.q_pos + 4 * (int64_t)(d.q0 + i);
    q.x = (float)p[1], q.y = (float)p[2], q.z = (float)p[3];
  }
  return q;
}

// Four consecutive values of a row of the output, or of its partial result.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  else *reinterpret_cast<u32x2*>(p) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
}

// ---------------------------------------------------------------------------
// Many queries: a workgroup of four waves takes 128 NQ queries of one head and one range of
// keys, 64 keys at a time through LDS; each wave has 32 NQ of the queries.
// ---------------------------------------------------------------------------
constexpr int kTileKeys = 64;

template <typename T, int D, int NQ>
__global__ __launch_bounds__(256) void k_attn_tile(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr int QT = 128 * NQ, E = sizeof(T), ROW = D * E;
  typedef Lds<ROW> L;
  constexpr int P = kTileKeys * L::CH / 256;  // chunks of K (and of V) a thread stages
  __shared__ __align__(16) char sk[kTileKeys * ROW], sv[kTileKeys * ROW];
  __shared__ f32x4 spos[kTileKeys];

  int first;
  const int doc = find_doc(a, blockIdx.x, QT, &first);
  const Doc d = load_doc(a, doc);
  const int i0 = (blockIdx.x - first) * QT;
  if (i0 >= d.len_q) return;
  const int head = blockIdx.y, kvh = head / (a.heads / a.kv_heads);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, c32 = lane % 32, half = lane / 32;

  // the rows of this wave, and what they see
  Query q[NQ];
  int row[NQ];
  Frag fq[NQ][D / 16];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    row[n] = i0 + (wave * NQ + n) * 32 + c32;
    const int i = std::min(row[n], d.len_q - 1);
    q[n] = make_query(a, d, i, head);
    const T* p = static_cast<const T*>(a.q) + (int64_t)(d.q0 + i) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int at = 16 * k + 8 * half;
      fq[n][k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int wave_i0 = std::min(i0 + wave * NQ * 32, d.len_q - 1);
  const int lim_lo = seen(a, d, wave_i0), lim_hi = seen(a, d, std::min(wave_i0 + NQ * 32 - 1, d.len_q - 1));
  const int tile_lo = seen(a, d, i0), tile_hi = seen(a, d, std::min(i0 + QT, d.len_q) - 1);
  const int k_begin = blockIdx.z * a.chunk, k_end = std::min(tile_hi, k_begin + a.chunk);

  f32x16 o[NQ][D / 32];
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = a.floor;
    l[n] = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][t][i] = 0.0f;
  }
  const T* kp = static_cast<const T*>(a.k) + d.k0 * a.k_row + (int64_t)kvh * a.k_head;
  const T* vp = static_cast<const T*>(a.v) + d.k0 * a.v_row + (int64_t)kvh * a.v_head;

  for (int k0 = k_begin; k0 < k_end; k0 += kTileKeys) {
    u32x4 rk[P], rv[P];
    bool bad = false;
    const bool tile_masked = k0 + kTileKeys > tile_lo;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = threadIdx.x + 256 * i, r = p / L::CH, c = p % L::CH;
      rk[i] = rv[i] = u32x4{0, 0, 0, 0};
      if (k0 + r < d.len_k && c * (16 / E) < a.d) {
        rk[i] = *reinterpret_cast<const u32x4*>(kp + (int64_t)(k0 + r) * a.k_row + c * (16 / E));
        rv[i] = *reinterpret_cast<const u32x4*>(vp + (int64_t)(k0 + r) * a.v_row + c * (16 / E));
      }
      if (tile_masked) bad |= odd_values<T>(rv[i]);
    }
    f32x4 pos = {0, 0, 0, 0};
    if (a.k_pos && threadIdx.x < kTileKeys && k0 + (int)threadIdx.x < d.len_k) {
      const int32_t* p = a.k_pos + 4 * (d.k0 + k0 + threadIdx.x);
      pos = f32x4{(float)p[1], (float)p[2], (float)p[3], 0};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = threadIdx.x + 256 * i, r = p / L::CH, c = p % L::CH;
      *reinterpret_cast<u32x4*>(sk + r * ROW + 16 * L::k_chunk(r, c)) = rk[i];
      *reinterpret_cast<u32x4*>(sv + r * ROW + 16 * L::v_chunk(r, c)) = rv[i];
    }
    if (threadIdx.x < kTileKeys) spos[threadIdx.x] = pos;
    // a hidden key's value is multiplied by 0, which must not make an infinity or a NaN of
    // it part of the sum: such tiles take the careful form below
    const bool careful = __syncthreads_or(tile_masked && bad);
    if (k0 >= lim_hi) continue;  // nothing for this wave

    f32x16 s[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][h][i] = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 32 * h + c32;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        Frag f;
        if constexpr (E == 4) {
          const int c = 4 * k + 2 * half;
          const f32x4 x = *reinterpret_cast<const f32x4*>(sk + r * ROW + 16 * L::k_chunk(r, c));
          const f32x4 y = *reinterpret_cast<const f32x4*>(sk + r * ROW + 16 * L::k_chunk(r, c + 1));
          f = f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        } else {
          f = *reinterpret_cast<const Frag*>(sk + r * ROW + 16 * L::k_chunk(r, 2 * k + half));
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][h] = Mat<T>::mma32(f, fq[n][k], s[n][h]);
      }
    }
    const bool masked = k0 + kTileKeys > lim_lo;
    Frag fp[NQ][4];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float* sc = reinterpret_cast<float*>(s[n]);
      const auto at = [&](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * half + i % 4; };
      to_scores<32>(a, q[n], sc, masked, [&](int i) { return k0 + at(i); }, [&](int i) { return spos[at(i)]; });
      float top = m[n];
#pragma unroll
      for (int i = 0; i < 32; ++i) top = fmaxf(top, sc[i]);
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m[n])) {
        const float by = __builtin_amdgcn_exp2f((m[n] - top) * a.exp_by);
        l[n] *= by;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[n][t][i] *= by;
        m[n] = top;
      }
      const float off = m[n] * a.exp_by;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.exp_by, -off));
        sum += sc[i];
      }
      l[n] += sum;
#pragma unroll
      for (int c = 0; c < 4; ++c) fp[n][c] = to_frag<T>(sc + 8 * c);
    }
    // columns of V: fragment (t, c) of out^T's rows 32 t .. and keys 16 c + {4 half + j, 8 + 4 half + j}
    const auto columns = [&](int t, int c) {
      Frag f;
      if constexpr (E == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = 16 * c + 8 * (j / 4) + 4 * half + j % 4, x = 32 * t + c32;
          f[j] = *reinterpret_cast<const float*>(sv + r * ROW + 16 * L::v_chunk(r, x / 4) + 4 * (x % 4));
        }
      } else {
        const int i = lane % 16, x = 32 * t + 16 * (lane / 16 % 2) + 4 * (i % 4);
        i16x4 w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = 16 * c + 8 * j + 4 * half + i / 4;
          w[j] = read_columns(sv + r * ROW + 16 * L::v_chunk(r, x / 8) + 2 * (x % 8));
        }
        f = __builtin_bit_cast(Frag, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
      return f;
    };
    if (!(careful && masked)) {
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const Frag f = columns(t, c);
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[n][t] = Mat<T>::mma32(f, fp[n][c], o[n][t]);
        }
    } else {
      // the finite values, then whatever infinities and NaN the seen keys have
#pragma unroll
      for (int t = 0; t < D / 32; ++t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const Frag f = finite_only<T>(columns(t, c));
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[n][t] = Mat<T>::mma32(f, fp[n][c], o[n][t]);
        }
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind)
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            f32x16 hit;
#pragma unroll
            for (int i = 0; i < 16; ++i) hit[i] = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float v[8];
#pragma unroll
              for (int j = 0; j < 8; ++j)
                v[j] = k0 + 16 * c + 8 * (j / 4) + 4 * half + j % 4 < q[n].lim ? 1.0f : 0.0f;
              hit = Mat<T>::mma32(odd_ones<T>(columns(t, c), kind), to_frag<T>(v), hit);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) o[n][t][i] += hit[i] > 0.0f ? odd_value(kind) : 0.0f;
          }
      }
    }
  }

#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float sum = l[n] + __shfl_xor(l[n], 32);
    if (row[n] >= d.len_q) continue;
    const int64_t at = (int64_t)(d.q0 + row[n]) * a.heads + head;
    if (a.splits > 1) {
      const int64_t part = (int64_t)blockIdx.z * a.n_q * a.heads + at;
      if (half == 0) a.part_ml[part] = f32x2{m[n], sum};
      if (sum != 0.0f) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const int x = 32 * t + 8 * (i / 4) + 4 * half;
            const float v[4] = {o[n][t][i], o[n][t][i + 1], o[n][t][i + 2], o[n][t][i + 3]};
            if (x < a.d) store4(a.part_o + part * a.d + x, v);
          }
      }
    } else {
      const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* out = static_cast<T*>(a.out) + (int64_t)(d.q0 + row[n]) * a.out_row + (int64_t)head * a.out_head;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int x = 32 * t + 8 * (i / 4) + 4 * half;
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = sum == 0.0f ? 0.0f : o[n][t][i + j] * by;
          if (x < a.d) store4(out + x, v);
        }
    }
  }
}

// ---------------------------------------------------------------------------
// Few queries: a workgroup takes the queries of all heads that share one key head (up to 16
// NC of them as columns) and one range of keys; its four waves go through the range 32 keys
// at a time, each on its own, and join their results through LDS at the end.  K comes from
// memory straight into registers, V through a strip of LDS that only its wave uses.
// ---------------------------------------------------------------------------
template <typename T, int D, int NC>
__global__ __launch_bounds__(256) void k_attn_rows(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr int E = sizeof(T), ROW = D * E, KT = 32;
  typedef Lds<ROW> L;
  constexpr int P = KT * L::CH / kWave;
  constexpr int STRIP = KT * ROW > D * 16 * 4 ? KT * ROW : D * 16 * 4;
  __shared__ __align__(16) char strips[4][STRIP];
  __shared__ f32x4 spos[4][KT];
  __shared__ float sm[4][16 * NC], sl[4][16 * NC];

  const int doc = blockIdx.z, kvh = blockIdx.y;
  const Doc d = load_doc(a, doc);
  const int group = a.heads / a.kv_heads, cols = d.len_q * group;
  if (cols <= 0) return;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, c16 = lane % 16, g = lane / 16;
  char* sv = strips[wave];

  Query q[NC];
  Frag fq[NC][D / 32];
  int64_t row[NC];  // row of the packed queries times heads, plus the head
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int col = std::min(16 * n + c16, cols - 1), i = col / group, head = kvh * group + col % group;
    row[n] = (int64_t)(d.q0 + i) * a.heads + head;
    q[n] = make_query(a, d, i, head);
    const T* p = static_cast<const T*>(a.q) + (int64_t)(d.q0 + i) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const int at = 32 * k + 8 * g;
      fq[n][k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int lim_lo = seen(a, d, 0), lim_hi = seen(a, d, d.len_q - 1);
  const int k_begin = blockIdx.x * a.chunk, k_end = std::min(lim_hi, k_begin + a.chunk);

  f32x4 o[NC][D / 16];
  float m[NC], l[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = a.floor;
    l[n] = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[n][t] = f32x4{0, 0, 0, 0};
  }
  const T* kp = static_cast<const T*>(a.k) + d.k0 * a.k_row + (int64_t)kvh * a.k_head;
  const T* vp = static_cast<const T*>(a.v) + d.k0 * a.v_row + (int64_t)kvh * a.v_head;

  for (int k0 = k_begin + wave * KT; k0 < k_end; k0 += 4 * KT) {
    const bool masked = k0 + KT > lim_lo;
    Frag fk[2][D / 32];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = k0 + 16 * h + c16;
      const T* p = kp + (int64_t)key * a.k_row;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const int at = 32 * k + 8 * g;
        fk[h][k] = key < d.len_k && at < a.d ? load_frag(p + at) : zero_frag<T>();
      }
    }
    bool bad = false;
    u32x4 rv[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + kWave * i, r = p / L::CH, c = p % L::CH;
      rv[i] = u32x4{0, 0, 0, 0};
      if (k0 + r < d.len_k && c * (16 / E) < a.d)
        rv[i] = *reinterpret_cast<const u32x4*>(vp + (int64_t)(k0 + r) * a.v_row + c * (16 / E));
      if (masked) bad |= odd_values<T>(rv[i]);
    }
    if (a.k_pos && lane < KT) {
      f32x4 pos = {0, 0, 0, 0};
      if (k0 + lane < d.len_k) {
        const int32_t* p = a.k_pos + 4 * (d.k0 + k0 + lane);
        pos = f32x4{(float)p[1], (float)p[2], (float)p[3], 0};
      }
      spos[wave][lane] = pos;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + kWave * i, r = p / L::CH, c = p % L::CH;
      *reinterpret_cast<u32x4*>(sv + r * ROW + 16 * L::v_chunk16(r, c)) = rv[i];
    }
    const bool careful = masked && __any(bad);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    Frag fp[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < D / 32; ++k) s[h] = Mat<T>::mma16(fk[h][k], fq[n][k], s[h]);
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = s[i / 4][i % 4];
      const auto at = [&](int i) { return 16 * (i / 4) + 4 * g + i % 4; };
      to_scores<8>(a, q[n], sc, masked, [&](int i) { return k0 + at(i); }, [&](int i) { return spos[wave][at(i)]; });
      float top = m[n];
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, sc[i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m[n])) {
        const float by = __builtin_amdgcn_exp2f((m[n] - top) * a.exp_by);
        l[n] *= by;
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][t][i] *= by;
        m[n] = top;
      }
      const float off = m[n] * a.exp_by;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.exp_by, -off));
        l[n] += sc[i];
      }
      fp[n] = to_frag<T>(sc);
    }
    // columns of V: rows 16 t .. of out^T and keys {4 g + j, 16 + 4 g + j}
    const auto columns = [&](int t) {
      Frag f;
      if constexpr (E == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = 16 * (j / 4) + 4 * g + j % 4, x = 16 * t + c16;
          f[j] = *reinterpret_cast<const float*>(sv + r * ROW + 16 * L::v_chunk16(r, x / 4) + 4 * (x % 4));
        }
      } else {
        const int x = 16 * t + 4 * (c16 % 4);
        i16x4 w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = 16 * j + 4 * g + c16 / 4;
          w[j] = read_columns(sv + r * ROW + 16 * L::v_chunk16(r, x / 8) + 2 * (x % 8));
        }
        f = __builtin_bit_cast(Frag, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
      return f;
    };
    if (!careful) {
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        const Frag f = columns(t);
#pragma unroll
        for (int n = 0; n < NC; ++n) o[n][t] = Mat<T>::mma16(f, fp[n], o[n][t]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        const Frag f = columns(t);
#pragma unroll
        for (int n = 0; n < NC; ++n) o[n][t] = Mat<T>::mma16(finite_only<T>(f), fp[n], o[n][t]);
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind)
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = k0 + 16 * (j / 4) + 4 * g + j % 4 < q[n].lim ? 1.0f : 0.0f;
            const f32x4 hit = Mat<T>::mma16(odd_ones<T>(f, kind), to_frag<T>(v), f32x4{0, 0, 0, 0});
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][t][i] += hit[i] > 0.0f ? odd_value(kind) : 0.0f;
          }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  // join of the four waves
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
    if (g == 0) sm[wave][16 * n + c16] = m[n], sl[wave][16 * n + c16] = l[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    float top = a.floor, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][16 * n + c16]);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      sum += sl[w][16 * n + c16] * __builtin_amdgcn_exp2f((sm[w][16 * n + c16] - top) * a.exp_by);
    const float by = __builtin_amdgcn_exp2f((m[n] - top) * a.exp_by);
    if (n) __syncthreads();
    f32x4* mine = reinterpret_cast<f32x4*>(sv);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      f32x4 v = o[n][t];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = l[n] == 0.0f ? 0.0f : v[i] * by;  // an unused wave adds nothing
      mine[t * kWave + lane] = v;
    }
    __syncthreads();
    if (16 * n + c16 < cols) {
      const int64_t part = (int64_t)blockIdx.x * a.n_q * a.heads + row[n];
      if (a.splits > 1 && wave == 0 && g == 0) a.part_ml[part] = f32x2{top, sum};
      const float inv = 1.0f / sum;
      for (int t = wave; t < D / 16; t += 4) {
        const int x = 16 * t + 4 * g;
        if (x >= a.d) continue;
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) v += reinterpret_cast<const f32x4*>(strips[w])[t * kWave + lane];
        if (a.splits > 1) {
          const float r[4] = {v[0], v[1], v[2], v[3]};
          if (sum != 0.0f) store4(a.part_o + part * a.d + x, r);
        } else {
          float r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = sum == 0.0f ? 0.0f : v[i] * inv;
          const int64_t i = row[n] / a.heads, head = row[n] % a.heads;
          store4(static_cast<T*>(a.out) + i * a.out_row + head * a.out_head + x, r);
        }
      }
    }
  }
}

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
hipError_t attention_t(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
  {
    ProfScope ps(KN_ATTENTION, s);
    if (p.rows) {
      const dim3 grid((unsigned)a.splits, (unsigned)a.kv_heads, (unsigned)a.n_docs);
#define SPC_D(DD, NC) hipLaunchKernelGGL((k_attn_rows<T, DD, NC>), grid, dim3(256), 0, s, a)
#define SPC_C(DD)                \
  if (p.cols <= 16) SPC_D(DD, 1); \
  else if (p.cols <= 32) SPC_D(DD, 2); \
  else SPC_D(DD, 4)
      if (a.d <= 32) { SPC_C(32); }
      else if (a.d <= 64) { SPC_C(64); }
      else if (a.d <= 128) { SPC_C(128); }
      else { SPC_C(256); }
#undef SPC_C
#undef SPC_D
    } else {
      const dim3 grid((unsigned)p.slots, (unsigned)a.heads, (unsigned)a.splits);
#define SPC_D(DD) hipLaunchKernelGGL((k_attn_tile<T, DD, 1>), grid, dim3(256), 0, s, a)
      if (a.d <= 32) SPC_D(32);
      else if (a.d <= 64) SPC_D(64);
      else if (a.d <= 128) SPC_D(128);
      else SPC_D(256);
#undef SPC_D
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.splits > 1) {
    ProfScope ps(KN_ATTENTION_JOIN, s);
    hipLaunchKernelGGL((k_attn_join<T>), dim3((unsigned)((a.n_q * a.heads + 3) / 4)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
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
  if (dtype == 0) return attention_t<float>(a, p, s);
  if (dtype == 1) return attention_t<_Float16>(a, p, s);
  return attention_t<__bf16>(a, p, s);
}

}  // namespace spc
