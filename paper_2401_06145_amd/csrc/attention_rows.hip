// Attention with few queries per document (one new token over a cache, above all).
#include "attention_device.h"

namespace spc {
namespace {
using namespace attn;

// ---------------------------------------------------------------------------
// Few queries: a workgroup takes the queries of all heads that share one key head (up to 16
// NC of them as columns) and one range of keys; its four waves go through the range 32 keys
// at a time, each on its own, and join their results through LDS at the end.  K comes from
// memory straight into registers, V through a strip of LDS that only its wave uses.
// ---------------------------------------------------------------------------
//
// What bounds it: memory.  48 caches of up to 8192 keys (8 key heads of 128, 16 bits, 801 MB) take
// 155 to 160 us, 5.0 TB/s, what a large copy reaches; two workgroups a CU keep enough loads under
// way (one: 183 us), except for rows of more than 256 bytes, whose registers would spill.
// 32 and 64 columns a workgroup only where their sums fit its registers, else more workgroups
// for a key head's columns (two documents of 49, 8 heads of 96, float32: 9.5 us, with 64 columns a
// workgroup 42.8; a document of 11, two heads a key head of 256, bfloat16 9.2, with 32 22.7).
constexpr int most_columns(int row) { return row <= 128 ? 64 : row <= 256 ? 32 : 16; }

template <typename T, int D, int NC>
__global__ __launch_bounds__(256, NC == 1 && D * sizeof(T) <= 256 ? 2 : 1) void k_attn_rows(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr int E = sizeof(T), ROW = lds_columns(D) * E, KT = 32;
  constexpr bool AHEAD = ROW < 1024;  // registers for the next tile while one is used
  typedef Lds<ROW> L;
  constexpr int P = KT * (int)L::CH / kWave;
  constexpr int STRIP = KT * ROW > D * 16 * 4 ? KT * ROW : D * 16 * 4;
  __shared__ __align__(16) char strips[4][STRIP];
  __shared__ f32x4 spos[4][KT];
  __shared__ float sm[4][16 * NC], sl[4][16 * NC];

  // Workgroups go around the 8 XCDs: each document and head begins with another range, or some
  // XCDs would get the ranges that only long documents fill (8 ranges of 48 caches: 219 us, so 160).
  const int doc = blockIdx.z, kvh = blockIdx.y % a.kv_heads, col0 = blockIdx.y / a.kv_heads * 16 * NC;
  const int split = (blockIdx.x + doc + kvh) % a.splits;
  const Doc d = load_doc(a, doc);
  const int group = a.heads / a.kv_heads, cols = d.len_q * group;
  if (cols <= col0) return;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, c16 = lane % 16, g = lane / 16;
  char* sv = strips[wave];

  const int32_t* origin = a.q_pos ? a.q_pos + 4 * (int64_t)d.q0 : nullptr;
  Query q[NC];
  Frag fq[NC][D / 32];
  int64_t row[NC];  // row of the packed queries times heads, plus the head
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int col = std::min(col0 + 16 * n + c16, cols - 1), i = col / group, head = kvh * group + col % group;
    row[n] = (int64_t)(d.q0 + i) * a.heads + head;
    q[n] = make_query(a, d, i, head, origin);
    const T* p = static_cast<const T*>(a.q) + (int64_t)(d.q0 + i) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const int at = 32 * k + 8 * g;
      fq[n][k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int lim_lo = seen(a, d, 0), lim_hi = seen(a, d, d.len_q - 1);
  const int k_begin = split * a.chunk, k_end = std::min(lim_hi, k_begin + a.chunk);

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

  // A tile's operands: K's rows as the product takes them, V's as they lie, the voxels of the
  // first KT lanes.  Their registers take the next tile as soon as they are used, so that its
  // loads are under way for the rest of the work on this one.
  Frag fk[2][D / 32];
  u32x4 rv[P];
  int32_t pos[4] = {0, 0, 0, 0};
  const auto fetch_k = [&](int k0) {
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
  };
  const auto fetch_v = [&](int k0) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + kWave * i, r = p / (int)L::CH, c = p % (int)L::CH;
      rv[i] = u32x4{0, 0, 0, 0};
      if (k0 + r < d.len_k && c * (16 / E) < a.d)
        rv[i] = *reinterpret_cast<const u32x4*>(vp + (int64_t)(k0 + r) * a.v_row + c * (16 / E));
    }
    if (a.k_pos && lane < KT && k0 + lane < d.len_k) {
#pragma unroll
      for (int i = 1; i < 4; ++i) pos[i] = a.k_pos[4 * (d.k0 + k0 + lane) + i];
    }
  };
  const int k_first = k_begin + wave * KT;
  if (AHEAD && k_first < k_end) {
    fetch_v(k_first);
    fetch_k(k_first);
  }
  for (int k0 = k_first; k0 < k_end; k0 += 4 * KT) {
    const bool masked = k0 + KT > lim_lo;
    if (!AHEAD) fetch_v(k0);
    bool bad = false;
    if (masked) {
#pragma unroll
      for (int i = 0; i < P; ++i) bad |= odd_values<T>(rv[i]);
    }
    if (a.k_pos && lane < KT) {  // keys that do not exist are hidden, wherever they are
      const Voxel v = voxel_from(pos, origin);
      spos[wave][lane] = f32x4{v.x, v.y, v.z, 0};
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + kWave * i, r = p / (int)L::CH, c = p % (int)L::CH;
      *reinterpret_cast<u32x4*>(sv + r * ROW + 16 * L::v_chunk16(r, c)) = rv[i];
    }
    const bool more = AHEAD && k0 + 4 * KT < k_end;
    if (!AHEAD) fetch_k(k0);
    if (more) fetch_v(k0 + 4 * KT);
    const bool careful = masked && __any(bad);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    f32x4 s[NC][2];
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[n][h] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < D / 32; ++k) s[n][h] = Mat<T>::mma16(fk[h][k], fq[n][k], s[n][h]);
      }
    if (more) fetch_k(k0 + 4 * KT);
    Frag fp[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = s[n][i / 4][i % 4];
      const auto at = [&](int i) { return 16 * (i / 4) + 4 * g + i % 4; };
      const auto key = [&](int i) { return k0 + at(i); };
      if (a.cap > 0.0f) cap_scores<8, E == 4>(a, sc);
      if (a.k_pos) {
        add_voxel_bias<8>(q[n], sc, [&](int i) {
          const f32x4 p = spos[wave][at(i)];
          return Voxel{p[0], p[1], p[2]};
        });
      } else if (a.slopes) {
        add_place_bias<8>(q[n], sc, key);
      }
      if (masked) hide<8>(q[n], sc, key);
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
      const float off = fmaf(m[n], a.exp_by, -kExpRaise<T>);
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
    if (col0 + 16 * n + c16 < cols) {
      const int64_t part = (int64_t)split * a.n_q * a.heads + row[n];
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

template <typename T>
hipError_t rows_t(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
#define SPC_D(D, NC)                                                                                                \
  hipLaunchKernelGGL((k_attn_rows<T, D, NC>),                                                                       \
                     dim3((unsigned)a.splits, (unsigned)(a.kv_heads * ((p.cols + 16 * NC - 1) / (16 * NC))), \
                        (unsigned)a.n_docs), dim3(256), 0, s, a)
#define SPC_C(D)                                                                      \
  do {                                                                                \
    constexpr int most = most_columns(lds_columns(D) * (int)sizeof(T));               \
    if (most == 16 || p.cols <= 16) SPC_D(D, 1);                                      \
    else if (most == 32 || p.cols <= 32) SPC_D(D, (most < 32 ? 1 : 2));               \
    else SPC_D(D, (most < 64 ? 1 : 4));                                               \
  } while (0)
  if (a.d <= 32) SPC_C(32);
  else if (a.d <= 64) SPC_C(64);
  else if (a.d <= 96) SPC_C(96);
  else if (a.d <= 128) SPC_C(128);
  else SPC_C(256);
#undef SPC_C
#undef SPC_D
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_rows(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  if (dtype == 0) return rows_t<float>(a, p, s);
  if (dtype == 1) return rows_t<_Float16>(a, p, s);
  return rows_t<__bf16>(a, p, s);
}

}  // namespace spc
