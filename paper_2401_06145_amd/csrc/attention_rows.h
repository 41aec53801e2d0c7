// Attention with few queries per document (one new token over a cache, above all).
#pragma once

#include "attention_device.h"

namespace spc {
namespace attn {

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

// Pages: a lane keeps the page of one of the tile's 32 keys, looked up a tile ahead, and gives it to
// the lanes that load that key's row.  8-bit rows: K comes 16 columns a lane (the product's columns
// may be in any order, as long as the queries' are in the same), V widened into the strip.  Bound by
// memory as packed keys are, 8 bits by the loads under way: one token for each of 48 documents of up to 8192
// keys, 32 heads of 128 on 8, 1.20 GB: 230 us (5.2 TB/s); in 8 bits, 0.62 GB, 144 us (4.3 TB/s, the join included); in float32,
// 2.40 GB, 520 us (4.6 TB/s; packed keys 435).
template <typename T, int D, int NC, int SRC>
__global__ __launch_bounds__(256, NC == 1 && D * sizeof(T) <= 256 ? 2 : 1) void k_attn_rows(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr int E = sizeof(T), ROW = lds_columns(D) * E, KT = 32;
  constexpr bool AHEAD = ROW < 1024;  // registers for the next tile while one is used
  typedef Lds<ROW> L;
  constexpr bool BITS8 = is_bits8(SRC);
  // Tiles on their way beside the one in use: two of 8 bits, which take half of the registers (one token for
  // each of 48 documents of up to 8192 keys, 32 heads of 128 on 8: 150 us with one).
  constexpr int DEPTH = BITS8 && NC == 1 && ROW <= 256 ? 2 : 1;
  typedef std::integral_constant<int, 0> Set0;
  typedef std::integral_constant<int, DEPTH - 1> Set1;
  constexpr int CB = BITS8 ? ROW / E / 16 : (int)L::CH;  // 16-byte chunks of a row of V in memory
  constexpr int P = (KT * CB + kWave - 1) / kWave;
  constexpr int STRIP = KT * ROW > D * 16 * 4 ? KT * ROW : D * 16 * 4;
  __shared__ __align__(16) char strips[4][STRIP];
  __shared__ f32x4 spos[4][KT];
  __shared__ float sm[4][16 * NC], sl[4][16 * NC];
  __shared__ f32x4 sscale[BITS8 ? 4 : 1][2][KT / 4];  // of the keys, and what of the values' the exponentials take

  // Workgroups go around the 8 XCDs: each document and head begins with another range, or some
  // XCDs would get the ranges that only long documents fill (8 ranges of 48 caches: 219 us, so 160).
  const int doc = blockIdx.z, kvh = blockIdx.y % a.kv_heads, col0 = blockIdx.y / a.kv_heads * 16 * NC;
  const int split = (blockIdx.x + doc + kvh) % a.splits;
  // Pages: the first ones are looked up beside the document's lengths, and may be none of its.
  const int k_begin = split * a.chunk, k_first = k_begin + (int)threadIdx.x / kWave * KT;
  const auto entry = [&](int place) {
    place += threadIdx.x % KT;
    if (place >= 0 && place >> a.shift < a.table_row) return a.table[(int64_t)doc * a.table_row + (place >> a.shift)];
    return -1;
  };
  [[maybe_unused]] int first_page = -1, second_page = -1;
  if constexpr (SRC != kPacked) {
    first_page = entry(k_first);
    if constexpr (DEPTH == 2) second_page = entry(k_first + 4 * KT);
  }
  const Doc d = load_doc<SRC>(a, doc);
  const int group = a.heads / a.kv_heads, cols = d.len_q * group;
  if (cols <= col0) return;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, c16 = lane % 16, g = lane / 16;
  char* sv = strips[wave];

  // the first of the eight columns that a lane has of a product's 32
  const auto col_of = [&](int k) { return BITS8 && (k | 1) < D / 32 ? 64 * (k / 2) + 16 * g + 8 * (k % 2) : 32 * k + 8 * g; };

  const int32_t* origin = SRC != kPacked ? nullptr : a.q_pos ? a.q_pos + 4 * (int64_t)d.q0 : nullptr;
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
      const int at = col_of(k);
      fq[n][k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int lim_lo = seen(a, d, 0), lim_hi = seen(a, d, d.len_q - 1);
  const int k_end = std::min(lim_hi, k_begin + a.chunk);

  f32x4 o[NC][D / 16];
  float m[NC], l[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = a.floor;
    l[n] = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[n][t] = f32x4{0, 0, 0, 0};
  }
  const T* kp = static_cast<const T*>(a.k);
  const T* vp = static_cast<const T*>(a.v);
  if constexpr (SRC == kPacked) kp += d.k0 * a.k_row + (int64_t)kvh * a.k_head, vp += d.k0 * a.v_row + (int64_t)kvh * a.v_head;
  // Pages: this head's part of the first one, and the way to the next.  A row's address is one product of
  // 32 bits and a sum.
  constexpr int B = BITS8 ? 1 : E;  // bytes of an element
  const uint32_t row_bytes = a.d * B, page_rows = (uint32_t)a.kv_heads << a.shift, page_bytes = page_rows * row_bytes;
  const int64_t head_rows = (int64_t)kvh << a.shift;
  const char *const kb = static_cast<const char*>(a.k) + head_rows * row_bytes, *const vb = static_cast<const char*>(a.v) + head_rows * row_bytes;
  const auto offset = [&](int page, int place) {
    return (uint64_t)(uint32_t)page * page_bytes + (uint32_t)((place & ((1 << a.shift) - 1)) * row_bytes);
  };

  // A tile's operands: K's rows as the product takes them (8 bits: as they lie), V's as they lie, the
  // voxels of the first KT lanes.  Their registers take the next tile as soon as they are used, so that
  // its loads are under way for the rest of the work on this one.
  Frag fk[2][BITS8 ? 1 : D / 32];
  u32x4 rk[DEPTH][2][BITS8 ? (D / 32 + 1) / 2 : 1];
  u32x4 rv[DEPTH][P];
  float scale[DEPTH] = {};  // of K's rows in the first KT lanes, of V's in the others
  int page = -1;       // of key lane % KT of the tile whose rows are loaded next
  int32_t pos[4] = {0, 0, 0, 0};
  const auto fetch_pages = [&](int k0) {
    if constexpr (SRC != kPacked) page = page_at(a, doc, d, k0 + lane % KT);
  };
  const auto checked = [&](int of, int k0) { return k0 + lane % KT < d.len_k && (uint32_t)of < (uint32_t)a.n_pages ? of : -1; };
  const auto fetch_k = [&](int k0, auto set) {
    constexpr int S = decltype(set)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 16 * h + c16, key = k0 + r;
      if constexpr (SRC == kPacked) {
        const T* p = kp + (int64_t)key * a.k_row;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          const int at = 32 * k + 8 * g;
          fk[h][k] = key < d.len_k && at < a.d ? load_frag(p + at) : zero_frag<T>();
        }
      } else {
        const int from = __shfl(page, r);
        const char* p = kb + offset(from, key);
        if constexpr (!BITS8) {
#pragma unroll
          for (int k = 0; k < D / 32; ++k) {
            const int at = 32 * k + 8 * g;
            fk[h][k] = from >= 0 && at < a.d ? load_frag(reinterpret_cast<const T*>(p) + at) : zero_frag<T>();
          }
        } else {
#pragma unroll
          for (int k = 0; k < (D / 32 + 1) / 2; ++k) {
            const int at = col_of(2 * k);
            rk[S][h][k] = u32x4{0, 0, 0, 0};
            if (from < 0 || at >= a.d) continue;
            if (2 * k + 1 < D / 32) {
              rk[S][h][k] = *reinterpret_cast<const u32x4*>(p + at);
            } else {
              const u32x2 w = *reinterpret_cast<const u32x2*>(p + at);
              rk[S][h][k] = u32x4{w[0], w[1], 0, 0};
            }
          }
        }
      }
    }
  };
  const auto fetch_v = [&](int k0, auto set) {
    constexpr int S = decltype(set)::value;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lane + kWave * i, r = p / CB, c = p % CB;
      rv[S][i] = u32x4{0, 0, 0, 0};
      if constexpr (SRC == kPacked) {
        if (k0 + r < d.len_k && c * (16 / E) < a.d)
          rv[S][i] = *reinterpret_cast<const u32x4*>(vp + (int64_t)(k0 + r) * a.v_row + c * (16 / E));
      } else {
        const int from = __shfl(page, r % KT);
        if (r < KT && from >= 0 && c * (16 / B) < a.d) rv[S][i] = *reinterpret_cast<const u32x4*>(vb + offset(from, k0 + r) + 16 * c);
      }
    }
    if constexpr (BITS8) {
      scale[S] = 0.0f;
      if (page >= 0)
        scale[S] = ((lane < KT ? a.k_scale : a.v_scale) + head_rows)[(uint64_t)(uint32_t)page * page_rows + ((k0 + lane % KT) & ((1 << a.shift) - 1))];
    }
    if (SRC == kPacked && a.k_pos && lane < KT && k0 + lane < d.len_k) {
#pragma unroll
      for (int i = 1; i < 4; ++i) pos[i] = a.k_pos[4 * (d.k0 + k0 + lane) + i];
    }
  };
  if constexpr (SRC != kPacked) page = checked(first_page, k_first);
  if (AHEAD && k_first < k_end) {
    fetch_v(k_first, Set0());
    fetch_k(k_first, Set0());
    if constexpr (DEPTH == 2) {
      page = checked(second_page, k_first + 4 * KT);
      if (k_first + 4 * KT < k_end) {
        fetch_v(k_first + 4 * KT, Set1());
        fetch_k(k_first + 4 * KT, Set1());
      }
    }
    fetch_pages(k_first + 4 * DEPTH * KT);
  }
  const auto tile = [&](int k0, auto set) {
    constexpr int S = decltype(set)::value;
    const bool masked = k0 + KT > lim_lo;
    if (!AHEAD) fetch_v(k0, set);
    bool bad = false;
    if (masked && !BITS8) {
#pragma unroll
      for (int i = 0; i < P; ++i) bad |= odd_values<T>(rv[S][i]);
    }
    if (SRC == kPacked && a.k_pos && lane < KT) {  // keys that do not exist are hidden, wherever they are
      const Voxel v = voxel_from(pos, origin);
      spos[wave][lane] = f32x4{v.x, v.y, v.z, 0};
    }
    if constexpr (!BITS8) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int p = lane + kWave * i, r = p / CB, c = p % CB;
        *reinterpret_cast<u32x4*>(sv + r * ROW + 16 * L::v_chunk16(r, c)) = rv[S][i];
      }
    } else {
      const Scale mine = split_scale<T>(scale[S]);
      reinterpret_cast<float*>(sscale[wave])[lane] = lane < KT ? scale[S] : mine.rest;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int p = lane + kWave * i, r = p / CB, c = p % CB;
        const float power = __shfl(mine.power, KT + r % KT);
        const uint32_t nan = __shfl((int)mine.nan, KT + r % KT);
        if (r >= KT) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const Frag f = from_e4m3<T>(rv[S][i][2 * j] | nan, rv[S][i][2 * j + 1] | nan, power);
#pragma unroll
          for (int m = 0; m < E / 2; ++m) {
            u32x4 w;
            __builtin_memcpy(&w, reinterpret_cast<const char*>(&f) + 16 * m, 16);
            if (masked) bad |= odd_values<T>(w);
            *reinterpret_cast<u32x4*>(sv + r * ROW + 16 * L::v_chunk16(r, c * E + (E / 2) * j + m)) = w;
          }
        }
      }
    }
    const int next = k0 + 4 * DEPTH * KT;
    const bool more = AHEAD && next < k_end;
    if (!AHEAD) fetch_k(k0, set);
    if (more) fetch_v(next, set);
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
        for (int k = 0; k < D / 32; ++k) {
          if constexpr (BITS8) s[n][h] = Mat<T>::mma16(from_e4m3<T>(rk[S][h][k / 2][2 * (k % 2)], rk[S][h][k / 2][2 * (k % 2) + 1], 1.0f), fq[n][k], s[n][h]);
          else s[n][h] = Mat<T>::mma16(fk[h][k], fq[n][k], s[n][h]);
        }
      }
    if (more) {
      fetch_k(next, set);
      fetch_pages(next + 4 * KT);
    } else if (!AHEAD) {
      fetch_pages(k0 + 4 * KT);
    }
    Frag fp[NC];  // rounded to the rows' type (attention.hip has why, and what it costs in the result)
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = s[n][i / 4][i % 4] * (BITS8 ? sscale[wave][0][4 * (i / 4) + g][i % 4] : 1.0f);
      const auto at = [&](int i) { return 16 * (i / 4) + 4 * g + i % 4; };
      const auto key = [&](int i) { return k0 + at(i); };
      if (a.cap > 0.0f) cap_scores<8, E == 4>(a, sc);
      if (SRC == kPacked && a.k_pos) {
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
      float off = fmaf(m[n], a.exp_by, -kExpRaise<T, BITS8>);
      const bool large = fabsf(off) > kMostOffset;
      if (__any(large)) {  // (of this row: others keep their bits)
        const float first = large ? m[n] : 0.0f;
        off = large ? -kExpRaise<T, BITS8> : off;
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] -= first;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.exp_by, -off));
        l[n] += sc[i];
        if constexpr (BITS8) sc[i] *= sscale[wave][1][4 * (i / 4) + g][i % 4];
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
  };
  for (int k0 = k_first; k0 < k_end; k0 += 4 * DEPTH * KT) {
    tile(k0, Set0());
    if (DEPTH == 2 && k0 + 4 * KT < k_end) tile(k0 + 4 * KT, Set1());
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

template <typename T, int SRC>
hipError_t rows_t(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
#define SPC_D(D, NC)                                                                                                \
  hipLaunchKernelGGL((k_attn_rows<T, D, NC, SRC>),                                                                  \
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

template <int SRC>
hipError_t launch_rows(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  if (dtype == 0) return rows_t<float, SRC>(a, p, s);
  if (dtype == 1) return rows_t<_Float16, SRC>(a, p, s);
  return rows_t<__bf16, SRC>(a, p, s);
}

}  // namespace attn
}  // namespace spc
