// Attention with many queries per document: whole prompts and scenes.
#include "attention_device.h"

namespace spc {
namespace {
using namespace attn;

// What the scores go through.  kBare: nothing but their scale.  kCapped: a cap of at most 60
// and no bias, in types of float32's exponents: a row whose scores are all within 0.11 of the cap
// takes that bound for their maximum (exponentials of e^-13.2 at least), so that most tiles need
// not look for it (whole documents 717 us; 4096 rows of 8 heads of 128 77 us, 93 with scores
// beyond the bound, 83 and 92 by kAny, as measured in float16).  kVoxel: a bias by the
// distance of voxels, with or without a cap.  kAny: everything else.
enum Mode { kBare, kCapped, kVoxel, kAny };
constexpr float kMostBoundedCap = 60.0f;

// 16 bytes a lane from memory straight into LDS, P times: those at `at[i]` of the `bytes` that
// begin at `from` (zeros where they end before, and at kNowhere) to the wave's 1024 bytes at
// `to` + 4096 i.
// Written as assembly because of the waits: of the builtin's loads the compiler awaits the
// tile under way before it reads the tile that is there.  The caller waits (vmcnt) itself.
constexpr uint32_t kNowhere = 0xfffffff0u;  // behind every buffer: 16 bytes from here on still have 32-bit offsets
template <int P>
__device__ __forceinline__ void bring_rows(const char* from, uint32_t bytes, char* to, const uint32_t* at) {
  const uint64_t base = reinterpret_cast<uint64_t>(from);
  const u32x4 rsrc = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)base),
                      (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xffffu),
                      (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)to;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    uint32_t kept;  // M0 holds the LDS address
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(kept)
        : "s"(__builtin_amdgcn_readfirstlane(lds + 4096 * i)), "v"(at[i]), "s"(rsrc)
        : "memory");
  }
}

// Workgroups a CU holds, by the registers that rows of this many bytes need.
constexpr int waves_a_simd(int row, int mode) {
  return row <= 64 ? (mode == kVoxel ? 3 : 4) : row <= 128 ? (mode == kVoxel ? 2 : 3) : row <= 256 ? 2 : 1;
}

// Distances of voxels by the matrix unit: |k - q|^2 = |q|^2 - 2 k.q + |k|^2 is a product of five
// columns, float32, two instructions for 32 x 32 distances instead of six a distance (voxels of two
// frames 214 -> 199 us).  It must not lose small distances in the difference of large
// squares: it is taken where every sum is a whole number of float32, that is where the voxels
// of a tile, as multiples of 2^shift that the queries have in common, are at most 1182 apart
// from the origin in each axis (3 1182^2 < 2^22, and four such squares still fit 2^24).
constexpr int kVoxelReach = 1182;
struct Near {
  int shift;
  __device__ bool operator()(const int32_t* p, const int32_t* origin) const {
    uint32_t all = 0;
    int64_t most = 0;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const int64_t v = (int64_t)p[i] - origin[i];
      all |= (uint32_t)v;
      most = std::max(most, v < 0 ? -v : v);
    }
    return (all & ((1u << shift) - 1)) == 0 && most <= (int64_t)kVoxelReach << shift;
  }
};

// A workgroup of four waves takes 128 queries of one head and one range of keys, KT or 2 KT
// keys at a time through LDS; each wave has 32 of the queries.  The next tile of K and V is on its way
// from memory straight into the other half of LDS while one is multiplied.
//
// What bounds it: the vector and the matrix unit, busy for 52 and 44 % of the cycles (documents of
// up to 8192, 16 heads of 128, capped: 711 to 775 us by the machine, 0.9 to 0.96 PFLOP/s); with voxels
// and short rows the vector unit, 62 %: a root, an exponential and eight more instructions a
// score and head (160 us).
//
// Workgroups with the same key head are neighbours in time on one XCD (workgroups go around
// the 8 XCDs), so that its L2 serves K and V; the longest rows (the last of a document,
// where the call is causal) start first.
template <typename T, int D, int MODE>
__global__ __launch_bounds__(256, waves_a_simd(lds_columns(D) * sizeof(T), MODE)) void k_attn_tile(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr int QT = kQueryTile, E = sizeof(T), ROW = lds_columns(D) * E;
  constexpr int KT = ROW >= 1024 ? 32 : 64;
  // Rows of 256 bytes leave registers for operands ahead of their use: all of a tile of K before
  // the first product, a strip of V while the exponentials are computed (784 -> 770 us on whole
  // documents of 128 columns; with distances, or 2 strips, the registers spill; shorter
  // rows gain nothing).
  constexpr bool AHEAD = ROW == 256 && MODE < kVoxel;
  constexpr int VA = AHEAD ? 1 : 0;
  typedef Lds<ROW> L;
  // Keys between two barriers: two tiles for short rows with voxels, whose coordinates one or two
  // waves prepare while the others wait (two frames, 8 heads of 32: 169 us, so 159; of 64
  // 125, so 119; without voxels it is even, and longer rows would lose a workgroup a CU).
  constexpr int KB = MODE == kVoxel && ROW <= 128 ? 2 * KT : KT;
  constexpr int P = KB * (int)L::CH / 256;  // chunks of K (and of V) a thread brings
  __shared__ __align__(16) char sk[2][KB * ROW], sv[2][KB * ROW];
  __shared__ f32x4 spos[2][KB];       // voxels of the keys: x, z, y, x^2 + y^2 + z^2
  __shared__ uint32_t snear[2][KB / KT], sbits[4];  // whether they all are near; bits of the waves' queries' voxels
  __shared__ uint32_t odd_at[3 * KB * (D / 32)];  // NaN, +inf and -inf of a tile's values, a bit each

  // which slot, head and range of keys
  const int per = a.heads * a.slots, split = blockIdx.x / per, in = blockIdx.x - split * per;
  const int h = in % a.heads, head = a.heads % 8 == 0 ? h % 8 * (a.heads / 8) + h / 8 : h;
  const int slot = a.slots - 1 - in / a.heads;
  int first;
  const int doc = find_doc(a, slot, QT, &first);
  const Doc d = load_doc(a, doc);
  const int i0 = (slot - first) * QT;
  if (i0 < 0 || i0 >= d.len_q) return;  // slots before the first document's are nobody's
  const int kvh = head / (a.heads / a.kv_heads);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x % kWave, c32 = lane % 32, half = lane / 32;

  // the rows of this wave, and what they see
  const int row = i0 + wave * 32 + c32;
  const int32_t* origin = MODE == kVoxel ? a.q_pos + 4 * (int64_t)(d.q0 + i0) : nullptr;
  const Query q = make_query(a, d, std::min(row, d.len_q - 1), head, origin);
  Frag fq[D / 16];
  {
    const T* p = static_cast<const T*>(a.q) + (int64_t)(d.q0 + std::min(row, d.len_q - 1)) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int at = 16 * k + 8 * half;
      fq[k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int wave_i0 = std::min(i0 + wave * 32, d.len_q - 1);
  const int lim_lo = seen(a, d, wave_i0), lim_hi = seen(a, d, std::min(wave_i0 + 31, d.len_q - 1));
  const int tile_lo = seen(a, d, i0), tile_hi = seen(a, d, std::min(i0 + QT, d.len_q) - 1);
  const int k_begin = split * a.chunk, k_end = std::min(tile_hi, k_begin + a.chunk);

  f32x16 o[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
  float m = MODE == kCapped ? -a.cap_log2 : a.floor, l = 0.0f;
  float m_of = -INFINITY;  // kCapped: the product whose score m is,
  bool bounded = false;    // and whether it is low_most at least in all of the wave's rows

  // A thread's chunks of a tile: 16 bytes that lie in LDS where the wave's lanes follow each
  // other, and in memory where the exchanged order puts them.  Columns that do not exist lie
  // out of the buffer's range, which gives zeros, as do rows behind the last key.
  const char* kp = static_cast<const char*>(a.k) + (d.k0 * a.k_row + (int64_t)kvh * a.k_head) * E;
  const char* vp = static_cast<const char*>(a.v) + (d.k0 * a.v_row + (int64_t)kvh * a.v_head) * E;
  const uint32_t k_bytes = (uint32_t)a.k_row * E, v_bytes = (uint32_t)a.v_row * E;
  static_assert((KB - 1) * (uint64_t)kMostRowBytes + 256 * 4 <= kNowhere, "a tile's rows have offsets of 32 bits, unsigned");
  uint32_t at_k[P], at_v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t p = (4 * i + wave) * kWave + lane, r = p / L::CH, c = p % L::CH;
    const int ck = L::k_chunk(r, c), cv = L::v_chunk(r, c);
    at_k[i] = ck * (16 / E) < a.d ? r * k_bytes + 16 * ck : kNowhere;
    at_v[i] = cv * (16 / E) < a.d ? r * v_bytes + 16 * cv : kNowhere;
  }
  const auto bring = [&](int k0, int b) {
    const uint32_t rows = std::min(d.len_k - k0, KB);
    bring_rows<P>(kp + (int64_t)k0 * k_bytes, (rows - 1) * k_bytes + a.d * E, sk[b] + 1024 * wave, at_k);
    bring_rows<P>(vp + (int64_t)k0 * v_bytes, (rows - 1) * v_bytes + a.d * E, sv[b] + 1024 * wave, at_v);
  };
  // the first KT threads, one wave: a key's voxel each
  Near near = {0};
  bool near_q = false;
  if constexpr (MODE == kVoxel) {
    const int32_t* p = a.q_pos + 4 * (int64_t)(d.q0 + std::min(row, d.len_q - 1));
    const uint32_t bits = ((uint32_t)p[1] - (uint32_t)origin[1]) | ((uint32_t)p[2] - (uint32_t)origin[2]) |
                          ((uint32_t)p[3] - (uint32_t)origin[3]);
    uint32_t all = 1u << 4;  // 16 is the spacing of the coarsest level
#pragma unroll
    for (int i = 0; i < 4; ++i) all |= __any(bits >> i & 1) ? 1u << i : 0;
    if (lane == 0) sbits[wave] = all;
    __syncthreads();
    near.shift = __builtin_ctz(sbits[0] | sbits[1] | sbits[2] | sbits[3]);
    near_q = __all(near(p, origin));
  }
  // Loaded beside a tile, looked at when the tile before is done: looked at at once, all of the
  // tile's loads were awaited (voxels of two frames 177 us, so 170).
  int32_t voxel[4] = {0, 0, 0, 0};
  int voxels = 0;
  const auto fetch_voxel = [&](int k0) {
    voxels = MODE == kVoxel ? d.len_k - k0 : 0;
    if ((int)threadIdx.x < std::min(KB, voxels)) {
#pragma unroll
      for (int i = 1; i < 4; ++i) voxel[i] = a.k_pos[4 * (d.k0 + k0 + threadIdx.x) + i];
    }
  };
  const auto keep_voxel = [&](int b) {
    static_assert(KT == 64 || MODE != kVoxel || KB == KT, "a wave looks at one tile");
    if (MODE == kVoxel && (int)threadIdx.x < (KB + 63) / 64 * 64) {
      bool ok = true;
      if ((int)threadIdx.x < KB) {
        f32x4 at = {0, 0, 0, 0};
        if ((int)threadIdx.x < voxels) {
          const Voxel v = voxel_from(voxel, origin);
          at = f32x4{v.x, v.z, v.y, fmaf(v.x, v.x, fmaf(v.y, v.y, v.z * v.z))};
          ok = near(voxel, origin);
        }
        spos[b][threadIdx.x] = at;
      }
      ok = __all(ok);
      if (lane == 0) snear[b][wave] = ok;
    }
  };
  // this lane's part of the second operand of the distances, and |q|^2
  const float vq0 = -2.0f * (half ? q.y : q.x), vq1 = half ? 1.0f : -2.0f * q.z;
  const float vq2 = fmaf(q.x, q.x, fmaf(q.y, q.y, q.z * q.z));

  if (k_begin < k_end) {
    bring(k_begin, 0);
    fetch_voxel(k_begin);
    keep_voxel(0);
  }
  int b = 0;
  const int last = std::min(lim_hi, k_end);  // behind it there is nothing for this wave
  for (int kb = k_begin; kb < k_end; kb += KB, b ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of the tile is in LDS
    __syncthreads();                     // and so are the others'; the other half is free
    // A hidden key's value is multiplied by 0, which must not make an infinity or a NaN of it
    // part of the sum.  Where a tile with hidden keys has such values they leave the tile, and
    // go to the queries that see them after the product.
    bool odd = false;
    if (kb + KB > tile_lo) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        odd |= odd_values<T>(*reinterpret_cast<const u32x4*>(sv[b] + 16 * (threadIdx.x + 256 * i)));
      odd = __syncthreads_or(odd);
      if (odd) {
        for (int i = threadIdx.x; i < 3 * KB * (D / 32); i += 256) odd_at[i] = 0;
        __syncthreads();
        for (uint32_t p = threadIdx.x; p < KB * L::CH; p += 256) {
          const int r = p / L::CH, x = L::v_chunk(r, p % L::CH) * (16 / E);
          for (int j = 0; j < 16 / E; ++j) {
            T* v = reinterpret_cast<T*>(sv[b] + 16 * p) + j;
            const int kind = odd_kind((float)*v);
            if (kind < 0) continue;
            atomicOr(&odd_at[(kind * KB + r) * (D / 32) + (x + j) / 32], 1u << ((x + j) % 32));
            *v = (T)0.0f;
          }
        }
        __syncthreads();
      }
    }
    if (kb + KB < k_end) {
      bring(kb + KB, b ^ 1);
      fetch_voxel(kb + KB);
    }
#pragma unroll 1
    for (int k0 = kb; k0 < std::min(kb + KB, last); k0 += KT) {
      const int sub = (k0 - kb) / KT;
      const char *const tk = sk[b] + sub * KT * ROW, *const tv = sv[b] + sub * KT * ROW;
      float s[KT / 2];
      {
        f32x16 acc[KT / 32];
#pragma unroll
        for (int h = 0; h < KT / 32; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[h][i] = 0.0f;
        const auto key_rows = [&](int h, int k) {
          const int r = 32 * h + c32;
          if constexpr (E == 4) {
            const int c = 4 * k + 2 * half;
            const f32x4 x = *reinterpret_cast<const f32x4*>(tk + r * ROW + 16 * L::k_chunk(r, c));
            const f32x4 y = *reinterpret_cast<const f32x4*>(tk + r * ROW + 16 * L::k_chunk(r, c + 1));
            return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
          } else {
            return *reinterpret_cast<const Frag*>(tk + r * ROW + 16 * L::k_chunk(r, 2 * k + half));
          }
        };
        if constexpr (AHEAD) {
          Frag f[KT / 32][D / 16];
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int h = 0; h < KT / 32; ++h) f[h][k] = key_rows(h, k);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int h = 0; h < KT / 32; ++h) acc[h] = Mat<T>::mma32(f[h][k], fq[k], acc[h]);
        } else {
#pragma unroll
          for (int h = 0; h < KT / 32; ++h)
#pragma unroll
            for (int k = 0; k < D / 16; ++k) acc[h] = Mat<T>::mma32(key_rows(h, k), fq[k], acc[h]);
        }
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) s[i] = acc[i / 16][i % 16];
      }
      // columns of V: fragment (t, c) of out^T's rows 32 t .. and keys 16 c + {4 half + j, 8 + 4 half + j}
      const auto columns = [&](int t, int c) {
        Frag f;
        if constexpr (E == 4) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int r = 16 * c + 8 * (j / 4) + 4 * half + j % 4, x = 32 * t + c32;
            f[j] = *reinterpret_cast<const float*>(tv + r * ROW + 16 * L::v_chunk(r, x / 4) + 4 * (x % 4));
          }
        } else {
          const int i = lane % 16, x = 32 * t + 16 * (lane / 16 % 2) + 4 * (i % 4);
          i16x4 w[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = 16 * c + 8 * j + 4 * half + i / 4;
            w[j] = read_columns(tv + r * ROW + 16 * L::v_chunk(r, x / 8) + 2 * (x % 8));
          }
          f = __builtin_bit_cast(Frag, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return f;
      };
      Frag fv[D / 32][VA + 1];
      if constexpr (VA > 0) {
#pragma unroll
        for (int c = 0; c < VA; ++c)
#pragma unroll
          for (int t = 0; t < D / 32; ++t) fv[t][c] = columns(t, c);
        __builtin_amdgcn_sched_barrier(0);
      }

      const bool masked = k0 + KT > lim_lo;
      const auto at = [&](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * half + i % 4; };
      const auto key = [&](int i) { return k0 + at(i); };
      if constexpr (MODE == kCapped) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) most = fmaxf(most, fabsf(s[i]));
        const bool low = !__any(most > a.low_most);
        if (!low || !bounded) {
          // The largest product that is seen, or the bound where all of them lie within.  (Products
          // grow with scores, and are compared without computing the latter.)
          float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          if (masked) {
#pragma unroll
            for (int i = 0; i < KT / 2; ++i) t[i % 4] = fmaxf(t[i % 4], key(i) < q.lim ? s[i] : -INFINITY);
          } else {
            t[0] = most <= a.low_most ? a.low_most : -INFINITY;
#pragma unroll
            for (int i = 0; i < KT / 2; ++i) t[i % 4] = fmaxf(t[i % 4], s[i]);
          }
          const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
          if (__any(top > m_of)) {
            m_of = fmaxf(fmaxf(m_of, top), __shfl_xor(top, 32));
            bounded = !__any(m_of < a.low_most);
            const float to = cap_exactly(a, m_of, a.cap_log2), by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[t][i] *= by;
            m = to;
          }
        }
        cap_scores_less<KT / 2, E == 4>(a, s, low, most, m);
        if (masked) hide<KT / 2>(q, s, key);
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) s[i] = __builtin_amdgcn_exp2f(s[i]);
      } else {
        if (MODE != kBare && a.cap > 0.0f) cap_scores<KT / 2, E == 4>(a, s);
        if constexpr (MODE == kVoxel) {
          if (near_q && snear[b][sub]) {
#pragma unroll
            for (int h = 0; h < KT / 32; ++h) {
              const f32x2 k = *reinterpret_cast<const f32x2*>(reinterpret_cast<const char*>(&spos[b][sub * KT + 32 * h + c32]) + 8 * half);
              f32x16 far;
#pragma unroll
              for (int i = 0; i < 16; ++i) far[i] = vq2;
              far = __builtin_amdgcn_mfma_f32_32x32x2f32(k[0], vq0, far, 0, 0, 0);
              far = __builtin_amdgcn_mfma_f32_32x32x2f32(k[1], vq1, far, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 16; ++i) s[16 * h + i] = fmaf(-q.slope, __builtin_amdgcn_sqrtf(far[i]), s[16 * h + i]);
            }
          } else {
            add_voxel_bias<KT / 2>(q, s, [&](int i) {
              const f32x4 p = spos[b][sub * KT + at(i)];
              return Voxel{p[0], p[2], p[1]};
            });
          }
        } else if (MODE == kAny && a.slopes) {
          add_place_bias<KT / 2>(q, s, key);
        }
        if (masked) hide<KT / 2>(q, s, key);
        float top = m;
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) {
          const float by = __builtin_amdgcn_exp2f((m - top) * a.exp_by);
          l *= by;
#pragma unroll
          for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= by;
          m = top;
        }
        const float off = fmaf(m, a.exp_by, -kExpRaise<T>);
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.exp_by, -off));
      }
      {
        float sum[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i < KT / 2; ++i) sum[i % 4] += s[i];
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      Frag fp[KT / 16];
#pragma unroll
      for (int c = 0; c < KT / 16; ++c) fp[c] = to_frag<T>(s + 8 * c);
      // all exponentials before the products: 712 -> 702 us where nothing else stands between them
      // (other modes lose 1 to 6 %)
      if constexpr (AHEAD && MODE == kCapped) __builtin_amdgcn_sched_barrier(0);

#pragma unroll
      for (int c = 0; c < KT / 16; ++c)
#pragma unroll
        for (int t = 0; t < D / 32; ++t) {
          o[t] = Mat<T>::mma32(c < VA ? fv[t][c < VA ? c : 0] : columns(t, c), fp[c], o[t]);
        }
      if (odd) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll 1
          for (int kr = 0; kr < 3 * KT; ++kr) {
            const uint32_t bits = odd_at[(kr / KT * KB + sub * KT + kr % KT) * (D / 32) + t];
            if (bits == 0 || k0 + kr % KT >= q.lim) continue;
            const float v = odd_value(kr / KT);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] += bits >> (8 * (i / 4) + 4 * half + i % 4) & 1 ? v : 0.0f;
          }
      }
    }
    if (kb + KB < k_end) keep_voxel(b ^ 1);
  }

  const float sum = l + __shfl_xor(l, 32);
  if (row >= d.len_q) return;
  const int64_t out_at = (int64_t)(d.q0 + row) * a.heads + head;
  if (a.splits > 1) {
    const int64_t part = (int64_t)split * a.n_q * a.heads + out_at;
    if (half == 0) a.part_ml[part] = f32x2{m, sum};
    if (sum == 0.0f) return;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int x = 32 * t + 8 * (i / 4) + 4 * half;
        const float v[4] = {o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
        if (x < a.d) store4(a.part_o + part * a.d + x, v);
      }
  } else {
    const float by = 1.0f / sum;
    T* out = static_cast<T*>(a.out) + (int64_t)(d.q0 + row) * a.out_row + (int64_t)head * a.out_head;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int x = 32 * t + 8 * (i / 4) + 4 * half;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = sum == 0.0f ? 0.0f : o[t][i + j] * by;
        if (x < a.d) store4(out + x, v);
      }
  }
}

template <typename T, int MODE>
void tile_mode(const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.heads * a.slots * a.splits));
#define SPC_D(D) hipLaunchKernelGGL((k_attn_tile<T, D, MODE>), grid, dim3(256), 0, s, a)
  if (a.d <= 32) SPC_D(32);
  else if (a.d <= 64) SPC_D(64);
  else if (a.d <= 96) SPC_D(96);
  else if (a.d <= 128) SPC_D(128);
  else SPC_D(256);
#undef SPC_D
}

template <typename T>
void tile_t(const AttnArgs& a, hipStream_t s) {
  if (a.cap == 0.0f && !a.slopes) return tile_mode<T, kBare>(a, s);
  if (a.k_pos) return tile_mode<T, kVoxel>(a, s);
  if constexpr (!std::is_same_v<T, _Float16>) {
    if (!a.slopes && a.cap <= kMostBoundedCap) return tile_mode<T, kCapped>(a, s);
  }
  tile_mode<T, kAny>(a, s);
}

}  // namespace

hipError_t launch_attention_tile(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  if (!fits_launch((int64_t)a.heads * p.slots * p.splits, 256)) return hipErrorInvalidConfiguration;
  if (dtype == 0) tile_t<float>(a, s);
  else if (dtype == 1) tile_t<_Float16>(a, s);
  else tile_t<__bf16>(a, s);
  return hipGetLastError();
}

}  // namespace spc
