// Attention with many queries per document: whole prompts and scenes, and chunks of new tokens.
#pragma once

#include "attention_device.h"

namespace spc {
namespace attn {

// What the scores go through.  kBare: nothing but their scale.  kCapped: a cap of at most 60
// and no bias, in types of float32's exponents: a row whose scores are all within 0.11 of the cap
// takes that bound for their maximum (exponentials of e^-13.2 at least), so that most tiles need
// not look for it (whole documents 717 us; 4096 rows of 8 heads of 128 77 us, 93 with scores
// beyond the bound, 83 and 92 by kAny, as measured in float16).  kVoxel: a bias by the
// distance of voxels, with or without a cap.  kPlace (pages): a bias by place and no cap; in tiles before
// or behind the wave's queries it is a line in the key's place, two instructions a score fewer than the
// distance (3 x 512 float16 queries of 12,001 keys, 16 heads of 64: 141 us, so 125).  kAny: everything else.
enum Mode { kBare, kCapped, kVoxel, kPlace, kAny };
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

// The same 16 bytes a lane from an address of its own, and from one that the wave shares plus an offset.
__device__ __forceinline__ void bring_from(const char* from, char* to) {
  uint32_t kept;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(kept)
      : "s"(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)to)), "v"(from)
      : "memory");
}
__device__ __forceinline__ void bring_from(const char* from, uint32_t at, char* to) {
  uint32_t kept;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(kept)
      : "s"(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)to)), "v"(at), "s"(from)
      : "memory");
}
// What rows that do not exist are brought from: 16 bytes for each lane of a wave.
__device__ __align__(16) const uint32_t kZeros[4 * kWave] = {};

// Workgroups a CU holds, by the registers that rows of this many bytes need.
constexpr int waves_a_simd(int row, int mode, int src, int e) {
  if (src != kPacked && e == 4 && row == 512) return 2;
  if (is_bits8(src)) return row <= 64 ? 3 : row <= 256 ? 2 : 1;
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
//
// Pages: a tile's rows are the queries of all heads of a key head, next to each other.  A wave's load covers rows_of_load rows.  Pages of that many rows or more (a power of two, as all
// are) hold them together: the page's number is looked up a tile ahead and the rows' address is the
// wave's, by scalar instructions.  Smaller ones (kSmall): each lane looks up the page of its row and
// computes its address (4 x 1024 queries of 16,384 keys, 32 heads of 128: pages of 64 to 4 rows 1169 to 1226 us, of
// 2 and 1, which go so, 1605 and 1712; in 8 bits of 64 and 8 1392 and 1407, of 4 to 1 1606 to 1701).
// 8 bits: rows come into registers, and are widened into the other half of LDS when the tile is
// done, once for all waves.  4 x 1024 queries of 16,384 keys, 32 heads of 128 on 8, bfloat16: packed keys
// 1085 to 1134 us, pages 1134 to 1177 (0.94 PFLOP/s), 8 bits 1360 to 1400 (0.78): two products a score, its scales from
// LDS and the widening are 53 % more vector instructions, and the waves wait for LDS.  Capped at 30: 1354, 1435, 1635.
constexpr int rows_of_load(int d, int e, bool bits8) {
  const int chunks = lds_columns(d) * (bits8 ? 1 : e) / 16;  // of a row
  return chunks >= kWave ? 1 : kWave / chunks;
}
template <typename T, int D, int MODE, int SRC>
__global__ __launch_bounds__(256, waves_a_simd(lds_columns(D) * sizeof(T), MODE, SRC, sizeof(T))) void k_attn_tile(AttnArgs a) {
  typedef typename Mat<T>::Frag Frag;
  constexpr bool BITS8 = is_bits8(SRC), EVEN = SRC == kPages || SRC == kPages8;
  constexpr int QT = kQueryTile, E = sizeof(T), ROW = lds_columns(D) * E;
  constexpr int KT = ROW >= 1024 || (SRC != kPacked && E == 4 && ROW == 512) ? 32 : 64;
  // Rows of 256 bytes leave registers for operands ahead of their use: all of a tile of K before
  // the first product, a strip of V while the exponentials are computed (784 -> 770 us on whole
  // documents of 128 columns; with distances, or 2 strips, the registers spill; shorter
  // rows gain nothing).
  constexpr bool AHEAD = ROW == 256 && MODE < kVoxel && !BITS8;
  constexpr int VA = AHEAD ? 1 : 0;
  typedef Lds<ROW> L;
  // Keys between two barriers: two tiles for short rows with voxels, whose coordinates one or two
  // waves prepare while the others wait (two frames, 8 heads of 32: 169 us, so 159; of 64
  // 125, so 119; without voxels it is even, and longer rows would lose a workgroup a CU).
  constexpr int KB = MODE == kVoxel && ROW <= 128 ? 2 * KT : KT;
  constexpr int P = KB * (int)L::CH / 256;  // chunks of K (and of V) a thread brings
  constexpr int CB = BITS8 ? ROW / E / 16 : (int)L::CH;  // 16-byte chunks of a row in memory
  constexpr int PB = (KB * CB + 255) / 256;              // and of them a thread's
  __shared__ __align__(16) char sk[2][KB * ROW], sv[2][KB * ROW];
  __shared__ f32x4 spos[2][KB];       // voxels of the keys: x, z, y, x^2 + y^2 + z^2
  __shared__ uint32_t snear[2][KB / KT], sbits[4];  // whether they all are near; bits of the waves' queries' voxels
  __shared__ f32x4 sscale[2][BITS8 ? 2 : 1][KB / 4];  // of the keys, and what of the values' the exponentials take
  __shared__ uint32_t odd_at[3 * KB * (D / 32)];  // NaN, +inf and -inf of a tile's values, a bit each

  // which slot, head and range of keys
  const int units = SRC == kPacked ? a.heads : a.kv_heads;
  const int per = units * a.slots, split = blockIdx.x / per, in = blockIdx.x - split * per;
  const int h = in % units, unit = units % 8 == 0 ? h % 8 * (units / 8) + h / 8 : h;
  const int slot = a.slots - 1 - in / units;
  // rows of the tiles: a document's queries, or (pages) theirs of all heads of a key head, next to each other
  const int group = SRC == kPacked ? 1 : a.heads / a.kv_heads;
  int doc, first;
  if (SRC != kPacked && a.doc_slots) doc = slot / a.doc_slots, first = doc * a.doc_slots;
  else doc = find_doc(a, slot, QT, group, &first);
  const Doc d = load_doc<SRC>(a, doc);
  const int i0 = (slot - first) * QT, rows = d.len_q * group;
  if (i0 < 0 || i0 >= rows) return;  // slots before the first document's are nobody's
  const int kvh = SRC == kPacked ? unit / (a.heads / a.kv_heads) : unit;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x % kWave, c32 = lane % 32, half = lane / 32;

  // the rows of this wave, and what they see
  const int row = i0 + wave * 32 + c32;
  const int query = std::min(row, rows - 1) / group, head = SRC == kPacked ? unit : kvh * group + std::min(row, rows - 1) % group;
  const int32_t* origin = MODE == kVoxel ? a.q_pos + 4 * (int64_t)(d.q0 + i0) : nullptr;
  const Query q = make_query(a, d, query, head, origin);
  Frag fq[D / 16];
  {
    const T* p = static_cast<const T*>(a.q) + (int64_t)(d.q0 + query) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int at = 16 * k + 8 * half;
      fq[k] = at < a.d ? load_frag(p + at) : zero_frag<T>();
    }
  }
  const int wave_i0 = std::min(i0 + wave * 32, rows - 1);
  const int lim_lo = seen(a, d, wave_i0 / group);
  // (pages: a wave without rows multiplies nothing)
  const int lim_hi = SRC != kPacked && i0 + wave * 32 >= rows ? 0 : seen(a, d, std::min(wave_i0 + 31, rows - 1) / group);
  const int tile_lo = seen(a, d, i0 / group), tile_hi = seen(a, d, (std::min(i0 + QT, rows) - 1) / group);
  const int k_begin = split * a.chunk, k_end = std::min(tile_hi, k_begin + a.chunk);

  // kPlace: the least place of the wave's queries, and whether 2^31 places keep every slope's bias finite
  [[maybe_unused]] const int wave_place = d.len_k - d.len_q + wave_i0 / group;
  [[maybe_unused]] const bool even_slopes = MODE == kPlace && !__any(!(fabsf(q.slope) < 1e28f));

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
  const char *kp = static_cast<const char*>(a.k), *vp = static_cast<const char*>(a.v);
  if constexpr (SRC == kPacked) kp += (d.k0 * a.k_row + (int64_t)kvh * a.k_head) * E, vp += (d.k0 * a.v_row + (int64_t)kvh * a.v_head) * E;
  const uint32_t k_bytes = (uint32_t)a.k_row * E, v_bytes = (uint32_t)a.v_row * E;
  static_assert((KB - 1) * (uint64_t)kMostRowBytes + 256 * 4 <= kNowhere, "a tile's rows have offsets of 32 bits, unsigned");
  uint32_t at_k[P], at_v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t p = (4 * i + wave) * kWave + lane, r = p / L::CH, c = p % L::CH;
    const int ck = L::k_chunk(r, c), cv = L::v_chunk(r, c);
    at_k[i] = ck * (16 / E) < a.d ? r * k_bytes + 16 * ck : kNowhere;
    at_v[i] = cv * (16 / E) < a.d ? r * v_bytes + 16 * cv : kNowhere;
    if constexpr (SRC != kPacked) at_k[i] = ck * (16 / E) < a.d ? lane / CB * (a.d * E) + 16 * ck : kNowhere,
                                  at_v[i] = cv * (16 / E) < a.d ? lane / CB * (a.d * E) + 16 * cv : kNowhere;
  }
  // Pages: rows RG (4 i + wave) .. of a tile are this wave's i-th, one for each CB lanes.
  constexpr int RG = rows_of_load(D, E, BITS8);
  // A lane's row and chunk of them.  8 bits: four lanes a row and four of the next one, or the widened chunks
  // of eight lanes, every second one of a row, would meet in the same banks of LDS.
  constexpr bool PAIRED = BITS8 && CB >= 8;
  const int my_row = PAIRED ? lane / (2 * CB) * 2 + lane / 4 % 2 : lane / CB;
  const int my_chunk = PAIRED ? lane % 4 + 4 * (lane / 8 % (CB / 4)) : lane % CB;
  const bool whole = EVEN && 1 << a.shift >= KB;  // a tile lies in one page
  int page[PB];  // of those rows of the tile that is brought next (EVEN), or of the lane's row
  u32x4 rk[BITS8 ? PB : 1], rv[BITS8 ? PB : 1];
  float k_scale[BITS8 ? PB : 1], v_scale[BITS8 ? PB : 1];
  const auto look_up = [&](int k0) {
#pragma unroll
    for (int i = 0; i < PB && SRC != kPacked; ++i) {
      const int place = k0 + RG * (4 * i + wave);
      if constexpr (EVEN) {
        if (i > 0 && whole) {
          page[i] = page[0];
          continue;
        }
        page[i] = -1;
        if (place < d.len_k)
          page[i] = ((__attribute__((address_space(4))) const int32_t*)a.table)[(int64_t)doc * a.table_row + (place >> a.shift)];
      } else {
        page[i] = page_at(a, doc, d, place + my_row);
      }
    }
  };
  // The first of a wave's rows (EVEN; else the lane's row) among those of its head in the pages.
  const uint32_t page_rows = (uint32_t)a.kv_heads << a.shift;
  if constexpr (SRC != kPacked) kp += ((int64_t)kvh << a.shift) * a.d * (BITS8 ? 1 : E), vp += ((int64_t)kvh << a.shift) * a.d * (BITS8 ? 1 : E);
  const auto row_at = [&](int i, int place) {
    return (uint64_t)(uint32_t)page[i] * page_rows + ((place + (EVEN ? 0 : my_row)) & ((1 << a.shift) - 1));
  };
  const auto bring = [&](int k0, int b) {
    if constexpr (SRC == kPacked) {
      const uint32_t keys = std::min(d.len_k - k0, KB);
      bring_rows<P>(kp + (int64_t)k0 * k_bytes, (keys - 1) * k_bytes + a.d * E, sk[b] + 1024 * wave, at_k);
      bring_rows<P>(vp + (int64_t)k0 * v_bytes, (keys - 1) * v_bytes + a.d * E, sv[b] + 1024 * wave, at_v);
    } else if constexpr (!BITS8) {
      const char* const none = reinterpret_cast<const char*>(kZeros);
      if (whole && k0 + KB <= d.len_k && (uint32_t)page[0] < (uint32_t)a.n_pages) {
        const uint64_t at = row_at(0, k0 + RG * wave) * (uint32_t)(a.d * E);
        const char *from_k = kp + at, *from_v = vp + at;
#pragma unroll
        for (int i = 0; i < PB; ++i, from_k += 4 * RG * a.d * E, from_v += 4 * RG * a.d * E) {
          if (at_k[i] != kNowhere) bring_from(from_k, at_k[i], sk[b] + 1024 * (wave + 4 * i));
          if (at_v[i] != kNowhere) bring_from(from_v, at_v[i], sv[b] + 1024 * (wave + 4 * i));
        }
        return;
      }
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        const int place = k0 + RG * (4 * i + wave);
        char *const to_k = sk[b] + 1024 * (wave + 4 * i), *const to_v = sv[b] + 1024 * (wave + 4 * i);
        const uint64_t at = row_at(i, place) * (uint32_t)(a.d * E);
        const int have = (uint32_t)page[i] < (uint32_t)a.n_pages ? d.len_k - place : 0;  // rows from here on
        if constexpr (EVEN) {
          // columns that do not exist were zeros before, and stay so
          if (have >= RG) {
            if (at_k[i] != kNowhere) bring_from(kp + at, at_k[i], to_k);
            if (at_v[i] != kNowhere) bring_from(vp + at, at_v[i], to_v);
          } else if (lane / CB < have) {
            if (at_k[i] != kNowhere) bring_from(kp + at, at_k[i], to_k);
            if (at_v[i] != kNowhere) bring_from(vp + at, at_v[i], to_v);
          } else {
            bring_from(none, 16 * lane, to_k);
            bring_from(none, 16 * lane, to_v);
          }
        } else {
          const uint64_t from = at - lane / CB * (a.d * E);
          bring_from(have > lane / CB && at_k[i] != kNowhere ? kp + from + at_k[i] : none, to_k);
          bring_from(have > lane / CB && at_v[i] != kNowhere ? vp + from + at_v[i] : none, to_v);
        }
      }
    } else {
      const float *const ks = a.k_scale + ((int64_t)kvh << a.shift), *const vs = a.v_scale + ((int64_t)kvh << a.shift);
      // (columns that do not exist are others of the row: they meet zeros, and what they add goes nowhere)
      const uint32_t r = EVEN ? my_row : 0, at = r * a.d + std::min(16 * my_chunk, a.d - 16);
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        const int first = RG * (4 * i + wave), place = k0 + first;
        const int have = first < KB && (uint32_t)page[i] < (uint32_t)a.n_pages ? d.len_k - place : 0;
        const uint64_t row = row_at(i, place);
        const auto load = [&] {
          k_scale[i] = (ks + row)[r];
          v_scale[i] = (vs + row)[r];
          rk[i] = *reinterpret_cast<const u32x4*>(kp + row * (uint32_t)a.d + at);
          rv[i] = *reinterpret_cast<const u32x4*>(vp + row * (uint32_t)a.d + at);
        };
        if (EVEN && have >= RG) {
          load();
        } else {
          rk[i] = rv[i] = u32x4{0, 0, 0, 0};
          k_scale[i] = v_scale[i] = 0.0f;
          if (my_row < have) load();
        }
      }
    }
  };
  const auto widen = [&](int b) {
    if constexpr (BITS8) {
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        const int r = RG * (4 * i + wave) + my_row, c = my_chunk;
        if (KB * CB % 256 != 0 && r >= KB) continue;
        const Scale split = split_scale<T>(v_scale[i]);
        if (c == 0) {
          reinterpret_cast<float*>(sscale[b][0])[r] = k_scale[i];
          reinterpret_cast<float*>(sscale[b][1])[r] = split.rest;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const Frag fk = from_e4m3<T>(rk[i][2 * j], rk[i][2 * j + 1], 1.0f);
          const Frag fv = from_e4m3<T>(rv[i][2 * j] | split.nan, rv[i][2 * j + 1] | split.nan, split.power);
#pragma unroll
          for (int m = 0; m < E / 2; ++m) {
            const int ch = c * E + (E / 2) * j + m;
            __builtin_memcpy(sk[b] + r * ROW + 16 * L::k_chunk(r, ch), reinterpret_cast<const char*>(&fk) + 16 * m, 16);
            __builtin_memcpy(sv[b] + r * ROW + 16 * L::v_chunk(r, ch), reinterpret_cast<const char*>(&fv) + 16 * m, 16);
          }
        }
      }
    }
  };
  // the first KT threads, one wave: a key's voxel each
  Near near = {0};
  bool near_q = false;
  if constexpr (MODE == kVoxel) {
    const int32_t* p = a.q_pos + 4 * (int64_t)(d.q0 + query);
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

  if (EVEN && !BITS8 && a.d * E < ROW) {
    for (int i = threadIdx.x; i < 2 * KB * (int)L::CH; i += 256)
      reinterpret_cast<u32x4*>(sk[0])[i] = reinterpret_cast<u32x4*>(sv[0])[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  if (k_begin < k_end) {
    look_up(k_begin);
    bring(k_begin, 0);
    look_up(k_begin + KB);
    fetch_voxel(k_begin);
    keep_voxel(0);
    widen(0);
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
          if (x >= D) continue;  // no product takes these (rows of 96 columns; of 8 bits they repeat the row's last)
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
      look_up(kb + 2 * KB);
      fetch_voxel(kb + KB);
    }
#pragma unroll 1
    for (int k0 = kb; k0 < std::min(kb + KB, last); k0 += KT) {
      const int sub = (k0 - kb) / KT;
      const char *const tk = sk[b] + sub * KT * ROW, *const tv = sv[b] + sub * KT * ROW;
      float s[KT / 2];
      const auto at = [&](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * half + i % 4; };
      const auto key = [&](int i) { return k0 + at(i); };
      // kPlace: the sums begin with the bias less that of the tile's first key, a line of at most 63 slopes; the
      // first key's, which is as large as the document is long, joins the maximum.  (Sums that began with
      // all of it would round each of their steps at its size, which shows where far keys count: negative slopes.)
      // Tiles beside the queries' own places have small distances, and begin with all of theirs.
      [[maybe_unused]] float bias[MODE == kPlace ? KT / 2 : 1], bias0 = 0.0f;
      if constexpr (MODE == kPlace) {
        const bool before = k0 + KT <= wave_place;
        if (even_slopes && (before || k0 >= wave_place + 32)) {
          const float slope = before ? q.slope : -q.slope, from = slope * (float)(4 * half);
          bias0 = slope * (float)(k0 - q.place);
#pragma unroll
          for (int i = 0; i < KT / 2; ++i) bias[i] = fmaf(slope, (float)(at(i) - 4 * half), from);
        } else {
#pragma unroll
          for (int i = 0; i < KT / 2; ++i) bias[i] = 0.0f;
          add_place_bias<KT / 2>(q, bias, key);
        }
      }
      {
        f32x16 acc[KT / 32];
#pragma unroll
        for (int h = 0; h < KT / 32; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[h][i] = MODE == kPlace && !BITS8 ? bias[16 * h + i] : 0.0f;
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
        if constexpr (BITS8) {
#pragma unroll
          for (int i = 0; i < KT / 2; ++i) {
            const float by = sscale[b][0][8 * (i / 16) + 2 * (i % 16 / 4) + half][i % 4];
            s[i] = MODE == kPlace ? fmaf(s[i], by, bias[i]) : s[i] * by;
          }
        }
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
        if (MODE != kBare && MODE != kPlace && a.cap > 0.0f) cap_scores<KT / 2, E == 4>(a, s);
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
        // (kPlace: the tile's scores and the maximum's both lack bias0)
        float top = MODE == kPlace ? -INFINITY : m;
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        float base = MODE == kPlace ? m - bias0 : m;
        if (__any(top > base)) {
          const float to = MODE != kPlace ? top : top > base ? top + bias0 : m, by = __builtin_amdgcn_exp2f((m - to) * a.exp_by);
          l *= by;
#pragma unroll
          for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= by;
          m = to;
          base = MODE == kPlace ? m - bias0 : m;
        }
        float off = fmaf(base, a.exp_by, -kExpRaise<T, BITS8>);
        const bool large = fabsf(off) > kMostOffset;
        if (__any(large)) {  // (of this row: others keep their bits)
          const float first = large ? base : 0.0f;
          off = large ? -kExpRaise<T, BITS8> : off;
#pragma unroll
          for (int i = 0; i < KT / 2; ++i) s[i] -= first;
        }
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.exp_by, -off));
      }
      {
        float sum[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i < KT / 2; ++i) sum[i % 4] += s[i];
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      if constexpr (BITS8) {
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) s[i] *= sscale[b][1][8 * (i / 16) + 2 * (i % 16 / 4) + half][i % 4];
      }
      Frag fp[KT / 16];  // rounded to the rows' type (attention.hip has why, and what it costs in the result)
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
    if (kb + KB < k_end) {
      keep_voxel(b ^ 1);
      widen(b ^ 1);
    }
  }

  const float sum = l + __shfl_xor(l, 32);
  if (row >= rows) return;
  const int64_t out_at = (int64_t)(d.q0 + query) * a.heads + head;
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
    T* out = static_cast<T*>(a.out) + (int64_t)(d.q0 + query) * a.out_row + (int64_t)head * a.out_head;
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

template <typename T, int MODE, int SRC>
void tile_mode(const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)(SRC == kPacked ? a.heads : a.kv_heads) * a.slots * a.splits));
#define SPC_D(D) hipLaunchKernelGGL((k_attn_tile<T, D, MODE, SRC>), grid, dim3(256), 0, s, a)
  if (a.d <= 32) SPC_D(32);
  else if (a.d <= 64) SPC_D(64);
  else if (a.d <= 96) SPC_D(96);
  else if (a.d <= 128) SPC_D(128);
  else SPC_D(256);
#undef SPC_D
}

template <typename T, int SRC>
void tile_t(const AttnArgs& a, hipStream_t s) {
  if constexpr (SRC != kSmall && SRC != kSmall8) {
    if (a.cap == 0.0f && !a.slopes) return tile_mode<T, kBare, SRC>(a, s);
    if constexpr (SRC == kPacked) {
      if (a.k_pos) return tile_mode<T, kVoxel, SRC>(a, s);
    }
    if constexpr (!std::is_same_v<T, _Float16>) {
      if (!a.slopes && a.cap <= kMostBoundedCap) return tile_mode<T, kCapped, SRC>(a, s);
    }
    if constexpr (SRC != kPacked) {
      if (a.cap == 0.0f) return tile_mode<T, kPlace, SRC>(a, s);
    }
  }
  tile_mode<T, kAny, SRC>(a, s);
}

template <int SRC>
hipError_t launch_tile(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  if (!fits_launch((SRC == kPacked ? a.heads : a.kv_heads) * p.slots * p.splits, 256)) return hipErrorInvalidConfiguration;
  if (dtype == 0) tile_t<float, SRC>(a, s);
  else if (dtype == 1) tile_t<_Float16, SRC>(a, s);
  else tile_t<__bf16, SRC>(a, s);
  return hipGetLastError();
}

}  // namespace attn
}  // namespace spc
