// Product of 8-bit rows and 8-bit weights (e4m3), with a float32 scale for each row and 128
// columns of the rows and for each 128 x 128 block of the weights:
//   y[r][n] = relu?( sum_b xs[r][b] ws[n / 128][b] sum_{k in block b} x[r][k] w[n][k] )
//
// One matrix instruction multiplies 16 weights' rows by 16 rows over exactly one block of
// 128 columns (v_mfma_f32_16x16x128_f8f6f4); its float32 result is scaled and added to the
// float32 sums with one fma an element.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  void* y;
  int64_t ld_x, ld_xs, ld_w, ld_ws, ld_y;
  int64_t m;
  int n, k, kb;  // kb: blocks of 128 columns
  int relu;
  int wide_y;   // rows of y take 16-byte stores
  int wide_xs;  // rows of xs take 16-byte loads
};

// Eight e4m3 numbers as float16, exactly.
__device__ __forceinline__ f16x8 widen(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Product over a block of 128 columns: 32 consecutive bytes of a row a lane.  The 8-bit
// instruction drops a product that is 2^13 times smaller than the largest of its group of
// eight (measured): at most 7 2^-13 of the sum of magnitudes, and 1.4e-5 of the result where
// rows are quantised from normal values, which a 16-bit result's rounding covers.  EXACT
// widens both operands to float16, which holds every e4m3 number, and sums their products in
// float32, at half the rate.
template <bool EXACT>
__device__ __forceinline__ f32x4 mma128(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1) {
  if constexpr (!EXACT) {
    const i32x8 a = __builtin_bit_cast(i32x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
    const i32x8 b = __builtin_bit_cast(i32x8, __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7));
    // both operands e4m3; no hardware scales
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
  } else {
    f32x4 t = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 &x = i < 2 ? a0 : a1, &y = i < 2 ? b0 : b1;
      t = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(x[i % 2 * 2], x[i % 2 * 2 + 1]),
                                                 widen(y[i % 2 * 2], y[i % 2 * 2 + 1]), t, 0, 0, 0);
    }
    return t;
  }
}

// `count` consecutive outputs (a multiple of 4) of one row from column n0 on.
template <typename T, int COUNT>
__device__ __forceinline__ void store_y(const LinearArgs& a, int64_t row, int n0, const float* v) {
  if (row >= a.m) return;
  T* y = static_cast<T*>(a.y) + row * a.ld_y + n0;
  float r[COUNT];
#pragma unroll
  for (int i = 0; i < COUNT; ++i) r[i] = a.relu ? (v[i] < 0.0f ? 0.0f : v[i]) : v[i];
  constexpr int V = 16 / (int)sizeof(T) < COUNT ? 16 / (int)sizeof(T) : COUNT;
#pragma unroll
  for (int i = 0; i < COUNT; i += V) {
    if (a.wide_y && n0 + i + V <= a.n) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4*>(y + i) = f32x4{r[i], r[i + 1], r[i + 2], r[i + 3]};
      } else if constexpr (V == 8) {
        *reinterpret_cast<u32x4*>(y + i) = u32x4{pack2<T>(r[i], r[i + 1]), pack2<T>(r[i + 2], r[i + 3]),
                                                 pack2<T>(r[i + 4], r[i + 5]), pack2<T>(r[i + 6], r[i + 7])};
      } else {
        *reinterpret_cast<u32x2*>(y + i) = u32x2{pack2<T>(r[i], r[i + 1]), pack2<T>(r[i + 2], r[i + 3])};
      }
    } else {
#pragma unroll
      for (int j = i; j < i + V; ++j)
        if (n0 + j < a.n) y[j] = (T)r[j];
    }
  }
}

// ---------------------------------------------------------------------------
// Tiles: a workgroup of WM x WN waves takes BM rows and BN outputs, a block of 128 columns at
// a time through LDS.  With DEEP = 2 the next block of rows, weights and row scales is on its
// way from memory straight into the other half of LDS while one is multiplied.  Rows of 128 bytes: the
// 16-byte chunk c of row r lies at chunk c ^ r % 8, and a lane's 32 bytes of an operand row are
// its chunks g and g + 4: every read of 16 rows then meets every bank once (240 bytes a clock and
// CU measured; neighbouring chunks 2 g and 2 g + 1 in the same order give 126).  Rows and
// weights take their columns in the same order, so the products are the same.
//
// What bounds it: the parts of a step (256 x 256 x 128, 2.0 us) follow each other as much as they
// overlap, as the 8 waves of a CU go in step: of the cycles the matrix unit is busy in 49 %, the
// vector unit in 46 %, LDS in 26 % (3 % of them conflicts).  16,384 x 8192 x 4096: 505 to 526 us, 2.2
// PFLOP/s; a plain library product of e4m3, without scales, takes 357 us.  Tried: 128 x 128 tiles, two workgroups a CU (621 us where
// this took 519: twice the loads); weights two steps ahead (541); columns of 2 or 8 tiles per XCD (541,
// 544); loads spread over the products (557).
// ---------------------------------------------------------------------------

// WORDS times 4 bytes a lane from memory straight into LDS: those at `at` of the buffer (zeros
// outside of it) to where the wave's lanes follow each other from `to` on.  The caller waits
// (vmcnt); the compiler would await loads under way before every read of LDS.
template <int WORDS>
__device__ __forceinline__ void bring(u32x4 rsrc, int at, const void* to) {
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)to);
  uint32_t kept;  // M0 holds the LDS address
  if constexpr (WORDS == 4)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds), "v"(at), "s"(rsrc) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds), "v"(at), "s"(rsrc) : "memory");
}
__device__ __forceinline__ u32x4 buffer(const void* from, int64_t bytes) {
  const uint64_t base = reinterpret_cast<uint64_t>(from);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)base),
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xffffu),
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)bytes), 0x00020000u};
}

template <typename T, bool EXACT, int BM, int BN, int WM, int WN, int DEEP>
__global__ __launch_bounds__(64 * WM * WN, DEEP == 1 ? 3 : 2) void k_linear_tile(LinearArgs a) {
  constexpr int TH = 64 * WM * WN;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  constexpr int PX = BM * 8 / TH, PW = BN * 8 / TH;  // 16-byte chunks a thread brings
  static_assert(TH >= BM, "a thread brings at most one row scale");
  __shared__ __align__(16) u32x4 blocks[DEEP * (BM + BN) * 8];
  u32x4(*const sx)[BM * 8] = reinterpret_cast<u32x4(*)[BM * 8]>(blocks);
  u32x4(*const sw)[BN * 8] = reinterpret_cast<u32x4(*)[BN * 8]>(blocks + DEEP * BM * 8);
  __shared__ __align__(16) float sxs[2][BM * 4];  // row scales of four blocks
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int wm = wave / WN, wn = wave % WN;
  const int r16 = lane % 16, g = lane / 16;

  // Workgroups go around the 8 XCDs: each takes a run of tiles, in columns of 4 tiles of rows,
  // so that the 32 under way share rows and weights in its L2.
  const int tiles_m = (int)((a.m + BM - 1) / BM), tiles_n = (a.n + BN - 1) / BN;
  const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8, each = total / 8, rest = total % 8;
  const int tile = xcd * each + std::min(xcd, rest) + blockIdx.x / 8;
  const int strip = tile / (4 * tiles_n) * 4, high = std::min(4, tiles_m - strip), in = tile - strip * tiles_n;
  const int64_t m0 = (int64_t)(strip + in % high) * BM;
  const int n0 = in / high * BN;

  const int rows = (int)std::min<int64_t>(a.m - m0, BM), outs = std::min(a.n - n0, BN);
  const uint8_t* x = a.x + m0 * a.ld_x;
  const uint8_t* w = a.w + (int64_t)n0 * a.ld_w;
  int at_x[PX], at_w[PW];
#pragma unroll
  for (int i = 0; i < PX; ++i) {
    const int p = threadIdx.x + TH * i, r = p / 8, c = p % 8 ^ r % 8;
    at_x[i] = r < rows ? r * (int)a.ld_x + 16 * c : INT32_MIN;
  }
  // LDS row 16 t + 4 q + b of a wave's weights holds output 4 NT q + 4 t + b, so that a lane
  // ends with 4 NT consecutive outputs of its row
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int p = threadIdx.x + TH * i, r = p / 8, c = p % 8 ^ r % 8;
    const int in_wave = r % (16 * NT), out = r - in_wave + 4 * NT * (in_wave / 4 % 4) + 4 * (in_wave / 16) + in_wave % 4;
    at_w[i] = out < outs ? out * (int)a.ld_w + 16 * c : INT32_MIN;
  }
  const int at_s = (int)threadIdx.x < rows ? (int)threadIdx.x * (int)a.ld_xs * 4 : INT32_MIN;
  const int by_row = a.wide_xs ? 4 : 1, by_block = a.wide_xs ? 1 : BM;
  // constant memory: a scalar load, which does not wait for the tiles under way as a vector load would
  const auto ws = (const __attribute__((address_space(4))) float*)(
      a.ws + (int64_t)std::min((n0 + wn * 16 * NT) / kScaleBlock, (a.n - 1) / kScaleBlock) * a.ld_ws);

  const auto bring_block = [&](int b, int buf) {
    const int left = a.k - b * kScaleBlock;
    const u32x4 rx = buffer(x + (int64_t)b * kScaleBlock, (int64_t)(rows - 1) * a.ld_x + std::min(left, kScaleBlock));
    const u32x4 rw = buffer(w + (int64_t)b * kScaleBlock, (int64_t)(outs - 1) * a.ld_w + std::min(left, kScaleBlock));
    if (left < kScaleBlock) {  // the last block: its missing columns are zeros
#pragma unroll
      for (int i = 0; i < PX; ++i) {
        const int p = threadIdx.x + TH * i;
        if (16 * (p % 8 ^ p / 8 % 8) >= left) at_x[i] = INT32_MIN;
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        const int p = threadIdx.x + TH * i;
        if (16 * (p % 8 ^ p / 8 % 8) >= left) at_w[i] = INT32_MIN;
      }
    }
#pragma unroll
    for (int i = 0; i < PX; ++i) bring<4>(rx, at_x[i], &sx[buf][TH * i + 64 * wave]);
#pragma unroll
    for (int i = 0; i < PW; ++i) bring<4>(rw, at_w[i], &sw[buf][TH * i + 64 * wave]);
    if (b % 4 == 0 && 64 * wave < BM) {  // a row's scales of four blocks at once, where they are aligned
      const u32x4 rs = buffer(a.xs + m0 * a.ld_xs + b, ((int64_t)(rows - 1) * a.ld_xs + a.kb - b) * 4);
      if (a.wide_xs) {
        bring<4>(rs, at_s, &sxs[b / 4 % 2][256 * wave]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) bring<1>(rs, at_s + 4 * i, &sxs[b / 4 % 2][BM * i + 64 * wave]);
      }
    }
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  if (DEEP == 2 && a.kb > 0) bring_block(0, 0);
  for (int b = 0; b < a.kb; ++b) {
    const int buf = DEEP == 2 ? b & 1 : 0;
    if (DEEP == 1) {
      if (b > 0) __syncthreads();  // the block before is read
      bring_block(b, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of the block is in LDS
    __syncthreads();                     // and so are the others'; the other half is free
    if (DEEP == 2 && b + 1 < a.kb) bring_block(b + 1, buf ^ 1);
    const float sb = ws[b];
    u32x4 f[2][2], fw[NT][2];
    float scale[2];
    const auto rows_of = [&](int i) {
      const int r = wm * 16 * MT + 16 * i + r16;
#pragma unroll
      for (int h = 0; h < 2; ++h) f[i & 1][h] = sx[buf][r * 8 + ((g + 4 * h) ^ r % 8)];
      scale[i & 1] = sxs[b / 4 % 2][by_row * r + by_block * (b % 4)];
    };
    rows_of(0);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = wn * 16 * NT + 16 * j + r16;
#pragma unroll
      for (int h = 0; h < 2; ++h) fw[j][h] = sw[buf][r * 8 + ((g + 4 * h) ^ r % 8)];
    }
    // Strip by strip of 16 rows: a product of the strip before is scaled and added, then its
    // registers take one of this strip; the next strip's rows are read meanwhile.  The order
    // stands as written (left to itself the compiler keeps one strip's rows only: 537 us).
    f32x4 t[NT];
#pragma unroll
    for (int i = 0; i <= MT; ++i) {
      const float by = i > 0 ? scale[(i & 1) ^ 1] * sb : 0.0f;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (i > 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i > 0 ? i - 1 : 0][j][e] = fmaf(by, t[j][e], acc[i > 0 ? i - 1 : 0][j][e]);
        }
        if (i < MT) t[j] = mma128<EXACT>(fw[j][0], fw[j][1], f[i & 1][0], f[i & 1][1]);
        if (j == 1 && i + 1 < MT) rows_of(i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Through LDS, so that whole lines of a row are stored together, past the caches (11,003 x 768 x
  // 256 in float16: 10.5 us with a lane's 32 bytes stored by itself, so 7.5; stored together but
  // cached 8.9, by itself past the caches 13.5).  The 16-byte chunk c of row r lies at c ^ r % 16
  // (8, where a row has 8).
  constexpr int PER = 16 / (int)sizeof(T), CH = BN / PER, SW = CH < 16 ? CH : 16;
  static_assert(BM * CH <= DEEP * (BM + BN) * 8, "the tile fits the blocks' place");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = wm * 16 * MT + 16 * i + r16;
    float v[4 * NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = a.relu && acc[i][j][e] < 0.0f ? 0.0f : acc[i][j][e];
#pragma unroll
    for (int h = 0; h < 4 * NT / PER; ++h) {
      u32x4 w;
      if constexpr (PER == 4) {
        w = __builtin_bit_cast(u32x4, (f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]}));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack2<T>(v[8 * h + 2 * e], v[8 * h + 2 * e + 1]);
      }
      blocks[r * CH + ((wn * 16 * NT + 4 * NT * g) / PER + h ^ r % SW)] = w;
    }
  }
  __syncthreads();
  T* y = static_cast<T*>(a.y) + m0 * a.ld_y + n0;
  if (a.wide_y) {
#pragma unroll
    for (int i = 0; i < BM * CH / TH; ++i) {
      const int p = threadIdx.x + TH * i, r = p / CH, c = p % CH;
      if (r >= rows || PER * c >= outs) continue;
      const u32x4 w = blocks[r * CH + (c ^ r % SW)];
      if (PER * (c + 1) <= outs) {
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(y + r * a.ld_y + PER * c));
      } else {
        for (int e = 0; PER * c + e < outs; ++e)
          y[r * a.ld_y + PER * c + e] = reinterpret_cast<const T*>(&blocks[r * CH + (c ^ r % SW)])[e];
      }
    }
  } else {  // rows that no wide store fits: element by element
    for (int p = threadIdx.x; p < BM * BN; p += TH) {
      const int r = p / BN, c = p % BN;
      if (r < rows && c < outs)
        y[r * a.ld_y + c] = reinterpret_cast<const T*>(&blocks[r * CH + (c / PER ^ r % SW)])[c % PER];
    }
  }
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup takes 16 NT outputs and 16 MT rows; its waves share the blocks of 128
// columns out among themselves and add their sums through LDS at the end, in the order of
// the waves.  Operands go from memory straight into registers, up to 48 rows a block
// ahead of their products: a matrix operand's lane reads 32 consecutive bytes of its row, four
// lanes a whole 128-byte line.  What bounds it: latency.  A wave's first two blocks are under way
// together, each further one is a round trip to memory; then the waves join, all by the first
// of them where 16 rows and 16 outputs are a workgroup's.  (33 x 1001 x 4096 in float32 7.0 us.)
// ---------------------------------------------------------------------------
template <typename T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_linear_rows(LinearArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int r16 = lane % 16, g = lane / 16;
  const int n0 = blockIdx.x * 16 * NT;
  const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
  const uint8_t* w[NT];
  const uint8_t* x[MT];
  const float* xs[MT];
  const float* ws = a.ws + (int64_t)(n0 / kScaleBlock) * a.ld_ws;
#pragma unroll
  for (int j = 0; j < NT; ++j) w[j] = a.w + (int64_t)std::min(n0 + 16 * j + r16, a.n - 1) * a.ld_w + 32 * g;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = std::min<int64_t>(m0 + 16 * i + r16, a.m - 1);
    x[i] = a.x + row * a.ld_x + 32 * g;
    xs[i] = a.xs + row * a.ld_xs;
  }
  struct Block {
    u32x4 w[NT][2], x[MT][2];
    float xs[MT], ws;
  };
  const auto fetch = [&](int b, Block& k) {
    const int at = b * kScaleBlock;
    const bool in[2] = {at + 32 * g < a.k, at + 32 * g + 16 < a.k};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
        k.w[j][h] = in[h] ? *reinterpret_cast<const u32x4*>(w[j] + at + 16 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < MT; ++i)
        k.x[i][h] = in[h] ? *reinterpret_cast<const u32x4*>(x[i] + at + 16 * h) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) k.xs[i] = xs[i][b];
    k.ws = ws[b];
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  constexpr bool AHEAD = MT * NT <= 3;
  Block now, next;
  if (AHEAD && wave < a.kb) fetch(wave, now);
  for (int b = wave; b < a.kb; b += WAVES) {
    if (!AHEAD) fetch(b, now);
    else if (b + WAVES < a.kb) fetch(b + WAVES, next);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float by = now.xs[i] * now.ws;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const f32x4 t = mma128<true>(now.w[j][0], now.w[j][1], now.x[i][0], now.x[i][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(by, t[e], acc[i][j][e]);
      }
    }
    if (AHEAD) now = next;
  }
  __shared__ f32x4 part[WAVES][MT * NT][kWave];
#pragma unroll
  for (int i = 0; i < MT * NT; ++i) part[wave][i][lane] = acc[i / NT][i % NT];
  __syncthreads();
  for (int i = wave; i < MT * NT; i += WAVES) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int q = 1; q < WAVES; ++q) v += part[q][i][lane];
    float r[4] = {v[0], v[1], v[2], v[3]};
    store_y<T, 4>(a, m0 + 16 * (i / NT) + r16, n0 + 16 * (i % NT) + 4 * g, r);
  }
}

// The few-row form reads every row for each 16 or 32 outputs, but shares out the columns: it
// takes up to 64 rows, and more of them where one workgroup of 64 rows x 32 outputs a CU does
// the whole (float32; the best tiles in brackets: 281 x 143 x 672 5.1 us [7.4], 1000 x 256 x 2048 9.0
// [11.8], 70 x 4096 x 2048 9.9 [11.7], 281 x 1024 x 672 5.1 [6.5]; beyond it 1000 x 1024 x 512 6.4 [5.6],
// 2500 x 256 x 640 8.4 [5.9]).
bool few_rows(const LinearArgs& a) { return a.m <= 64 || (a.m + 63) / 64 * (((int64_t)a.n + 31) / 32) <= 256; }

template <typename T>
hipError_t linear_t(const LinearArgs& a, bool exact, hipStream_t s) {
  const auto launch = [&](auto kernel, int64_t x, int64_t y, int threads) {
    if (!fits_launch(x, threads) || y > 65535) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3((unsigned)x, (unsigned)y), dim3(threads), 0, s, a);
    return hipGetLastError();
  };
  const int64_t n = a.n;
#define SPC_R(MT, NT, WAVES) \
  return launch(k_linear_rows<T, MT, NT, WAVES>, (n + 16 * NT - 1) / (16 * NT), (a.m + 16 * MT - 1) / (16 * MT), 64 * WAVES)
// a wave for each block of columns, up to WAVES
#define SPC_W(MT, NT, WAVES)              \
  do {                                    \
    if (a.kb <= 4) SPC_R(MT, NT, 4);      \
    else if (a.kb <= 8) SPC_R(MT, NT, 8); \
    else SPC_R(MT, NT, WAVES);            \
  } while (0)
  if (few_rows(a)) {
    // As few rows a workgroup as one workgroup a CU allows: reading 16 (MT + NT) rows is what takes
    // its time (64 x 1024 x 4096: 14.9 us with 64 rows a workgroup, 6.8 with 16).  Where the outputs alone
    // fill the CUs twice, 32 of them a workgroup, as rows are then read half as often (64 x
    // 8192 x 4096: 29.6 -> 18.1 us), but for one strip of rows 16 and shorter workgroups (1 x 8192 x 8192:
    // 14.8 -> 13.6 us, with 32 outputs 19.7).
    const auto fits = [&](int mt) { return (a.m + 16 * mt - 1) / (16 * mt) * ((n + 15) / 16) <= 256; };
    const bool many = n > 4096;
    if (many && a.m <= 16) SPC_W(1, 1, 8);
    else if (many && a.m <= 32) SPC_W(2, 2, 8);
    else if (many && a.m <= 48) SPC_W(3, 2, 8);
    else if (many) SPC_W(4, 2, 8);
    else if (a.m <= 16 || fits(1)) SPC_W(1, 1, 16);
    else if (a.m <= 32 || fits(2)) SPC_W(2, 1, 16);
    else if (a.m <= 48 || fits(3)) SPC_W(3, 1, 16);
    else if (a.m <= 64 || fits(4)) SPC_W(4, 1, 16);
    else SPC_W(4, 2, 8);
  }
#undef SPC_W
#undef SPC_R
#define SPC_T(EXACT, BM, BN, WM, WN, DEEP) \
  return launch(k_linear_tile<T, EXACT, BM, BN, WM, WN, DEEP>, (a.m + BM - 1) / BM * ((n + BN - 1) / BN), 1, 64 * WM * WN)
  // Tiles by how many of 128 x 128 there are.  Few leave CUs idle, for which smaller ones are
  // worth their reads (bfloat16, tiles of 64 x 64, 64 x 128, 128 x 128: 1500 x 2048 x 1024, 192 of
  // them: 8.3, 8.7, 9.9 us; 1000 x 1024 x 2048 9.1, 11.2, 14.9; 4000 x 1024 x 1024, 256 of them: 10.0, 8.8,
  // 9.8; 3000 x 1500 x 4096, 288: 42.3, 34.7, 39.0; 4000 x 2048 x 1024, 512: 17.8, 16.8, 13.6).
  //
  // Up to 512 columns: one block in LDS at a time, so that three workgroups share a CU and cover
  // each other's loads and stores (32,043 x 768 x 256: 15.3 us, with large tiles 20.5; 11,003 x 768 x 256: 7.5,
  // with two blocks 9; 1024 columns: 14.9, and 13.6 with two).  Float32 outputs of such a tile do
  // not fit its one block; 64 x 128 does there (11,003 x 768 x 256: 11.6 against 15.6).  Else
  // large tiles where they fill the CUs.
  const int64_t tiles = ((a.m + 127) / 128) * ((n + 127) / 128);
  if constexpr (!std::is_same_v<T, float>) {
    if (!exact) {
      if (tiles <= 192) SPC_T(false, 64, 64, 2, 2, 2);
      else if (tiles <= 384) SPC_T(false, 64, 128, 2, 2, 2);
      else if (a.kb <= 4) SPC_T(false, 128, 128, 2, 2, 1);
      else if (((a.m + 255) / 256) * ((n + 255) / 256) >= 256) SPC_T(false, 256, 256, 2, 4, 2);
      else SPC_T(false, 128, 128, 2, 2, 2);
    }
  }
  if (tiles <= 192) SPC_T(true, 64, 64, 2, 2, 2);
  else if (tiles <= 384 || a.kb <= 4) SPC_T(true, 64, 128, 2, 2, 2);
  else SPC_T(true, 128, 128, 2, 2, 2);
#undef SPC_T
}

}  // namespace

hipError_t launch_scaled_linear(const void* x, int64_t ld_x, const float* xs, int64_t ld_xs, const void* w, int64_t ld_w,
                                const float* ws, int64_t ld_ws, void* y, int64_t ld_y, int64_t m, int n, int k, int dtype,
                                int relu, bool exact, hipStream_t s) {
  if (m <= 0 || n <= 0) return hipSuccess;
  ProfScope ps(KN_SCALED_LINEAR, s);
  const int64_t e = dtype == 0 ? 4 : 2;
  LinearArgs a = {static_cast<const uint8_t*>(x), xs, static_cast<const uint8_t*>(w), ws, y, ld_x, ld_xs, ld_w, ld_ws,
                  ld_y, m, n, k, (k + kScaleBlock - 1) / kScaleBlock, relu, 0, 0};
  a.wide_xs = reinterpret_cast<uintptr_t>(xs) % 16 == 0 && ld_xs % 4 == 0;
  a.wide_y = reinterpret_cast<uintptr_t>(y) % 16 == 0 && ld_y * e % 16 == 0;
  if (dtype == 0) return linear_t<float>(a, true, s);
  if (dtype == 1) return linear_t<_Float16>(a, exact, s);
  return linear_t<__bf16>(a, exact, s);
}

}  // namespace spc
