// What the attention kernels and the C-ABI share.
#pragma once

#include "rows.h"

namespace spc {

constexpr int kQueryTile = 128;  // queries of a workgroup of the many-query form
// Strides of key and value rows, in bytes: a tile's rows (up to 128) are addressed with 32 bits, unsigned.
constexpr int64_t kMostRowBytes = 1 << 25;

struct AttnArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head;  // strides in elements
  const int32_t* q_start;  // [n_docs + 1] first query of each document
  const int32_t* k_start;  // [n_docs + 1] first key of each document
  const int32_t* k_len;    // [n_docs] keys of each document, or NULL: up to the next one's first
  const int32_t* prefix;   // [n_docs] keys that all queries see, or NULL
  const float* slopes;     // [heads] or NULL
  const int32_t* q_pos;    // [n_q][4] voxels (b, x, y, z), or NULL: distance of places
  const int32_t* k_pos;    // [n_k][4]
  int64_t n_q, n_k;
  int n_docs, max_q, max_k, heads, kv_heads, d, causal;
  float cap;         // > 0: scores are capped
  float cap_log2;    // cap log2(e)
  float cap_by;      // scale / cap
  float tanh_by;     // 2 log2(e) scale / cap
  float low[2], low_most;    // capped scores of products up to low_most, by two terms (16-bit rows)
  float low_top;             // the score of low_most, in units of log2
  float poly[5], poly_most;  // capped scores of products up to poly_most, as an odd polynomial
  float slope_by;    // from the slopes' units to the scores'
  float exp_by;      // from the scores' units to log2
  float floor;       // where the running maximum starts
  int slots;          // of query tiles (many-query form)
  int splits, chunk;  // key ranges, and keys of each
  f32x2* part_ml;     // [splits][n_q][heads] maximum and sum of a range
  float* part_o;      // [splits][n_q][heads][d] its unnormalised output
  // Keys in pages (pages.h): k and v are theirs, k_row to v_head and k_start not used.
  const int32_t* table;  // [n_docs][table_row]
  const float* k_scale;  // NULL: pages hold the rows' type
  const float* v_scale;
  int paged, table_row, n_pages, shift;  // paged 0: packed keys
  int doc_slots;  // (pages) slots of each document; 0: they go by their queries
};

// How a call runs: few queries per document (rows: their columns) or many (slots of tiles of a head's
// queries, or of all queries of a key head's where the keys are in pages), and how its keys are split.
struct AttnPlan {
  bool rows;
  int cols;
  int64_t slots;
  int doc_slots;
  int splits, chunk;
};
AttnPlan attention_plan(int64_t n_q, int n_docs, int max_q, int max_k, int heads, int kv_heads, int d, int dtype,
                        bool causal, bool paged);
hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
// attention_tile.hip, attention_rows.hip: the two forms over packed keys; attention_pages.hip,
// attention_pages8.hip: both over pages of the rows' type and of 8 bits; attention_small.hip,
// attention_small8.hip: many queries over pages of fewer rows than a wave loads at once.
hipError_t launch_attention_tile(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
hipError_t launch_attention_rows(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
hipError_t launch_attention_pages(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
hipError_t launch_attention_pages8(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
hipError_t launch_attention_small(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);
hipError_t launch_attention_small8(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s);

}  // namespace spc
