// A cache of pages, as its kernels see it: pages [n_pages][kv_heads][page][d] of keys and of
// values, in the rows' type or in e4m3 with a float32 scale for each row of a head, and a table
// of each document's pages.
#pragma once

#include "rows.h"

namespace spc {

struct PageArgs {
  void* k;
  void* v;
  float* k_scale;  // [n_pages][kv_heads][page], or NULL: pages hold the rows' type
  float* v_scale;
  const int32_t* table;  // [n_docs][table_row]
  int n_docs, table_row, n_pages, shift;  // 1 << shift rows a page
  int kv_heads, d;
};

// Where rows of [rows][kv_heads][d] lie outside of the pages, in elements.
struct HeadRows {
  void* p;
  int64_t row, head;
};

// cache.hip.  write: row i of the batch is token i - start[t] of its document t, which holds len[t]
// tokens with the new ones; read (len NULL): row i is key i - start[t].
hipError_t launch_cache(const PageArgs& a, const HeadRows& k, const HeadRows& v, const int32_t* start, const int32_t* len,
                        int64_t n, int dtype, hipStream_t s);

// The row of the pages that holds a key of one head, or -1 where the table names no page.
__device__ __forceinline__ int64_t page_row(const PageArgs& a, int page, int place, int head) {
  if ((uint32_t)page >= (uint32_t)a.n_pages) return -1;
  return (((int64_t)page * a.kv_heads + head) << a.shift) + (place & ((1 << a.shift) - 1));
}

}  // namespace spc
