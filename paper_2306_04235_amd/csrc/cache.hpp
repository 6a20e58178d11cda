// cache.hpp -- the paged key/value cache and the attention operators: what the
// entry points (cache.cpp) hand to the kernels (pages.hip, attn_*.hip).
#pragma once

#include "internal.h"

namespace mnmt {

// A checked mnmt_pages_cfg.
struct PagesShape {
  int n_layers, n_pages, page_size, shift, n_kv_heads, d_head, max_pages;  // page_size = 1 << shift
  size_t page_bytes;  // of one layer
};

constexpr int kMaxPages = 1 << 22, kMaxCacheRows = 1 << 20;
constexpr long kMaxAttnUnits = 1 << 23;  // query tiles of a launch

struct PagesFork {
  PagesShape s;
  int8_t* pool;
  const int32_t *table, *len;
  const int32_t *parent, *grow;  // null: each row its own parent; null: no new tokens
  int rows_in, rows;
};

struct PagesWrite {
  PagesShape s;
  int8_t* pool;  // of the layer
  const int32_t *table, *len, *start;
  const int8_t *k, *v;
  long ld;
  int n, rows;
};

size_t pages_ws_bytes(const PagesShape& s, int rows);
int pages_copy_parts(const PagesShape& s);  // blocks that copy one page of all layers
hipError_t launch_pages_fork(const PagesFork& f, int32_t* table_out, int32_t* len_out, int32_t* info, void* ws,
                             hipStream_t s);
hipError_t launch_pages_compact(const PagesFork& f, int32_t* table_out, int32_t* info, void* ws, hipStream_t s);
hipError_t launch_pages_write(const PagesWrite& w, int max_q, hipStream_t s);

// One attention call.  A row's queries (n of its tokens, G = group heads each
// per key head) are taken 16 (token, head) pairs at a time: a query tile.
struct AttnArgs {
  const int8_t* q;
  void* out;
  const int32_t *start, *len;
  int n, rows, ldq, ldo, group, n_kv_heads, kind, causal;
  float c2, c_pv;  // c_qk log2 e; values' scale
  // the launch (AttnPlan): query tiles per row and key head in the grid, key
  // ranges of `chunk` keys per tile, their partial results, a chunk's maxima
  int tiles, splits, chunk, waves, queries;
  bool is_short;
  float* part;
  int* tops;
  // keys and values: pages of one layer, or rows [sentence][S]
  const int8_t* pool;
  const int32_t* table;
  int n_pages, shift, max_pages;
  size_t page_bytes;
  const int8_t *k, *v;
  long ld, batch;
  int cap;  // longest length
};

// The launch of a call, by the caller's bounds, and the workspace that it needs.
struct AttnPlan {
  int tiles, splits, chunk;
  int waves;    // per query tile: 1 or 4; 0: the chunk kernels
  int queries;  // of a tile
  bool is_short;
  size_t part_bytes, ws_bytes;
};
AttnPlan plan_attn(int rows, int n, int n_kv_heads, int group, int d_head, int max_q, int max_len);
hipError_t launch_attn(const AttnArgs& a, bool paged, int d_head, hipStream_t s);
template <bool PAGED>
hipError_t launch_attn_kernel(const AttnArgs& a, int d_head, hipStream_t s);

}  // namespace mnmt
