// cache.cpp -- C ABI entry points of the paged key/value cache and of the
// attention operators: argument checks and launch plans.
#include "cache.hpp"

#include <algorithm>
#include <cmath>

namespace mnmt {
namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Checks a configuration within bounds that keep the kernels' products and
// grids in range; returns why it is refused, or null.
const char* shape_of(const mnmt_pages_cfg* c, PagesShape* s) {
  if (!c) return "the page configuration is null";
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return "page_size must be 16, 32, 64, 128 or 256";
  if (c->d_head < 16 || c->d_head > 128 || c->d_head % 16) return "d_head must be a multiple of 16 from 16 to 128";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256) return "n_kv_heads must be 1..256";
  if (c->n_layers < 1 || c->n_layers > 256) return "n_layers must be 1..256";
  if (c->n_pages < 1 || c->n_pages > kMaxPages) return "n_pages must be 1..4194304";
  if (c->max_pages < 1 || c->max_pages > (1 << 30) / c->page_size)
    return "max_pages must be at least 1 and max_pages * page_size at most 2^30";
  int shift = 4;
  while ((1 << shift) < c->page_size) ++shift;
  *s = PagesShape{c->n_layers, c->n_pages, c->page_size, shift, c->n_kv_heads, c->d_head, c->max_pages,
                  (size_t)2 * c->n_kv_heads * c->page_size * c->d_head};
  if (pages_copy_parts(*s) > 65534) return "a page of all layers must be at most 1 GB";
  return nullptr;
}

int bad(const char* why) { return set_error(MNMT_E_INVALID_ARG, why); }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

bool rows_fit(const PagesShape& s, int rows) {
  return rows >= 0 && rows <= kMaxCacheRows && (long)rows * s.max_pages <= (1L << 30);
}

// Tokens of a call: rows' starts on the device, or as many for each row.
const char* tokens_of(int rows, const void* start, int n) {
  if (n < 0) return "n must not be negative";
  if (!start && (rows < 1 ? n > 0 : n % rows != 0)) return "without d_start, n must be a multiple of rows";
  return nullptr;
}

// What both attention operators check and fill in.
const char* attn_of(const mnmt_attn_cfg* c, int n_kv_heads, int d_head, AttnArgs* a) {
  if (!c) return "the attention configuration is null";
  if (n_kv_heads < 1 || n_kv_heads > 256 || c->n_heads < 1 || c->n_heads > 4096 || c->n_heads % n_kv_heads)
    return "n_heads must be a multiple of n_kv_heads (1..256), at most 4096";
  if (d_head < 16 || d_head > 128 || d_head % 16) return "d_head must be a multiple of 16 from 16 to 128";
  if (c->kind != MNMT_ATTN_I8 && c->kind != MNMT_ATTN_F32) return "unknown output kind";
  if (c->ld_q % 16 || c->ld_q < c->n_heads * d_head) return "ld_q must be a multiple of 16, at least n_heads * d_head";
  if (c->ld_out % 4 || c->ld_out < c->n_heads * d_head)
    return "ld_out must be a multiple of 4, at least n_heads * d_head";
  if (!(c->c_qk >= 0.0f) || !std::isfinite(c->c_qk) || c->c_qk > 1e30f || !std::isfinite(c->c_pv))
    return "c_qk must be 0..1e30 and c_pv finite";
  if (c->max_q < 0 || c->max_len < 0) return "max_q and max_len must not be negative";
  a->group = c->n_heads / n_kv_heads;
  a->n_kv_heads = n_kv_heads;
  a->kind = c->kind;
  a->ldq = c->ld_q;
  a->ldo = c->ld_out;
  a->c2 = (float)((double)c->c_qk * 1.44269504088896340736);
  a->c_pv = c->c_pv;
  return nullptr;
}

int run_attn(AttnArgs& a, bool paged, int d_head, int max_q, int max_len, void* d_ws, size_t ws_bytes, void* stream) {
  if ((long)a.n * a.group > (1L << 30)) return bad("n * n_heads / n_kv_heads must be at most 2^30");
  const AttnPlan p = plan_attn(a.rows, a.n, a.n_kv_heads, a.group, d_head, std::min(max_q, a.n), max_len);
  if (p.ws_bytes > ws_bytes) return bad("the workspace is smaller than mnmt_attn_ws_bytes");
  if (p.ws_bytes && (!d_ws || !aligned(d_ws, 16))) return bad("the workspace must be 16-byte aligned and not null");
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.waves = p.waves;
  a.queries = p.queries;
  a.is_short = p.is_short;
  a.part = static_cast<float*>(d_ws);
  a.tops = reinterpret_cast<int*>(static_cast<char*>(d_ws) + p.part_bytes);
  const hipError_t h = launch_attn(a, paged, d_head, static_cast<hipStream_t>(stream));
  return h == hipSuccess ? MNMT_OK : hip_error(h, "attention launch");
}

}  // namespace

// A unit: a query tile (16 queries) of a row and key head.  Measured us, one form |
// the other:
// - The chunk kernels (waves 0) read keys and values once for a block's queries
//   but are two launches with barriers: from eight tiles per head and enough work
//   on.  Heads of 64: 4096 units x 700 keys 38 | 54, 1024 x 8000 87 | 109, 2048 x
//   700 27 | 26, 512 x 1500 37 | 29.  Heads of 128: 2048 x 700 33 | 44, 1024 x 8000
//   135 | 189, 1024 x 1000 35 | 32, 2048 x 200 21 | 20; of four tiles 2048 x 1000 72 | 50.
// - One wave per unit from 512 units on (heads of 64, against four: 1024 x 700 18 | 59,
//   512 x 1500 31 | 49, 256 x 1500 28 | 21), four below.
// - The keys of a unit go to several waves or blocks, and are joined, while that
//   fills the GPU twice over (16 rows of 8 key heads, 1000-32000 keys, 2048 blocks 117,
//   1024 138, 4096 125), in ranges of at least 512 keys for four waves and 1024 for one.
// - Rows of at most two steps (short) want waves more than keys a step ahead: 512
//   rows of 8 heads, 20-80 keys, 10.4 | 12.3.
AttnPlan plan_attn(int rows, int n, int n_kv_heads, int group, int d_head, int max_q, int max_len) {
  AttnPlan p{};
  const long heads = (long)rows * n_kv_heads;  // <= kMaxAttnUnits
  const long tiles = std::max(1L, ((long)max_q * group + 15) / 16);
  p.tiles = (int)std::min(tiles, kMaxAttnUnits / std::max(1L, heads));  // (a block goes on to further tiles)
  const long units = heads * p.tiles;
  p.queries = (int)std::max(1L, std::min(16L, (long)max_q * group));
  p.splits = 1;
  p.chunk = 1 << 30;
  // `want` ranges of at least `least` keys
  auto split = [&](long want, int least) {
    want = std::min(want, (long)max_len / least);
    if (want < 2) return;
    p.chunk = (int)((max_len + want - 1) / want + 255) / 256 * 256;
    p.splits = (max_len + p.chunk - 1) / p.chunk;
  };
  p.is_short = max_len <= 128;
  if (p.tiles >= 8 && units * max_len >= (d_head <= 64 ? 2800000L : 1000000L)) {
    p.waves = 0;
    p.tiles = (p.tiles + 7) / 8 * 8;
    const long blocks = heads * p.tiles / (d_head <= 64 ? 8 : 4);
    split((512 + blocks - 1) / blocks, 1024);
  } else if (p.is_short || units >= 512) {
    p.waves = 1;
    split((4096 + units - 1) / units, 1024);
  } else {
    p.waves = 4;
    split((2048 + units - 1) / units, 512);
  }
  const size_t slots = ((size_t)n * group / 16 + rows + 1) * n_kv_heads * p.splits;  // tile_slot
  if (p.splits > 1) p.part_bytes = slots * 16 * (d_head + 2) * sizeof(float);
  p.ws_bytes = p.part_bytes + (p.waves == 0 ? slots * 16 * sizeof(int) : 0);
  return p;
}

hipError_t launch_attn(const AttnArgs& a, bool paged, int d_head, hipStream_t s) {
  return paged ? launch_attn_kernel<true>(a, d_head, s) : launch_attn_kernel<false>(a, d_head, s);
}

}  // namespace mnmt

using namespace mnmt;

extern "C" size_t mnmt_pages_bytes(const mnmt_pages_cfg* cfg) {
  PagesShape s;
  return shape_of(cfg, &s) ? 0 : (size_t)s.n_layers * s.n_pages * s.page_bytes;
}

extern "C" size_t mnmt_pages_ws_bytes(const mnmt_pages_cfg* cfg, int rows) {
  PagesShape s;
  return shape_of(cfg, &s) || !rows_fit(s, rows) ? 0 : pages_ws_bytes(s, rows);
}

extern "C" int mnmt_pages_fork(const mnmt_pages_cfg* cfg, void* d_pool, const int32_t* d_table, const int32_t* d_len,
                               int rows_in, const int32_t* d_parent, const int32_t* d_new, int rows,
                               int32_t* d_table_out, int32_t* d_len_out, int32_t* d_info, void* d_ws, size_t ws_bytes,
                               void* stream) {
  PagesFork f{};
  if (const char* why = shape_of(cfg, &f.s)) return bad(why);
  if (!rows_fit(f.s, rows_in) || !rows_fit(f.s, rows)) return bad("rows must be 0..2^20 and rows * max_pages at most 2^30");
  if (!d_parent && rows > rows_in) return bad("without d_parent, there can be no more output rows than input rows");
  if (!d_info || !d_ws) return bad("null device pointer");
  if (rows > 0 && (!d_pool || !d_table_out || !d_len_out)) return bad("null device pointer");
  if (rows_in > 0 && (!d_table || !d_len)) return bad("null device pointer");
  if (!aligned(d_pool, 16) || !aligned(d_ws, 16)) return bad("the pool and the workspace must be 16-byte aligned");
  if (ws_bytes < pages_ws_bytes(f.s, rows)) return bad("the workspace is smaller than mnmt_pages_ws_bytes");
  if (rows > 0 && rows_in > 0) {
    const size_t tin = sizeof(int32_t) * rows_in * f.s.max_pages, tout = sizeof(int32_t) * rows * f.s.max_pages;
    const size_t lin = sizeof(int32_t) * rows_in, lout = sizeof(int32_t) * rows;
    if ((overlap(d_table, tin, d_table_out, tout) && (d_parent || d_table != d_table_out)) ||
        (overlap(d_len, lin, d_len_out, lout) && (d_parent || d_len != d_len_out)))
      return bad("the output tables may be the input tables only without d_parent, and may not overlap otherwise");
  }
  f.pool = static_cast<int8_t*>(d_pool);
  f.table = d_table;
  f.len = d_len;
  f.parent = d_parent;
  f.grow = d_new;
  f.rows_in = rows_in;
  f.rows = rows;
  const hipError_t h = launch_pages_fork(f, d_table_out, d_len_out, d_info, d_ws, static_cast<hipStream_t>(stream));
  return h == hipSuccess ? MNMT_OK : hip_error(h, "fork launch");
}

extern "C" int mnmt_pages_compact(const mnmt_pages_cfg* cfg, void* d_pool, const int32_t* d_table,
                                  const int32_t* d_len, int rows, int32_t* d_table_out, int32_t* d_info, void* d_ws,
                                  size_t ws_bytes, void* stream) {
  PagesFork f{};
  if (const char* why = shape_of(cfg, &f.s)) return bad(why);
  if (!rows_fit(f.s, rows)) return bad("rows must be 0..2^20 and rows * max_pages at most 2^30");
  if (!d_info || !d_ws || (rows > 0 && (!d_pool || !d_table || !d_len || !d_table_out)))
    return bad("null device pointer");
  if (!aligned(d_pool, 16) || !aligned(d_ws, 16)) return bad("the pool and the workspace must be 16-byte aligned");
  if (ws_bytes < pages_ws_bytes(f.s, rows)) return bad("the workspace is smaller than mnmt_pages_ws_bytes");
  const size_t bytes = sizeof(int32_t) * rows * f.s.max_pages;
  if (rows > 0 && d_table != d_table_out && overlap(d_table, bytes, d_table_out, bytes))
    return bad("the output table may be the input table but may not overlap it otherwise");
  f.pool = static_cast<int8_t*>(d_pool);
  f.table = d_table;
  f.len = d_len;
  f.rows_in = f.rows = rows;
  const hipError_t h = launch_pages_compact(f, d_table_out, d_info, d_ws, static_cast<hipStream_t>(stream));
  return h == hipSuccess ? MNMT_OK : hip_error(h, "compact launch");
}

extern "C" int mnmt_pages_write(const mnmt_pages_cfg* cfg, void* d_pool, int layer, const int32_t* d_table,
                                const int32_t* d_len, int rows, const int8_t* d_k, const int8_t* d_v, int64_t ld,
                                const int32_t* d_start, int n, int max_q, void* stream) {
  PagesWrite w{};
  if (const char* why = shape_of(cfg, &w.s)) return bad(why);
  if (layer < 0 || layer >= w.s.n_layers) return bad("no such layer");
  if (!rows_fit(w.s, rows)) return bad("rows must be 0..2^20 and rows * max_pages at most 2^30");
  if (const char* why = tokens_of(rows, d_start, n)) return bad(why);
  if (ld % 16 || ld < (int64_t)w.s.n_kv_heads * w.s.d_head)
    return bad("ld must be a multiple of 16, at least n_kv_heads * d_head");
  if (max_q < 0) return bad("max_q must not be negative");
  if (rows == 0 || n == 0) return MNMT_OK;
  if (!d_pool || !d_table || !d_len || !d_k || !d_v) return bad("null device pointer");
  if (!aligned(d_pool, 16) || !aligned(d_k, 16) || !aligned(d_v, 16))
    return bad("the pool, K and V must be 16-byte aligned");
  w.pool = static_cast<int8_t*>(d_pool) + (size_t)layer * w.s.n_pages * w.s.page_bytes;
  w.table = d_table;
  w.len = d_len;
  w.start = d_start;
  w.k = d_k;
  w.v = d_v;
  w.ld = ld;
  w.n = n;
  w.rows = rows;
  const hipError_t h = launch_pages_write(w, d_start ? std::min(max_q, n) : n / rows, static_cast<hipStream_t>(stream));
  return h == hipSuccess ? MNMT_OK : hip_error(h, "write launch");
}

extern "C" size_t mnmt_attn_ws_bytes(int rows, int n, int n_heads, int n_kv_heads, int d_head, int max_q,
                                     int max_len) {
  if (rows < 1 || n < 1 || n_kv_heads < 1 || (long)rows * n_kv_heads > kMaxAttnUnits || n_kv_heads > 256 || n_heads < 1 || n_heads > 4096 ||
      n_heads % n_kv_heads || (long)n * (n_heads / n_kv_heads) > (1L << 30) || d_head < 16 || d_head > 128 ||
      d_head % 16 || max_q < 0 || max_len < 0)
    return 0;
  return plan_attn(rows, n, n_kv_heads, n_heads / n_kv_heads, d_head, std::min(max_q, n), max_len).ws_bytes;
}

extern "C" int mnmt_attn_paged(const mnmt_pages_cfg* pages, const mnmt_attn_cfg* cfg, const void* d_pool, int layer,
                               const int32_t* d_table, const int32_t* d_len, int rows, const int8_t* d_q,
                               const int32_t* d_start, int n, void* d_out, void* d_ws, size_t ws_bytes, void* stream) {
  AttnArgs a{};
  PagesShape s;
  if (const char* why = shape_of(pages, &s)) return bad(why);
  if (const char* why = attn_of(cfg, s.n_kv_heads, s.d_head, &a)) return bad(why);
  if (layer < 0 || layer >= s.n_layers) return bad("no such layer");
  if (!rows_fit(s, rows)) return bad("rows must be 0..2^20 and rows * max_pages at most 2^30");
  if (const char* why = tokens_of(rows, d_start, n)) return bad(why);
  if ((long)rows * s.n_kv_heads > kMaxAttnUnits) return bad("rows * n_kv_heads must be at most 2^23");
  if (rows == 0 || n == 0) return MNMT_OK;
  if (!d_pool || !d_table || !d_len || !d_q || !d_out) return bad("null device pointer");
  if (!aligned(d_pool, 16) || !aligned(d_q, 16) || !aligned(d_out, 16))
    return bad("the pool, Q and the output must be 16-byte aligned");
  a.q = d_q;
  a.out = d_out;
  a.start = d_start;
  a.len = d_len;
  a.n = n;
  a.rows = rows;
  a.causal = cfg->causal != 0;
  a.pool = static_cast<const int8_t*>(d_pool) + (size_t)layer * s.n_pages * s.page_bytes;
  a.table = d_table;
  a.n_pages = s.n_pages;
  a.shift = s.shift;
  a.max_pages = s.max_pages;
  a.page_bytes = s.page_bytes;
  a.cap = s.max_pages << s.shift;
  return run_attn(a, true, s.d_head, cfg->max_q, std::min(cfg->max_len, a.cap), d_ws, ws_bytes, stream);
}

extern "C" int mnmt_attn_cross(const mnmt_attn_cfg* cfg, int n_kv_heads, int d_head, const int8_t* d_k,
                               const int8_t* d_v, int64_t ld, int64_t batch, int S, const int32_t* d_len, int rows,
                               const int8_t* d_q, const int32_t* d_start, int n, void* d_out, void* d_ws,
                               size_t ws_bytes, void* stream) {
  AttnArgs a{};
  if (const char* why = attn_of(cfg, n_kv_heads, d_head, &a)) return bad(why);
  if (rows < 0 || (long)rows * n_kv_heads > kMaxAttnUnits)
    return bad("rows must not be negative and rows * n_kv_heads at most 2^23");
  if (S < 0 || S > (1 << 30)) return bad("S must be 0..2^30");
  if (cfg->causal) return bad("cross attention is not causal");
  if (ld % 16 || ld < (int64_t)n_kv_heads * d_head || batch % 16 || batch < 0)
    return bad("ld must be a multiple of 16, at least n_kv_heads * d_head, and batch a multiple of 16");
  if (const char* why = tokens_of(rows, d_start, n)) return bad(why);
  if (rows == 0 || n == 0) return MNMT_OK;
  if ((S > 0 && (!d_k || !d_v)) || !d_len || !d_q || !d_out) return bad("null device pointer");
  if (!aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_q, 16) || !aligned(d_out, 16))
    return bad("K, V, Q and the output must be 16-byte aligned");
  a.q = d_q;
  a.out = d_out;
  a.start = d_start;
  a.len = d_len;
  a.n = n;
  a.rows = rows;
  a.k = d_k;
  a.v = d_v;
  a.ld = ld;
  a.batch = batch;
  a.cap = S;
  return run_attn(a, false, d_head, cfg->max_q, std::min(cfg->max_len, S), d_ws, ws_bytes, stream);
}
