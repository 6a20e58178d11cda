// pages.hip -- the paged key/value cache: fork (parents, freeing, copies on
// write, room for new tokens), compaction, and writing the codes of new tokens.
//
// No state beside the tables: which pages are free is what the output tables do
// not name, found anew by each call, so there are no reference counts to keep in
// step and a call can be repeated.
#include <algorithm>
#include <climits>

#include "blocks.hpp"
#include "cache.hpp"

namespace mnmt {
namespace {

__device__ __forceinline__ int clamped(long v, long lo, long hi) { return (int)(v < lo ? lo : v > hi ? hi : v); }

// What becomes of an output row before pages are handed out.
struct RowPlan {
  int parent;  // its row of the input table, or -1
  int kept;    // tokens it keeps
  int len;     // tokens it has room for afterwards
  int whole;   // first pages it shares
  int old;     // pages that hold the kept tokens: `whole`, or one more that it is to write to
  int pages;   // pages it has afterwards
};

__device__ __forceinline__ RowPlan plan_row(const PagesFork& f, int r) {
  RowPlan p;
  p.parent = f.parent ? f.parent[r] : r;
  if (p.parent < 0 || p.parent >= f.rows_in) p.parent = -1;
  const long cap = (long)f.s.max_pages << f.s.shift;
  const long len = p.parent < 0 ? 0 : clamped(f.len[p.parent], 0, cap);
  p.len = clamped(len + (f.grow ? (long)f.grow[r] : 0), 0, cap);
  p.kept = min((int)len, p.len);
  const int up = f.s.page_size - 1;
  p.old = (p.kept + up) >> f.s.shift;
  p.whole = p.len > p.kept ? p.kept >> f.s.shift : p.old;
  p.pages = (int)(((long)p.len + up) >> f.s.shift);
  return p;
}

// A page of the input table, or -1 where the entry names none.
__device__ __forceinline__ int page_at(const PagesShape& s, const int32_t* table, int row, int col) {
  const int p = table[(size_t)row * s.max_pages + col];
  return p < 0 || p >= s.n_pages ? -1 : p;
}

__global__ __launch_bounds__(256) void k_pages_clear(int* first, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) first[i] = INT_MAX;
}

// first[p] = -1 if a row shares page p, else the lowest row that is to write to
// it, else INT_MAX (free).  One block per row.
__global__ __launch_bounds__(64) void k_fork_mark(PagesFork f, int* first) {
  const int r = blockIdx.x;
  const RowPlan p = plan_row(f, r);
  if (p.parent < 0) return;
  for (int c = threadIdx.x; c < p.old; c += 64) {
    const int page = page_at(f.s, f.table, p.parent, c);
    if (page >= 0) atomicMin(&first[page], c < p.whole ? -1 : r);
  }
}

__global__ __launch_bounds__(64) void k_compact_mark(PagesFork f, int* first) {
  const int r = blockIdx.x, n = plan_row(f, r).old;
  for (int c = threadIdx.x; c < n; c += 64) {
    const int page = page_at(f.s, f.table, r, c);
    if (page >= 0) first[page] = -1;
  }
}

// Exclusive prefix sum of one value per thread of a 1024-thread block; *total
// gets the sum.  Every thread calls it.
__device__ __forceinline__ int block_scan(int v, int* total) {
  __shared__ int wsum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) wsum[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w < wave) before += wsum[w];
    all += wsum[w];
  }
  *total = all;
  return before + x - v;
}

// Rows' places in the list of free pages, and the list (one block).
__global__ __launch_bounds__(1024) void k_fork_plan(PagesFork f, const int* first, int* place, int* source, int* list,
                                                    int32_t* info) {
  const int tid = threadIdx.x;
  long want = 0;  // pages wanted by the rows before
  for (int r0 = 0; r0 < f.rows; r0 += 1024) {
    const int r = r0 + tid;
    int n = 0, src = -1;
    if (r < f.rows) {
      const RowPlan p = plan_row(f, r);
      if (p.old > p.whole) {
        src = page_at(f.s, f.table, p.parent, p.whole);
        if (src >= 0 && first[src] == r) src = -1;  // its own
      }
      n = p.pages - p.old + (src >= 0);
    }
    int all;
    const int at = block_scan(n, &all);
    if (r < f.rows) {
      place[r] = clamped(want + at, 0, INT_MAX);
      source[r] = src;
    }
    want += all;
  }
  long free_pages = 0;
  for (int p0 = 0; p0 < f.s.n_pages; p0 += 1024) {
    const int p = p0 + tid, is_free = p < f.s.n_pages && first[p] == INT_MAX;
    int all;
    const int at = block_scan(is_free, &all);
    if (is_free) list[free_pages + at] = p;
    free_pages += all;
  }
  if (tid == 0) {
    info[0] = clamped(free_pages - want, 0, INT_MAX);
    info[1] = clamped(want - free_pages, 0, INT_MAX);
    place[f.rows] = (int)free_pages;
  }
}

// The rows' new table and, block row y > 0, their copied pages: one chunk of a
// page of one layer.
constexpr int kCopyBytes = 16384;

__device__ __forceinline__ void copy_chunk(const PagesShape& s, int8_t* pool, int from, int to, int part) {
  const size_t page = s.page_bytes;
  const int chunks = (int)((page + kCopyBytes - 1) / kCopyBytes), layer = part / chunks, chunk = part % chunks;
  int8_t* base = pool + (size_t)layer * s.n_pages * page + (size_t)chunk * kCopyBytes;
  const int n = (int)min((size_t)kCopyBytes, page - (size_t)chunk * kCopyBytes) / 16;
  const v4i* src = (const v4i*)(base + (size_t)from * page);
  v4i* dst = (v4i*)(base + (size_t)to * page);
  v4i x[kCopyBytes / 16 / 256];
#pragma unroll
  for (int i = 0; i < kCopyBytes / 16 / 256; ++i)
    if (threadIdx.x + 256 * i < n) x[i] = src[threadIdx.x + 256 * i];
#pragma unroll
  for (int i = 0; i < kCopyBytes / 16 / 256; ++i)
    if (threadIdx.x + 256 * i < n) dst[threadIdx.x + 256 * i] = x[i];
}

__global__ __launch_bounds__(256) void k_fork_apply(PagesFork f, const int* place, const int* source, const int* list,
                                                    const int32_t* info, int32_t* table_out, int32_t* len_out) {
  const int r = blockIdx.x, src = source[r], free_pages = place[f.rows];
  int at = place[r];
  if (blockIdx.y > 0) {  // nothing is copied where pages are missing: the input tables still hold
    if (src >= 0 && info[1] == 0) copy_chunk(f.s, f.pool, src, list[at], blockIdx.y - 1);
    return;
  }
  const RowPlan p = plan_row(f, r);
  __syncthreads();  // the row is planned by every wave before its length is written (they may be the same array)
  if (threadIdx.x == 0) len_out[r] = p.len;
  for (int c = threadIdx.x; c < f.s.max_pages; c += 256) {
    int page = -1;
    const bool copied = c == p.whole && src >= 0;
    if (c < p.old && !copied) {
      page = page_at(f.s, f.table, p.parent, c);
    } else if (c < p.pages) {
      const int k = copied ? at : at + (src >= 0) + c - p.old;
      page = k < free_pages ? list[k] : -1;
    }
    table_out[(size_t)r * f.s.max_pages + c] = page;
  }
}

// to[p]: where page p goes.  One block.
__global__ __launch_bounds__(1024) void k_compact_plan(PagesFork f, const int* first, int* to, int* list,
                                                       int32_t* info) {
  const int tid = threadIdx.x, n = f.s.n_pages;
  int live = 0;
  for (int p0 = 0; p0 < n; p0 += 1024) {
    int all;
    block_scan(p0 + tid < n && first[p0 + tid] < 0, &all);
    live += all;
  }
  int holes = 0;
  for (int p0 = 0; p0 < live; p0 += 1024) {
    const int p = p0 + tid, hole = p < live && first[p] >= 0;
    int all;
    const int at = block_scan(hole, &all);
    if (hole) list[holes + at] = p;
    if (p < live) to[p] = p;
    holes += all;
  }
  __syncthreads();
  int moved = 0;
  for (int p0 = live; p0 < n; p0 += 1024) {
    const int p = p0 + tid, high = p < n && first[p] < 0;
    int all;
    const int at = block_scan(high, &all);
    if (p < n) to[p] = high ? list[moved + at] : p;
    moved += all;
  }
  if (tid == 0) {
    info[0] = live;
    info[1] = moved;
  }
}

__global__ __launch_bounds__(256) void k_compact_table(PagesFork f, const int* to, int32_t* table_out) {
  const int r = blockIdx.x, n = plan_row(f, r).old;
  for (int c = threadIdx.x; c < f.s.max_pages; c += 256) {
    const int page = c < n ? page_at(f.s, f.table, r, c) : -1;
    table_out[(size_t)r * f.s.max_pages + c] = page < 0 ? -1 : to[page];
  }
}

__global__ __launch_bounds__(256) void k_compact_move(PagesFork f, const int* to) {
  const int p = blockIdx.x, q = to[p];
  if (q != p) copy_chunk(f.s, f.pool, p, q, blockIdx.y);
}

// Codes of new tokens into their pages: one block per group of 16 tokens and
// row.  Values lie [dh][16] within a group, so a block that has the whole group
// transposes dwords of 16 tokens in registers and stores 64 bytes per thread;
// one that has part of it stores bytes.
__global__ __launch_bounds__(256) void k_pages_write(PagesWrite w) {
  const int r = blockIdx.x;
  int a, n;
  if (w.start) {
    a = clamped(w.start[r], 0, w.n);
    n = clamped(w.start[r + 1], a, w.n) - a;
  } else {
    n = w.n / w.rows;
    a = r * n;
  }
  if (n <= 0) return;
  const long cap = (long)w.s.max_pages << w.s.shift;
  const int len = max(w.len[r], 0), begin = max(len - n, 0);
  const int end = (int)min((long)len, cap);  // (past the table's capacity there is nothing to write to)
  const long off = (long)len - n - a;        // position of token t: t + off
  const int D = w.s.n_kv_heads * w.s.d_head, dh = w.s.d_head;
  const size_t vhalf = w.s.page_bytes / 2;
  for (int g = begin / 16 + blockIdx.y; g * 16L < end; g += gridDim.y) {
    const int page = page_at(w.s, w.table, r, g >> (w.s.shift - 4));
    if (page < 0) continue;
    int8_t* kp = w.pool + (size_t)page * w.s.page_bytes;
    int8_t* vp = kp + vhalf;
    const int lo = max(begin - 16 * g, 0), hi = min(end - 16 * g, 16), g_in = g & ((w.s.page_size >> 4) - 1);
    const long t0 = 16L * g - off;  // token at the group's first place (before the first new one where lo > 0)
    const int cpr = D / 16;
    for (int i = threadIdx.x; i < (hi - lo) * cpr; i += 256) {
      const int t = lo + i / cpr, c = 16 * (i % cpr), head = c / dh;
      *(v4i*)(kp + ((size_t)head * w.s.page_size + 16 * g_in + t) * dh + c % dh) =
          *(const v4i*)(w.k + (t0 + t) * w.ld + c);
    }
    if (hi - lo == 16) {
      for (int i = threadIdx.x; i < D / 4; i += 256) {
        const int c = 4 * i, head = c / dh;
        uint32_t x[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) x[t] = *(const uint32_t*)(w.v + (t0 + t) * w.ld + c);
        uint32_t y[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) transpose4(x + 4 * q, y[0][q], y[1][q], y[2][q], y[3][q]);
        v4i* out = (v4i*)(vp + ((size_t)(head * (w.s.page_size >> 4) + g_in) * dh + c % dh) * 16);
#pragma unroll
        for (int b = 0; b < 4; ++b) out[b] = v4i{(int)y[b][0], (int)y[b][1], (int)y[b][2], (int)y[b][3]};
      }
    } else {
      for (int i = threadIdx.x; i < (hi - lo) * (D / 4); i += 256) {
        const int t = lo + i / (D / 4), c = 4 * (i % (D / 4)), head = c / dh;
        const uint32_t x = *(const uint32_t*)(w.v + (t0 + t) * w.ld + c);
        int8_t* out = vp + ((size_t)(head * (w.s.page_size >> 4) + g_in) * dh + c % dh) * 16 + t;
#pragma unroll
        for (int b = 0; b < 4; ++b) out[16 * b] = (int8_t)(x >> (8 * b));
      }
    }
  }
}

struct PagesWs {
  int *first, *list, *place, *source;
};

PagesWs split_ws(const PagesShape& s, int rows, void* ws) {
  PagesWs w;
  w.first = static_cast<int*>(ws);
  w.list = w.first + s.n_pages;
  w.place = w.list + s.n_pages;
  w.source = w.place + rows + 1;
  return w;
}

int clear_blocks(int n) { return std::min((n + 1023) / 1024, 1024); }

}  // namespace

int pages_copy_parts(const PagesShape& s) {
  return s.n_layers * (int)((s.page_bytes + kCopyBytes - 1) / kCopyBytes);
}

size_t pages_ws_bytes(const PagesShape& s, int rows) {
  return sizeof(int) * (3 * (size_t)s.n_pages + 2 * (size_t)rows + 1);
}

hipError_t launch_pages_fork(const PagesFork& f, int32_t* table_out, int32_t* len_out, int32_t* info, void* ws,
                             hipStream_t s) {
  const PagesWs w = split_ws(f.s, f.rows, ws);
  hipLaunchKernelGGL(k_pages_clear, dim3(clear_blocks(f.s.n_pages)), dim3(256), 0, s, w.first, f.s.n_pages);
  if (f.rows > 0) hipLaunchKernelGGL(k_fork_mark, dim3(f.rows), dim3(64), 0, s, f, w.first);
  hipLaunchKernelGGL(k_fork_plan, dim3(1), dim3(1024), 0, s, f, w.first, w.place, w.source, w.list, info);
  if (f.rows > 0)
    hipLaunchKernelGGL(k_fork_apply, dim3(f.rows, 1 + pages_copy_parts(f.s)), dim3(256), 0, s, f, w.place, w.source,
                       w.list, info, table_out, len_out);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesFork& f, int32_t* table_out, int32_t* info, void* ws, hipStream_t s) {
  const PagesWs w = split_ws(f.s, 0, ws);
  int* to = w.place;
  hipLaunchKernelGGL(k_pages_clear, dim3(clear_blocks(f.s.n_pages)), dim3(256), 0, s, w.first, f.s.n_pages);
  if (f.rows > 0) hipLaunchKernelGGL(k_compact_mark, dim3(f.rows), dim3(64), 0, s, f, w.first);
  hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(1024), 0, s, f, w.first, to, w.list, info);
  if (f.rows == 0) return hipGetLastError();
  hipLaunchKernelGGL(k_compact_table, dim3(f.rows), dim3(256), 0, s, f, to, table_out);
  hipLaunchKernelGGL(k_compact_move, dim3(f.s.n_pages, pages_copy_parts(f.s)), dim3(256), 0, s, f, to);
  return hipGetLastError();
}

hipError_t launch_pages_write(const PagesWrite& w, int max_q, hipStream_t s) {
  const int groups = std::max(1, std::min((max_q + 14) / 16 + 1, 4096));
  hipLaunchKernelGGL(k_pages_write, dim3(w.rows, groups), dim3(256), 0, s, w);
  return hipGetLastError();
}

}  // namespace mnmt
