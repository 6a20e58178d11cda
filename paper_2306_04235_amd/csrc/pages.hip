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

// What the plans know of a page, in `first`: kShared if a row shares it, else the
// lowest row that is to write to it, else kFree.
constexpr int kShared = -1, kFree = INT_MAX;

__global__ __launch_bounds__(256) void k_pages_clear(int* first, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) first[i] = kFree;
}

// Marks an output row's pages; thread `t` of `step`.  Sharing wins whichever
// comes first.
template <class Share, class Write>
__device__ __forceinline__ void mark_row(const PagesFork& f, int r, int t, int step, Share share, Write write) {
  const RowPlan p = plan_row(f, r);
  if (p.parent < 0) return;
  constexpr int U = 4;  // loads under way at once
  for (int c0 = t; c0 < p.old; c0 += U * step) {
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) page[u] = c0 + u * step < p.old ? page_at(f.s, f.table, p.parent, c0 + u * step) : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (page[u] < 0) continue;
      if (c0 + u * step < p.whole)
        share(page[u]);
      else
        write(page[u]);
    }
  }
}

// Rows next to each other often share most of their pages (samples of one
// prompt): a block of 16 rows notes in LDS which of the pages it has marked
// (2048 rows of 63-126 pages, 32 rows to a prompt: 17 us without).
constexpr int kMarkRows = 16, kMarkBits = 1 << 18;

__global__ __launch_bounds__(1024) void k_pages_mark(PagesFork f, int* first) {
  __shared__ uint32_t seen[kMarkBits / 32];
  const int words = f.s.n_pages <= kMarkBits ? (f.s.n_pages + 31) / 32 : 0;
  for (int i = threadIdx.x; i < words; i += 1024) seen[i] = 0;
  __syncthreads();
  const int r = blockIdx.x * kMarkRows + (threadIdx.x >> 6);
  if (r >= f.rows) return;
  mark_row(
      f, r, threadIdx.x & 63, 64,
      [&](int page) {
        const uint32_t bit = 1u << (page & 31);
        if (words == 0 || !(atomicOr(&seen[page >> 5], bit) & bit))
          __hip_atomic_store(&first[page], kShared, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      },
      [&](int page) { atomicMin(&first[page], r); });
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

// take(i, k) for the k-th i in lo..n-1 with is(at(i)), in order; how many there
// are.  A wave has a range of its own and goes over it twice, 256 values at a time
// (at4(i): four from i on, i a multiple of 4): no barrier between the steps.  Every
// thread of a 1024-thread block calls it.
template <class At4, class Is, class Take>
__device__ __forceinline__ int block_list(int lo, int n, At4 at4, Is is, Take take) {
  __shared__ int wsum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, from = lo & ~3;
  const int span = (max(n - from, 0) + 4095) / 4096 * 256, begin = from + wave * span, end = min(begin + span, n);
  const unsigned long long below = (1ull << lane) - 1;
  auto look = [&](int i, bool (&it)[4]) {
    const int at = i + 4 * lane;
    const int4 x = at < end ? at4(at) : make_int4(0, 0, 0, 0);
    it[0] = at >= lo && at < end && is(x.x);
    it[1] = at + 1 >= lo && at + 1 < end && is(x.y);
    it[2] = at + 2 >= lo && at + 2 < end && is(x.z);
    it[3] = at + 3 >= lo && at + 3 < end && is(x.w);
  };
  int count = 0;
#pragma unroll 4
  for (int i = begin; i < end; i += 256) {
    bool it[4];
    look(i, it);
#pragma unroll
    for (int u = 0; u < 4; ++u) count += __popcll(__ballot(it[u]));
  }
  __syncthreads();
  if (lane == 0) wsum[wave] = count;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w < wave) before += wsum[w];
    all += wsum[w];
  }
#pragma unroll 4
  for (int i = begin; i < end; i += 256) {
    bool it[4];
    look(i, it);
    int k = before;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const unsigned long long b = __ballot(it[u]);
      k += __popcll(b & below);
      before += __popcll(b);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (it[u]) take(i + 4 * lane + u, k++);
  }
  return all;
}

// Rows' places in the list of free pages; places[rows + 1]: pages wanted in all.
template <class At>
__device__ __forceinline__ void plan_rows(const PagesFork& f, At at, int* place, int* source) {
  constexpr int U = 4;  // rows of a thread
  long want = 0;        // pages wanted by the rows before
  for (int r0 = 0; r0 < f.rows; r0 += 1024 * U) {
    int n[U], src[U], sum = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + U * threadIdx.x + u;
      n[u] = 0;
      src[u] = -1;
      if (r < f.rows) {
        const RowPlan p = plan_row(f, r);
        if (p.old > p.whole) src[u] = page_at(f.s, f.table, p.parent, p.whole);
        n[u] = p.pages - p.old;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (src[u] >= 0 && at(src[u]) == r0 + U * (int)threadIdx.x + u) src[u] = -1;  // its own
      n[u] += src[u] >= 0;
      sum += n[u];
    }
    int all;
    int k = block_scan(sum, &all);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + U * threadIdx.x + u;
      if (r < f.rows) {
        place[r] = clamped(want + k, 0, INT_MAX);
        source[r] = src[u];
      }
      k += n[u];
    }
    want += all;
  }
  if (threadIdx.x == 0) place[f.rows + 1] = clamped(want, 0, INT_MAX);
}

// The free pages in order; places[rows]: how many there are.
template <class At4>
__device__ __forceinline__ void plan_free(const PagesFork& f, At4 at4, int* place, int* list) {
  const int n = block_list(0, f.s.n_pages, at4, [](int x) { return x == kFree; }, [&](int p, int k) { list[k] = p; });
  if (threadIdx.x == 0) place[f.rows] = n;
}

// to[p]: where page p goes, -1 where it is free; list: the free pages below the
// live pages' count, and from its middle on the pages that move there (one block).
// (As many move as there are free ones below: at most half of all.)
template <class At4>
__device__ __forceinline__ void compact_plan(const PagesFork& f, At4 at4, int* to, int* list, int32_t* info) {
  const int n = f.s.n_pages;
  for (int p = threadIdx.x; p < n; p += 1024) to[p] = -1;
  __syncthreads();
  auto used = [](int x) { return x != kFree; };
  const int live = block_list(0, n, at4, used, [&](int p, int) { to[p] = p; });
  block_list(0, live, at4, [](int x) { return x == kFree; }, [&](int p, int k) { list[k] = p; });
  __syncthreads();
  const int moved = block_list(live, n, at4, used, [&](int p, int k) {
    to[p] = list[k];
    list[n / 2 + k] = p;
  });
  if (threadIdx.x == 0) {
    info[0] = live;
    info[1] = moved;
  }
}

// Block 0: the rows, block 1: the free pages.
__global__ __launch_bounds__(1024) void k_fork_plan(PagesFork f, const int* first, int* place, int* source, int* list) {
  if (blockIdx.x == 0)
    plan_rows(f, [&](int p) { return first[p]; }, place, source);
  else
    plan_free(f, [&](int p) { return *(const int4*)(first + p); }, place, list);
}
__global__ __launch_bounds__(1024) void k_compact_plan(PagesFork f, const int* first, int* to, int* list,
                                                       int32_t* info) {
  compact_plan(f, [&](int p) { return *(const int4*)(first + p); }, to, list, info);
}

// Small caches: marks and plan in one launch, the marks in LDS (512 rows of 6
// entries 6.6 us, bound by the chain parent - length - entry - list).
constexpr int kSmallPages = 12288, kSmallEntries = 32768;

template <bool COMPACT>
__global__ __launch_bounds__(1024) void k_pages_small(PagesFork f, int* place, int* source, int* list, int32_t* info) {
  __shared__ __attribute__((aligned(16))) int first[kSmallPages];
  for (int i = threadIdx.x; i < f.s.n_pages; i += 1024) first[i] = kFree;
  __syncthreads();
  int per = 1;  // threads of a row: all rows at once, if there are so few
  while (per < 64 && 2 * per * f.rows <= 1024) per *= 2;
  for (int r = threadIdx.x / per; r < f.rows; r += 1024 / per)
    mark_row(
        f, r, threadIdx.x % per, per, [&](int page) { first[page] = kShared; },
        [&](int page) { atomicMin(&first[page], r); });
  __syncthreads();
  auto at4 = [&](int p) { return *(const int4*)(first + p); };
  if (COMPACT) {
    compact_plan(f, at4, place, list, info);
  } else {
    plan_rows(f, [&](int p) { return first[p]; }, place, source);
    plan_free(f, at4, place, list);
  }
}

// One chunk of a page of one layer (47 MB of copies in 10.5 us).
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

// The rows' new table and, block row y > 0, their copied pages, chunk after chunk.
__global__ __launch_bounds__(256) void k_fork_apply(PagesFork f, int parts, const int* place, const int* source, const int* list,
                                                    int32_t* table_out, int32_t* len_out, int32_t* info) {
  const int r = blockIdx.x, src = r < f.rows ? source[r] : -1, free_pages = place[f.rows], want = place[f.rows + 1];
  const int at = r < f.rows ? place[r] : 0;
  if (blockIdx.y > 0) {  // nothing is copied where pages are missing: the input tables still hold
    if (src < 0 || want > free_pages) return;
    for (int part = blockIdx.y - 1; part < parts; part += gridDim.y - 1) copy_chunk(f.s, f.pool, src, list[at], part);
    return;
  }
  if (r == 0 && threadIdx.x == 0) {
    info[0] = max(free_pages - want, 0);
    info[1] = max(want - free_pages, 0);
  }
  if (r >= f.rows) return;  // (there are no rows: only the counts)
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

// The table's new numbers, a row to each of the first blocks; the others go over
// the chunks of the pages that move.
__global__ __launch_bounds__(256) void k_compact_apply(PagesFork f, int tables, int parts, const int* to,
                                                       const int* list, const int32_t* info, int32_t* table_out) {
  if ((int)blockIdx.x >= tables) {
    const int moved = info[1], *from = list + f.s.n_pages / 2;
    for (long i = blockIdx.x - tables; i < (long)moved * parts; i += gridDim.x - tables) {
      const int k = (int)(i / parts);
      copy_chunk(f.s, f.pool, from[k], list[k], (int)(i - (long)k * parts));
    }
    return;
  }
  for (int r = blockIdx.x; r < f.rows; r += tables) {
    const int n = plan_row(f, r).old;
    for (int c = threadIdx.x; c < f.s.max_pages; c += 256) {
      const int page = c < n ? page_at(f.s, f.table, r, c) : -1;
      table_out[(size_t)r * f.s.max_pages + c] = page < 0 ? -1 : to[page];
    }
  }
}

// Codes of new tokens into their pages: one block per group of 16 tokens and
// row.  Bound by HBM for chunks (82 MB in 22 us, 16 at a copy's rate: the loads all
// come first, then the stores), by latencies for steps (512 tokens 4.6 us).  Values lie [dh][16] within a group, so a block that has the whole group
// transposes dwords of 16 tokens in registers and stores 64 bytes per thread;
// one that has part of it stores bytes.
__global__ __launch_bounds__(256) void k_pages_write(PagesWrite w) {
  __shared__ v4i turn[4][256];
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
  const int len = clamped(w.len[r], 0, cap), begin = max(len - n, 0);
  const long off = (long)len - n - a;        // position of token t: t + off
  const int D = w.s.n_kv_heads * w.s.d_head, dh = w.s.d_head;
  const size_t vhalf = w.s.page_bytes / 2;
  for (int g = begin / 16 + blockIdx.y; 16 * g < len; g += gridDim.y) {
    const int page = page_at(w.s, w.table, r, g >> (w.s.shift - 4));
    if (page < 0) continue;
    int8_t* kp = w.pool + (size_t)page * w.s.page_bytes;
    int8_t* vp = kp + vhalf;
    const int lo = max(begin - 16 * g, 0), hi = min(len - 16 * g, 16), g_in = g & ((w.s.page_size >> 4) - 1);
    const long t0 = 16L * g - off;  // token at the group's first place (before the first new one where lo > 0)
    const int cpr = D / 16;
    auto key_to = [&](int i) {  // chunk i of the new keys' 16-byte chunks
      const int t = lo + i / cpr, c = 16 * (i % cpr), head = c / dh;
      return (v4i*)(kp + ((size_t)head * w.s.page_size + 16 * g_in + t) * dh + c % dh);
    };
    auto key_from = [&](int i) { return *(const v4i*)(w.k + (t0 + lo + i / cpr) * w.ld + 16 * (i % cpr)); };
    if (hi - lo == 16) {
      // D chunks of keys, four to a thread, beside D / 4 dword columns of
      // values, one to a thread: all loads before the stores.  A thread's four
      // columns pass through LDS, so that a wave stores whole kilobytes.
      for (int base = 0; base < D / 4; base += 256) {
        const int i0 = base + threadIdx.x, lane = threadIdx.x & 63, from = base + (threadIdx.x & ~63);
        const bool mine = i0 < D / 4;
        v4i k[4];
        uint32_t x[16], y[4][4];
        if (mine) {
#pragma unroll
          for (int q = 0; q < 4; ++q) k[q] = key_from(i0 + q * (D / 4));
#pragma unroll
          for (int t = 0; t < 16; ++t) x[t] = *(const uint32_t*)(w.v + (t0 + t) * w.ld + 4 * i0);
#pragma unroll
          for (int q = 0; q < 4; ++q) *key_to(i0 + q * (D / 4)) = k[q];
#pragma unroll
          for (int q = 0; q < 4; ++q) transpose4(x + 4 * q, y[0][q], y[1][q], y[2][q], y[3][q]);
#pragma unroll
          for (int b = 0; b < 4; ++b)  // (places swapped about by lane: no bank conflicts)
            turn[threadIdx.x >> 6][4 * lane + (b ^ (lane >> 1 & 3))] = v4i{(int)y[b][0], (int)y[b][1], (int)y[b][2], (int)y[b][3]};
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = 64 * q + lane, col = 4 * from + c, head = col / dh, at = c >> 2;
          if (col < D)
            *(v4i*)(vp + ((size_t)(head * (w.s.page_size >> 4) + g_in) * dh + col % dh) * 16) =
                turn[threadIdx.x >> 6][4 * at + ((c & 3) ^ (at >> 1 & 3))];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    } else {
      for (int i = threadIdx.x; i < (hi - lo) * cpr; i += 256) *key_to(i) = key_from(i);
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
  w.source = w.place + rows + 2;
  return w;
}

// Blocks that copy: not one to each chunk that there might be, most of which no
// call copies (compaction of 8192 pages of 32 layers and 256 KB, nothing to move: 453
// us with a block to each, 15 without).
constexpr int kCopyBlocks = 65536, kMoveBlocks = 8192;

int clear_blocks(int n) { return std::min((n + 1023) / 1024, 1024); }

}  // namespace

int pages_copy_parts(const PagesShape& s) {
  return s.n_layers * (int)((s.page_bytes + kCopyBytes - 1) / kCopyBytes);
}

size_t pages_ws_bytes(const PagesShape& s, int rows) {
  return sizeof(int) * (3 * (size_t)s.n_pages + 2 * (size_t)rows + 2);
}

// Whether one block marks and plans.  One CU then reads the whole table, which is
// soon done for a beam's (512 rows of 6 entries: 6 us for the launch instead of 12
// for three), but not for long rows of many (2048 of 126).
static bool small_cache(const PagesFork& f) {
  return f.s.n_pages <= kSmallPages && (long)f.rows * f.s.max_pages <= kSmallEntries;
}

static void mark_pages(const PagesFork& f, int* first, hipStream_t s) {
  hipLaunchKernelGGL(k_pages_clear, dim3(clear_blocks(f.s.n_pages)), dim3(256), 0, s, first, f.s.n_pages);
  if (f.rows > 0)
    hipLaunchKernelGGL(k_pages_mark, dim3((f.rows + kMarkRows - 1) / kMarkRows), dim3(1024), 0, s, f, first);
}

hipError_t launch_pages_fork(const PagesFork& f, int32_t* table_out, int32_t* len_out, int32_t* info, void* ws,
                             hipStream_t s) {
  const PagesWs w = split_ws(f.s, f.rows, ws);
  if (small_cache(f)) {
    hipLaunchKernelGGL(k_pages_small<false>, dim3(1), dim3(1024), 0, s, f, w.place, w.source, w.list, info);
  } else {
    mark_pages(f, w.first, s);
    hipLaunchKernelGGL(k_fork_plan, dim3(2), dim3(1024), 0, s, f, w.first, w.place, w.source, w.list);
  }
  const int parts = pages_copy_parts(f.s), rows = std::max(f.rows, 1);
  const int blocks = std::min(parts, std::max(1, kCopyBlocks / rows));  // of a row
  hipLaunchKernelGGL(k_fork_apply, dim3(rows, 1 + blocks), dim3(256), 0, s, f, parts, w.place, w.source, w.list,
                     table_out, len_out, info);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesFork& f, int32_t* table_out, int32_t* info, void* ws, hipStream_t s) {
  const PagesWs w = split_ws(f.s, 0, ws);
  int* to = w.place;
  if (small_cache(f)) {
    hipLaunchKernelGGL(k_pages_small<true>, dim3(1), dim3(1024), 0, s, f, to, nullptr, w.list, info);
  } else {
    mark_pages(f, w.first, s);
    hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(1024), 0, s, f, w.first, to, w.list, info);
  }
  if (f.rows > 0) {
    const int parts = pages_copy_parts(f.s), tables = std::min(f.rows, 1024);
    const int copies = (int)std::min((long)(f.s.n_pages / 2) * parts, (long)kMoveBlocks);
    hipLaunchKernelGGL(k_compact_apply, dim3(tables + copies), dim3(256), 0, s, f, tables, parts, to, w.list, info,
                       table_out);
  }
  return hipGetLastError();
}

hipError_t launch_pages_write(const PagesWrite& w, int max_q, hipStream_t s) {
  const int groups = std::max(1, std::min((max_q + 14) / 16 + 1, 4096));
  hipLaunchKernelGGL(k_pages_write, dim3(w.rows, groups), dim3(256), 0, s, w);
  return hipGetLastError();
}

}  // namespace mnmt
