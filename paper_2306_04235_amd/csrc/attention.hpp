// attention.hpp -- attention of int8 queries over int8 keys and values: the
// kernel that attn_paged.hip and attn_cross.hip compile.
//
// out[q] = c_pv sum_j p_j v_j / sum_j p_j,  p_j = exp(c_qk (q . k_j) - max).
//
// One wave takes 16 queries (token and head pairs of one key head) and 64 keys
// at a time.  The scores are computed transposed, S^T = K Q^T, with the rows of
// K taken in such an order that a lane holds 16 consecutive keys of its query:
// just the operand that the second product, O^T = V^T P^T, wants, so the weights
// never leave their lane.
//
// P V on the int8 matrix cores.  Values are codes already; widening them (to
// f16, say) would cost an instruction per value and half of the matrix rate.
// Instead p becomes a 23-bit fixed-point number, split into three digits of base
// 256 (the lower two in -128..127), each an int8 operand of its own: three
// products with exact int32 sums, joined as 65536 a + 256 b + c.  Adding 2^23 +
// 0x8080 to the scaled p rounds it and leaves the digits in the bytes of the
// float (0x8080 makes the lower digits signed once their top bits are flipped).
// An error of half a unit is 2^-24 of a row's largest weight, so that the
// softmax is fp32 throughout in effect, and the sums do not depend on order.
//
// Scores are taken relative to the largest so far (steps) or of all (chunks), an
// int32 that the products' accumulators start below for nothing.
#pragma once

#include <climits>
#include <type_traits>

#include "blocks.hpp"
#include "cache.hpp"

namespace mnmt {

constexpr int kAttnKeys = 64;         // keys per step of a wave
constexpr int kNoReference = -(1 << 22);  // below every score (|s| <= 127^2 128 < 2^21)
constexpr int kFoldSteps = 1024;      // steps that a chunk's int32 sums hold: 65536 keys * 2^14 < 2^31
constexpr float kOne = 8355711.f;     // the fixed-point 1: 0x7F7F7F, the largest number with digits in range
constexpr float kDigits = 8388608.f + 32896.f;
constexpr uint32_t kDigitBits = 0x4B008080u;  // its bits: p = 0
// The bits of 2^24.  Taken as a float, kScore + d is 2^24 + d for -2^23 <= d <= 0:
// scores' accumulators start there, and need no conversion (a chunk of 301-2048
// tokens over up to 8191 keys 311 -> 302 us).
constexpr int kScore = 0x4B800000;

__device__ __forceinline__ int attn_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ int quad_max(int v) {  // over the four lanes of a query
  uint32_t a, b;
  swap32((uint32_t)v, a, b);
  v = max((int)a, (int)b);
  swap16((uint32_t)v, a, b);
  return max((int)a, (int)b);
}
__device__ __forceinline__ float quad_sum(float v) {
  uint32_t a, b;
  swap32(__float_as_uint(v), a, b);
  v = __uint_as_float(a) + __uint_as_float(b);
  swap16(__float_as_uint(v), a, b);
  return __uint_as_float(a) + __uint_as_float(b);
}

// A row's queries and what they see.
struct AttnRow {
  int first, n;  // its tokens in q
  int len;       // keys
  __device__ __forceinline__ int seen(const AttnArgs& a, int token) const {
    return a.causal ? attn_clamp(len - n + token + 1, 0, len) : len;
  }
};

__device__ __forceinline__ AttnRow attn_row(const AttnArgs& a, int r) {
  AttnRow w;
  if (a.start) {
    w.first = attn_clamp(a.start[r], 0, a.n);
    w.n = attn_clamp(a.start[r + 1], w.first, a.n) - w.first;
  } else {
    w.n = a.n / a.rows;
    w.first = r * w.n;
  }
  w.len = attn_clamp(a.len[r], 0, a.cap);
  return w;
}

// Keys of the last visible position of a tile, and its key ranges that hold any.
__device__ __forceinline__ int tile_keys(const AttnArgs& a, const AttnRow& w, int tile) {
  return w.seen(a, min(w.n - 1, (16 * tile + 15) / a.group));
}
__device__ __forceinline__ int live_splits(const AttnArgs& a, int keys) {
  return min(a.splits, max(1, (keys + a.chunk - 1) / a.chunk));
}
// Place of a tile's key range in the workspace: rows' tiles one after the other,
// whatever the rows' sizes are (row r begins at a token's tile or behind it).
__device__ __forceinline__ size_t tile_slot(const AttnArgs& a, const AttnRow& w, int row, int head, int tile, int split) {
  const size_t slot = (size_t)w.first * a.group / 16 + row + tile;
  return (slot * a.n_kv_heads + head) * a.splits + split;
}

// The k-th row in the order in which blocks take them: the longest first, where
// there are few (a wave compares them), so that no long one is left to the end.
__device__ __forceinline__ int row_in_turn(const AttnArgs& a, int k) {
  if (a.rows > 64) return k;
  const int lane = threadIdx.x & 63, len = lane < a.rows ? attn_clamp(a.len[lane], 0, a.cap) : -1;
  int longer = 0;
  for (int r = 0; r < a.rows; ++r) {
    const int other = __builtin_amdgcn_readlane(len, r);
    longer += other > len || (other == len && r < lane);
  }
  return __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(lane < a.rows && longer == k)) - 1);
}

// Where a lane finds its keys and values: pages, values [token / 16][dh][16].
template <int NB>
struct PagedKeys {
  const AttnArgs& a;
  const int32_t* table;
  size_t koff, voff;
  int last, gk, gv, page_k, page_v;
  // `keys`: where the look-ups end
  __device__ __forceinline__ PagedKeys(const AttnArgs& args, int row, int head, int lane, int keys) : a(args) {
    constexpr int dh = 16 * NB;
    table = a.table + (size_t)row * a.max_pages;
    last = (keys - 1) >> a.shift;
    gk = (lane >> 2) & 3;
    gv = lane >> 4;
    koff = (((size_t)head << a.shift) + (lane & 3)) * dh;
    voff = a.page_bytes / 2 + (((size_t)head << (a.shift - 4)) * dh + (lane & 15)) * 16;
  }
  __device__ __forceinline__ void look(int key) {  // page numbers of the step at `key`
    page_k = table[min((key + 16 * gk) >> a.shift, last)];
    page_v = table[min((key + 16 * gv) >> a.shift, last)];
  }
  __device__ __forceinline__ bool there() const { return (unsigned)page_v < (unsigned)a.n_pages; }
  __device__ __forceinline__ const int8_t* keys_of(int key) const {
    const int page = (unsigned)page_k < (unsigned)a.n_pages ? page_k : 0;
    return a.pool + (size_t)page * a.page_bytes + koff +
           (size_t)((key + 16 * gk) & ((1 << a.shift) - 1)) * (16 * NB);
  }
  __device__ __forceinline__ const int8_t* values_of(int key) const {
    const int page = there() ? page_v : 0;
    return a.pool + (size_t)page * a.page_bytes + voff +
           (size_t)(((key >> 4) + gv) & ((1 << (a.shift - 4)) - 1)) * (16 * NB * 16);
  }
};

// Four columns of query m of a row and key head, from joined sums.
__device__ __forceinline__ void store_joined(const AttnArgs& a, const AttnRow& w, int kv_head, int m, int c, int dh,
                                             float4 y, float sum) {
  const int token = m / a.group;
  if (token >= w.n) return;
  const float inv = sum > 0.f ? a.c_pv / sum : 0.f;
  const size_t o = ((size_t)w.first + token) * a.ldo + (size_t)(kv_head * a.group + m - token * a.group) * dh + c;
  if (a.kind == MNMT_ATTN_F32)
    *(float4*)((float*)a.out + o) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
  else
    *(char4*)((int8_t*)a.out + o) =
        make_char4(code_of(y.x * inv), code_of(y.y * inv), code_of(y.z * inv), code_of(y.w * inv));
}

// The lane's query of a tile.
template <int NB>
struct TileQuery {
  bool real;
  int mine;      // keys it sees
  size_t out;    // its row of q and of out
  int head;
  v4i q[(NB + 3) / 4];
  __device__ __forceinline__ void load(const AttnArgs& a, const AttnRow& w, int kv_head, int tile, int lane) {
    constexpr int dh = 16 * NB;
    const int m = 16 * tile + (lane & 15), token = m / a.group;
    real = token < w.n;
    mine = real ? w.seen(a, token) : INT_MAX;
    out = (size_t)w.first + (real ? token : 0);
    head = kv_head * a.group + (real ? m - token * a.group : 0);
#pragma unroll
    for (int s = 0; s < (NB + 3) / 4; ++s) {
      const int c = 64 * s + 16 * (lane >> 4);
      q[s] = c < dh && real ? *(const v4i*)(a.q + out * a.ldq + (size_t)head * dh + c) : v4i{0, 0, 0, 0};
    }
  }
};

// The lane's largest of a step's scores; d[j][i]: its query and key 4 j + i of its
// 16, of which the first `count` are seen (all where not masked).
__device__ __forceinline__ int largest(v4i (&d)[4], bool masked, int count) {
  if (masked) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int v = 4 * j + i >= count ? INT_MIN / 2 : d[j][i];
        asm volatile("" : "+v"(v));  // (stays in this branch: as a select it would cost every step)
        d[j][i] = v;
      }
  }
  int top = max(max(d[0][0], d[0][1]), d[0][2]);
  top = max(top, d[0][3]);
#pragma unroll
  for (int j = 1; j < 4; ++j) {
    top = max(max(top, d[j][0]), d[j][1]);
    top = max(max(top, d[j][2]), d[j][3]);
  }
  return top;
}

// Exponents c2 d of kScore + d (one rounding: 2^24 c2 is exact), and -inf in the
// place of those of masked keys.
__device__ __forceinline__ void exponents(const v4i (&d)[4], float c2, float (&x)[4][4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[j][i] = fmaf(__int_as_float(d[j][i]), c2, -16777216.f * c2);
}
__device__ __forceinline__ void hide(int count, float (&x)[4][4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[j][i] = 4 * j + i >= count ? -__builtin_inff() : x[j][i];
      asm volatile("" : "+v"(x[j][i]));  // (as above)
    }
}

// Digits of the weights 2^x; returns the weights' sum.
__device__ __forceinline__ float digits(const float (&x)[4][4], v4i (&p)[3]) {
  uint32_t total = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = __float_as_uint(fmaf(__builtin_amdgcn_exp2f(x[j][i]), kOne, kDigits));
      total += u[i];
    }
    const uint32_t lo0 = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), lo1 = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);
    const uint32_t hi0 = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0602u), hi1 = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0602u);
    p[0][j] = (int)__builtin_amdgcn_perm(hi1, hi0, 0x05040100u);
    p[1][j] = (int)(__builtin_amdgcn_perm(lo1, lo0, 0x07060302u) ^ 0x80808080u);
    p[2][j] = (int)(__builtin_amdgcn_perm(lo1, lo0, 0x05040100u) ^ 0x80808080u);
  }
  return (float)(total - 16u * kDigitBits);
}

// The sums of a query tile: columns 16 b + 4 (lane / 16) + i of query lane % 16,
// relative to the weight of score ref.
template <int NB>
struct TileSums {
  float f[NB][4], sum;
  int ref;

  __device__ __forceinline__ TileSums() : sum(0.f), ref(kNoReference) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) f[b][i] = 0.f;
  }
  // f scale + the digits' products a, b, c
  __device__ __forceinline__ void fold(int block, float scale, v4i a, v4i b, v4i c) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      f[block][i] = fmaf(65536.f, (float)a[i], fmaf(256.f, (float)b[i], fmaf(f[block][i], scale, (float)c[i])));
  }
  // After the last step: the query's outputs, or its partial result [16][dh], sums [16], references [16].
  __device__ __forceinline__ void store(const AttnArgs& a, const TileQuery<NB>& t, int lane) const {
    if (!t.real) return;
    const float inv = sum > 0.f ? a.c_pv / sum : 0.f;
    const size_t o = t.out * a.ldo + (size_t)t.head * (16 * NB) + 4 * (lane >> 4);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const float x0 = f[b][0] * inv, x1 = f[b][1] * inv, x2 = f[b][2] * inv, x3 = f[b][3] * inv;
      if (a.kind == MNMT_ATTN_F32)
        *(float4*)((float*)a.out + o + 16 * b) = make_float4(x0, x1, x2, x3);
      else
        *(char4*)((int8_t*)a.out + o + 16 * b) = make_char4(code_of(x0), code_of(x1), code_of(x2), code_of(x3));
    }
  }
  __device__ __forceinline__ void store_part(float* part, int lane) const {
    constexpr int dh = 16 * NB;
    const int col = lane & 15, g = lane >> 4;
    if (g == 0) {
      part[16 * dh + col] = sum;
      part[16 * dh + 16 + col] = (float)ref;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
      *(float4*)(part + col * dh + 16 * b + 4 * g) = make_float4(f[b][0], f[b][1], f[b][2], f[b][3]);
  }
};

// One query tile per wave (WK 1) or per block, whose four waves take turns at
// the keys (WK 4).  For few queries per row: every wave loads its keys and
// values straight into the matrix operands.  SHORT: rows of one or two steps, where
// more waves at once are worth more than keys a step ahead.  Long rows are bound by
// HBM (16 rows, 32 heads on 8 key heads of 128, 2824-30176 keys: 541 MB in 110 us,
// 4.9 TB/s, of 5.2 that a read reaches), short ones by the latencies of length,
// page, keys and store one after the other (512 rows of 8 heads of 64, 20-80 keys:
// 10 us for 27 MB).  Folding the sums in every step is free in the first and takes
// no registers between steps; the integer sums would need 96 for heads of 128.
template <int NB, bool PAGED, int WK, bool SHORT>
__global__ __launch_bounds__(256, !SHORT ? 2 : NB <= 4 ? 4 : 3) void k_attn(AttnArgs a) {
  constexpr int dh = 16 * NB, KS = (NB + 3) / 4;  // 64-wide slices of the head
  constexpr int kStage = PAGED ? 0 : NB * 1024;   // a wave's values, transposed
  constexpr int kJoin = WK == 1 ? 0 : 16 * (dh + 4) * 4 + 128;
  constexpr int kWave = kStage > kJoin ? kStage : kJoin;
  __shared__ __attribute__((aligned(16))) int8_t lds[kWave ? 4 * kWave : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int unit = WK == 1 ? 4 * blockIdx.x + wave : blockIdx.x;
  const int per_head = a.tiles * a.splits, per_row = per_head * a.n_kv_heads;
  const int row = unit / per_row, head = unit % per_row / per_head;
  if (row >= a.rows) return;
  const int split = unit % per_head / a.tiles, tile0 = a.tiles - 1 - unit % a.tiles;
  const AttnRow w = attn_row(a, row);
  for (int tile = tile0; 16 * tile < w.n * a.group; tile += a.tiles) {
    const int keys = tile_keys(a, w, tile), live = live_splits(a, keys);
    if (split >= live) continue;
    const int kbegin = split * a.chunk, kend = split == live - 1 ? keys : kbegin + a.chunk;
    const int all_see = min(w.seen(a, 16 * tile / a.group), kend);  // keys that every query of the tile sees
    TileQuery<NB> t;
    t.load(a, w, head, tile, lane);
    TileSums<NB> y;
    // key rows of the lane in a step: 16 (l / 4 mod 4) + 4 j + l mod 4; slices past the head read its first bytes (their queries are 0)
    int slice[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) slice[s] = 64 * s + 16 * g < dh ? 64 * s + 16 * g : 0;
    // (a short row's look-ups do not wait for its length: what lies behind it may be
    // any number, and is hidden)
    PagedKeys<NB> at(a, PAGED ? row : 0, head, lane, SHORT ? a.cap : kend);
    const int8_t* kbase = PAGED ? nullptr : a.k + (size_t)row * a.batch + (size_t)head * dh;
    const int8_t* vbase = PAGED ? nullptr : a.v + (size_t)row * a.batch + (size_t)head * dh;
    int8_t* stage = lds + wave * kWave;
    int key = kbegin + (WK == 1 ? 0 : kAttnKeys * wave);
    v4i kf[4][KS], vf[NB];
    bool there = true;
    auto load_keys = [&](int key) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int8_t* kp;
        if constexpr (PAGED)
          kp = at.keys_of(key) + 4 * j * dh;
        else
          kp = kbase + (size_t)min(key + 16 * ((lane >> 2) & 3) + 4 * j + (lane & 3), kend - 1) * a.ld;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[j][s] = *(const v4i*)(kp + slice[s]);
      }
    };
    v4i vr[PAGED ? 1 : 4][KS];  // an encoder's values: 4 keys (4 (l mod 16) ..) and 16 columns of each slice
    auto load_values = [&](int key) {
      if constexpr (PAGED) {
        const int8_t* vp = at.values_of(key);
        there = at.there();
#pragma unroll
        for (int b = 0; b < NB; ++b) vf[b] = *(const v4i*)(vp + 256 * b);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int8_t* vp = vbase + (size_t)min(key + 4 * col + i, kend - 1) * a.ld;
#pragma unroll
          for (int s = 0; s < KS; ++s) vr[i][s] = *(const v4i*)(vp + slice[s]);
        }
      }
    };
    if (PAGED && (SHORT || key < kend)) at.look(key);
    if (!SHORT && key < kend) {
      load_keys(key);
      load_values(key);
      if constexpr (PAGED) at.look(min(key + kAttnKeys * WK, kend - 1));
    }
    for (; key < kend; key += kAttnKeys * WK) {
      const bool more = key + kAttnKeys * WK < kend;
      if (SHORT) {
        load_keys(key);
        load_values(key);
        if (PAGED && more) at.look(key + kAttnKeys * WK);
      }
      // scores less the reference: the lane's query, keys key + 16 g + 4 j + i
      v4i d[4], p[3];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] = mfma16(kf[j][0], t.q[0], v4i{kScore - y.ref, kScore - y.ref, kScore - y.ref, kScore - y.ref});
#pragma unroll
        for (int s = 1; s < KS; ++s) d[j] = mfma16(kf[j][s], t.q[s], d[j]);
      }
      // the next step's keys take these registers while this step's weights are
      // computed, its values the values' while the next scores are
      if (!SHORT && more) load_keys(key + kAttnKeys * WK);
      const bool masked = key + kAttnKeys > all_see || __any(!there);
      const int count = there ? min(t.mine, kend) - key - 16 * g : 0;
      const int up = max(quad_max(largest(d, masked, count)) - kScore, 0);
      const float scale = __builtin_amdgcn_exp2f(-(float)up * a.c2);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[j][i] -= up;  // (masked places stay far below)
      float x[4][4];
      exponents(d, a.c2, x);
      if (masked) hide(count, x);
      y.sum = fmaf(y.sum, scale, digits(x, p));
      y.ref += up;
      if constexpr (!PAGED) {
        // dwords of 4 keys go to LDS, chunks of 16 keys swapped about by column so
        // that neither side meets bank conflicts
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (64 * s + 16 * g < dh) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t x[4] = {(uint32_t)vr[0][s][c], (uint32_t)vr[1][s][c], (uint32_t)vr[2][s][c],
                                     (uint32_t)vr[3][s][c]};
              uint32_t z[4];
              transpose4(x, z[0], z[1], z[2], z[3]);
              // column 64 s + 16 g + 4 c + b: chunk (col / 4) ^ c ^ g
#pragma unroll
              for (int b = 0; b < 4; ++b)
                *(uint32_t*)(stage + (64 * s + 16 * g + 4 * c + b) * 64 + 16 * ((col >> 2) ^ c ^ g) + 4 * (col & 3)) = z[b];
            }
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int b = 0; b < NB; ++b)  // column 16 b + col: its c is col / 4, its g is b mod 4
          vf[b] = *(const v4i*)(stage + (16 * b + col) * 64 + 16 * (g ^ (col >> 2) ^ (b & 3)));
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const v4i none{0, 0, 0, 0};
        y.fold(b, scale, mfma16(vf[b], p[0], none), mfma16(vf[b], p[1], none), mfma16(vf[b], p[2], none));
      }
      if (!SHORT && more) {
        load_values(key + kAttnKeys * WK);
        if constexpr (PAGED) at.look(min(key + 2 * kAttnKeys * WK, kend - 1));
      }
    }
    y.sum = quad_sum(y.sum);
    if constexpr (WK == 1) {
      if (live == 1)
        y.store(a, t, lane);
      else
        y.store_part(a.part + tile_slot(a, w, row, head, tile, split) * (16 * (dh + 2)), lane);
    } else {
      // join the four waves' sums, each relative to its own reference
      float* mine_f = (float*)(lds + wave * kWave);
      if (g == 0) {
        mine_f[col] = y.sum;
        mine_f[16 + col] = (float)y.ref;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *(float4*)(mine_f + 32 + col * (dh + 4) + 16 * b + 4 * g) = make_float4(y.f[b][0], y.f[b][1], y.f[b][2], y.f[b][3]);
      __syncthreads();
      float* part = a.part + tile_slot(a, w, row, head, tile, split) * (16 * (dh + 2));
      for (int i = threadIdx.x; i < 16 * dh / 4; i += 256) {
        const int q = i / (dh / 4), c = 4 * (i % (dh / 4));
        float top = (float)kNoReference, wsum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int v = 0; v < 4; ++v) top = fmaxf(top, ((const float*)(lds + v * kWave))[16 + q]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float* src = (const float*)(lds + v * kWave);
          const float scale = __builtin_amdgcn_exp2f((src[16 + q] - top) * a.c2);
          const float4 x = *(const float4*)(src + 32 + q * (dh + 4) + c);
          wsum = fmaf(scale, src[q], wsum);
          o.x = fmaf(scale, x.x, o.x);
          o.y = fmaf(scale, x.y, o.y);
          o.z = fmaf(scale, x.z, o.z);
          o.w = fmaf(scale, x.w, o.w);
        }
        if (live == 1) {
          store_joined(a, w, head, 16 * tile + q, c, dh, o, wsum);
        } else if ((16 * tile + q) / a.group < w.n) {
          if (c == 0) {
            part[16 * dh + q] = wsum;
            part[16 * dh + 16 + q] = top;
          }
          *(float4*)(part + q * dh + c) = o;
        }
      }
      __syncthreads();
    }
  }
}

// The largest score of each query of eight tiles over a range of keys: the waves
// take turns at the keys, straight from memory, one step ahead in registers, each
// step against all of the block's queries.  Bound by what the L2s deliver: blocks
// of 2, 4 and 8 tiles take 172, 99 and 73 us (1699 queries of 16 heads over 6853
// keys, heads of 128, and three shorter rows).
constexpr int kTopTiles = 8;  // (their queries stay in registers)

template <int NB, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_attn_top(AttnArgs a) {
  constexpr int dh = 16 * NB, KS = (NB + 3) / 4, kStride = 4 * kAttnKeys;
  __shared__ int tops[4 * kTopTiles * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int groups = a.tiles / kTopTiles, per_head = groups * a.splits, per_row = per_head * a.n_kv_heads;
  const int row = row_in_turn(a, blockIdx.x / per_row), head = blockIdx.x % per_row / per_head;
  const int split = blockIdx.x % per_head / groups, group0 = groups - 1 - blockIdx.x % groups;
  const AttnRow w = attn_row(a, row);
  const int tiles = (w.n * a.group + 15) / 16;
  int slice[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) slice[s] = 64 * s + 16 * g < dh ? 64 * s + 16 * g : 0;
  for (int group = group0; kTopTiles * group < tiles; group += groups) {
    const int tile = kTopTiles * group;
    // (the chunk kernel's ranges: by its blocks' last tiles, which see no more than this block's)
    const int keys = tile_keys(a, w, min(tile + kTopTiles, tiles) - 1), live = live_splits(a, keys);
    if (split >= live) continue;
    const int kbegin = split * a.chunk, kend = split == live - 1 ? keys : kbegin + a.chunk;
    const int all_see = min(w.seen(a, 16 * tile / a.group), kend);
    v4i q[kTopTiles][KS];
    int seen[kTopTiles], top[kTopTiles];
#pragma unroll
    for (int x = 0; x < kTopTiles; ++x) {
      TileQuery<NB> t;
      t.load(a, w, head, min(tile + x, tiles), lane);
#pragma unroll
      for (int s = 0; s < KS; ++s) q[x][s] = t.q[s];
      seen[x] = min(t.mine, kend);
      top[x] = kNoReference;
    }
    PagedKeys<NB> at(a, PAGED ? row : 0, head, lane, kend);
    const int8_t* kbase = PAGED ? nullptr : a.k + (size_t)row * a.batch + (size_t)head * dh;
    v4i k[4][KS];
    bool there = true;
    auto look = [&](int key) {
      if constexpr (PAGED) at.look(min(key, kend - 1));
    };
    auto load = [&](int key) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int8_t* kp;
        if constexpr (PAGED)
          kp = at.keys_of(key) + 4 * j * dh;
        else
          kp = kbase + (size_t)min(key + 16 * ((lane >> 2) & 3) + 4 * j + (lane & 3), kend - 1) * a.ld;
#pragma unroll
        for (int s = 0; s < KS; ++s) k[j][s] = *(const v4i*)(kp + slice[s]);
      }
      if constexpr (PAGED) there = at.there();
    };
    int key = kbegin + kAttnKeys * wave;
    if (key < kend) {
      look(key);
      load(key);
      look(key + kStride);
    }
    while (key < kend) {
      v4i kc[4][KS];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int s = 0; s < KS; ++s) kc[j][s] = k[j][s];
      const bool here = there, masked = key + kAttnKeys > all_see || __any(!here);
      const int now = key;
      key += kStride;
      if (key < kend) {
        load(key);
        look(key + kStride);
      }
      auto tiles_of = [&](auto hidden) {
#pragma unroll
        for (int x = 0; x < kTopTiles; ++x) {
          v4i d[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            d[j] = mfma16(kc[j][0], q[x][0], v4i{0, 0, 0, 0});
#pragma unroll
            for (int s = 1; s < KS; ++s) d[j] = mfma16(kc[j][s], q[x][s], d[j]);
          }
          top[x] = max(top[x], largest(d, hidden, here ? seen[x] - now - 16 * g : 0));
        }
      };
      if (masked)
        tiles_of(std::true_type{});
      else
        tiles_of(std::false_type{});
    }
#pragma unroll
    for (int x = 0; x < kTopTiles; ++x) {
      const int m = quad_max(top[x]);
      if (g == 0) tops[(wave * kTopTiles + x) * 16 + lane] = m;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTopTiles * 16; i += 256) {
      int m = tops[i];
#pragma unroll
      for (int v = 1; v < 4; ++v) m = max(m, tops[v * kTopTiles * 16 + i]);
      if (tile + i / 16 < tiles) a.tops[tile_slot(a, w, row, head, tile + i / 16, split) * 16 + i % 16] = m;
    }
    __syncthreads();
  }
}

// The query tiles of a block's waves, over the same keys: 64 of them at a time pass
// through LDS, in the order of the matrix operands (a kilobyte per operand, lane
// by lane), so that a block reads them once.  A wave has two tiles where its
// registers hold their sums at two waves per SIMD (heads of up to 64), and reads
// each operand for both.  Keys, and the values of pages, come in by loads straight
// to LDS, one step ahead; an encoder's values are transposed on the way, each wave
// those of its 16 keys.  (Eight waves to a block of wide heads read half as much
// and are slower, 293 against 260 us in the case above: more of them wait for the
// slowest.)
//
// The references are the scores' maxima, from k_attn_top: they never move, so that
// the sums are integers throughout and no step branches.  Bound by the vector unit
// and the matrix cores, which overlap in part: per 16 queries and 64 keys of a head
// of 128, 32 products of 16 cycles beside 134 instructions of 4 (exponentials 16,
// digits 36), 1300-1600 cycles in all.
constexpr int chunk_tiles(int nb) { return nb <= 4 ? 2 : 1; }  // of a wave
constexpr int kChunkWaves = 4;
constexpr int kValueGap = 16;  // between values' operands: the transposing stores meet no bank conflicts

__device__ __forceinline__ void load_to_lds(const int8_t* from, int8_t* to) {  // 16 bytes per lane, to + 16 lane
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Waits for the wave's loads to LDS, then for the block's other waves.
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// LONG: ranges may hold more keys than the int32 sums (kFoldSteps); without it no
// register holds sums in fp32 meanwhile.
template <int NB, bool PAGED, bool LONG>
__global__ __launch_bounds__(64 * kChunkWaves, 2) void k_attn_chunk(AttnArgs a) {
  constexpr int dh = 16 * NB, KS = (NB + 3) / 4, QT = chunk_tiles(NB), W = kChunkWaves, kTiles = W * QT;
  constexpr int kKeyBytes = 4 * KS * 1024, kValueBytes = NB * (1024 + kValueGap);
  __shared__ __attribute__((aligned(16))) int8_t kbuf[2 * kKeyBytes], vbuf[3 * kValueBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4;
  // blocks of one row and head side by side, so that the L2s hold what they read,
  // the last tiles first (in a causal chunk they see most)
  const int groups = a.tiles / kTiles, per_head = groups * a.splits, per_row = per_head * a.n_kv_heads;
  const int row = row_in_turn(a, blockIdx.x / per_row), head = blockIdx.x % per_row / per_head;
  const int split = blockIdx.x % per_head / groups, group0 = groups - 1 - blockIdx.x % groups;
  const AttnRow w = attn_row(a, row);
  const int tiles = (w.n * a.group + 15) / 16;
  int slice[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) slice[s] = 64 * s + 16 * g < dh ? 64 * s + 16 * g : 0;
  for (int group = group0; kTiles * group < tiles; group += groups) {
    // ranges of keys by the block's last tile; a tile that sees fewer keys has nothing in the last ones
    const int tile = kTiles * group + QT * wave;
    const int block_keys = tile_keys(a, w, min(kTiles * (group + 1), tiles) - 1);
    const int live = live_splits(a, block_keys);
    if (split >= live) continue;
    const int kbegin = split * a.chunk, kend = split == live - 1 ? block_keys : kbegin + a.chunk;
    // the keys that every query of the wave's tiles sees
    const int all_see = tile < tiles ? min(w.seen(a, 16 * tile / a.group), kend) : 0;
    TileQuery<NB> t[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) t[x].load(a, w, head, min(tile + x, tiles), lane);
    TileSums<NB> y[QT];
    PagedKeys<NB> at(a, PAGED ? row : 0, head, lane, kend);
    const int8_t* kbase = PAGED ? nullptr : a.k + (size_t)row * a.batch + (size_t)head * dh;
    const int8_t* vbase = PAGED ? nullptr : a.v + (size_t)row * a.batch + (size_t)head * dh;
    const int dc = lane >> 2, kg = lane & 3;  // transposing: 16 columns, 4 keys of the wave's 16
    const bool transposes = dc < NB;
    v4i vr[4];
    bool there = true, next_there = true;
    auto fetch_keys = [&](int key, int8_t* buf) {  // operand (j, s) of keys 16 (l / 4 mod 4) + 4 j + l mod 4
      const int8_t* kp;
      if constexpr (PAGED) {
        kp = at.keys_of(key) + 4 * wave * dh;
        next_there = at.there();
      } else {
        kp = kbase + (size_t)min(key + 16 * ((lane >> 2) & 3) + 4 * wave + (lane & 3), kend - 1) * a.ld;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) load_to_lds(kp + slice[s], buf + (wave * KS + s) * 1024);
    };
    auto fetch_values = [&](int key, int8_t* buf) {
      if constexpr (PAGED) {
        const int8_t* vp = at.values_of(key);
#pragma unroll
        for (int b = 0; b < NB; b += W)
          if (b + wave < NB) load_to_lds(vp + 256 * (b + wave), buf + (b + wave) * (1024 + kValueGap));
      } else if (transposes) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vr[i] = *(const v4i*)(vbase + (size_t)min(key + 16 * wave + 4 * kg + i, kend - 1) * a.ld + 16 * dc);
      }
    };
    auto transpose = [&](int8_t* buf) {  // the values that fetch_values left in registers
      if constexpr (!PAGED) {
        if (transposes) {
          uint32_t* to = (uint32_t*)(buf + dc * (1024 + kValueGap) + 256 * wave) + kg;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t x[4] = {(uint32_t)vr[0][c], (uint32_t)vr[1][c], (uint32_t)vr[2][c], (uint32_t)vr[3][c]};
            uint32_t z[4];
            transpose4(x, z[0], z[1], z[2], z[3]);
#pragma unroll
            for (int b = 0; b < 4; ++b) to[4 * (4 * c + b)] = z[b];
          }
        }
      }
    };
    auto look = [&](int key) {
      if constexpr (PAGED) at.look(min(key, kend - 1));
    };
    auto scores = [&](const int8_t* buf, v4i (&d)[QT][4], const int (&from)[QT]) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v4i k[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) k[s] = *(const v4i*)(buf + (j * KS + s) * 1024 + 16 * lane);
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          d[x][j] = mfma16(k[0], t[x].q[0], v4i{from[x], from[x], from[x], from[x]});
#pragma unroll
          for (int s = 1; s < KS; ++s) d[x][j] = mfma16(k[s], t[x].q[s], d[x][j]);
        }
      }
    };
    __syncthreads();  // (the last group's reads of LDS are over)
    if (kbegin < kend) {
      int from[QT], cur = 0;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        y[x].ref =
            tile + x < tiles ? a.tops[tile_slot(a, w, row, head, tile + x, split) * 16 + (lane & 15)] : kNoReference;
        from[x] = kScore - y[x].ref;
      }
      // the weights of a step, and the products of the step before, which need
      // nothing of it: the matrix and the vector unit work side by side
      look(kbegin);
      fetch_keys(kbegin, kbuf);
      fetch_values(kbegin, vbuf);
      look(kbegin + kAttnKeys);
      transpose(vbuf);
      v4i acc[QT][3][NB], p[QT][3];
      int8_t *v_prev = vbuf + 2 * kValueBytes, *v_cur = vbuf, *v_next = vbuf + kValueBytes;
      auto values = [&](v4i (&v)[NB]) {
#pragma unroll
        for (int b = 0; b < NB; ++b) v[b] = *(const v4i*)(v_prev + b * (1024 + kValueGap) + 16 * lane);
      };
      auto products = [&](const v4i (&v)[NB]) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < QT; ++x)
#pragma unroll
            for (int i = 0; i < 3; ++i) acc[x][i][b] = mfma16(v[b], p[x][i], acc[x][i][b]);
      };
      int key = kbegin;
      do {
        const int pend = LONG ? min(kend - key, kAttnKeys * kFoldSteps) + key : kend;
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            p[x][i] = v4i{0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < NB; ++b) acc[x][i][b] = v4i{0, 0, 0, 0};
          }
        for (; key < pend; key += kAttnKeys, cur ^= 1) {
          there = next_there;
          landed();
          const bool more = key + kAttnKeys < kend;
          v4i d[QT][4], v[NB];
          float x[QT][4][4];
          scores(kbuf + cur * kKeyBytes, d, from);
          values(v);
          // nothing is read from LDS between here and the next step: a read would
          // wait for these loads
          if (more) {
            fetch_keys(key + kAttnKeys, kbuf + (cur ^ 1) * kKeyBytes);
            fetch_values(key + kAttnKeys, v_next);
            look(key + 2 * kAttnKeys);
          }
          const bool masked = key + kAttnKeys > all_see || __any(!there);
#pragma unroll
          for (int i = 0; i < QT; ++i) exponents(d[i], a.c2, x[i]);
          if (masked) {
#pragma unroll
            for (int i = 0; i < QT; ++i) hide(there ? min(t[i].mine, kend) - key - 16 * g : 0, x[i]);
          }
          __builtin_amdgcn_sched_barrier(0);
          v4i p_new[QT][3];
          products(v);
#pragma unroll
          for (int i = 0; i < QT; ++i) y[i].sum += digits(x[i], p_new[i]);
          // one matrix instruction, then its share of the others
#pragma unroll
          for (int i = 0; i < 3 * NB * QT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, (27 + NB - 1) / NB, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < QT; ++i)
#pragma unroll
            for (int j = 0; j < 3; ++j) p[i][j] = p_new[i][j];
          if (more) transpose(v_next);
          int8_t* const v_old = v_prev;
          v_prev = v_cur;
          v_cur = v_next;
          v_next = v_old;
        }
        v4i v[NB];
        values(v);
        products(v);
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int b = 0; b < NB; ++b) y[i].fold(b, 1.f, acc[i][0][b], acc[i][1][b], acc[i][2][b]);
      } while (LONG && key < kend);
    }
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      if (tile + x >= tiles) break;
      y[x].sum = quad_sum(y[x].sum);
      if (live == 1)
        y[x].store(a, t[x], lane);
      else
        y[x].store_part(a.part + tile_slot(a, w, row, head, tile + x, split) * (16 * (dh + 2)), lane);
    }
  }
}

// Joins the key ranges of a query tile.  A thread takes four columns of a query;
// where there are many ranges, kParts threads take every kParts-th of them, eight
// at once, and the first of them then joins theirs.
constexpr int kManySplits = 8;

template <int NB, bool MANY>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  constexpr int dh = 16 * NB, kPart = 16 * (dh + 2), U = 8;
  constexpr int kCols = dh / 4, kParts = !MANY ? 1 : 256 / kCols < 16 ? 256 / kCols : 16;
  constexpr int kQueries = 256 / (kCols * kParts) < 16 ? 256 / (kCols * kParts) : 16;  // of a block at once
  __shared__ float4 ys[MANY ? 256 : 1];
  __shared__ float tops[MANY ? 256 : 1], sums[MANY ? 256 : 1];
  const int per_row = a.n_kv_heads * a.tiles;
  const int row = blockIdx.x / per_row, head = blockIdx.x % per_row / a.tiles;
  const int slot = threadIdx.x / (kCols * kParts), mine = threadIdx.x / kCols % kParts, col = threadIdx.x % kCols;
  const AttnRow w = attn_row(a, row);
  for (int tile = blockIdx.x % a.tiles; 16 * tile < w.n * a.group; tile += a.tiles) {
    // a chunk's ranges go by its block's last tile
    const int span = a.waves == 0 ? kChunkWaves * chunk_tiles(NB) : 1, last = (w.n * a.group + 15) / 16 - 1;
    const int live = live_splits(a, tile_keys(a, w, min(tile / span * span + span - 1, last)));
    if (live == 1) continue;
    const float* part = a.part + tile_slot(a, w, row, head, tile, 0) * kPart;
    const int queries = min(16, w.n * a.group - 16 * tile);
    for (int q0 = blockIdx.y * kQueries; q0 < queries; q0 += gridDim.y * kQueries) {
      const int q = q0 + slot;
      const bool active = slot < kQueries && q < queries;
      float top = (float)kNoReference, sum = 0.f;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
      auto join = [&](float ref, float s, float4 x) {
        const float best = fmaxf(top, ref);
        const float old = __builtin_amdgcn_exp2f((top - best) * a.c2), now = __builtin_amdgcn_exp2f((ref - best) * a.c2);
        top = best;
        sum = fmaf(sum, old, s * now);
        y = make_float4(fmaf(y.x, old, x.x * now), fmaf(y.y, old, x.y * now), fmaf(y.z, old, x.z * now),
                        fmaf(y.w, old, x.w * now));
      };
      if (active) {
        for (int s0 = mine; s0 < live; s0 += U * kParts) {
          float s[U], ref[U];
          float4 x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (s0 + u * kParts >= a.splits) break;
            const float* src = part + (size_t)(s0 + u * kParts) * kPart;
            s[u] = src[16 * dh + q];
            ref[u] = src[16 * dh + 16 + q];
            x[u] = *(const float4*)(src + q * dh + 4 * col);
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (s0 + u * kParts < live) join(ref[u], s[u], x[u]);
        }
      }
      if constexpr (MANY) {
        ys[threadIdx.x] = y;
        tops[threadIdx.x] = top;
        sums[threadIdx.x] = sum;
        __syncthreads();
        if (active && mine == 0) {
#pragma unroll
          for (int p = 1; p < kParts; ++p)
            join(tops[threadIdx.x + p * kCols], sums[threadIdx.x + p * kCols], ys[threadIdx.x + p * kCols]);
        }
        __syncthreads();
      }
      if (active && mine == 0) store_joined(a, w, head, 16 * tile + q, 4 * col, dh, y, sum);
    }
  }
}

template <int NB, bool PAGED>
hipError_t launch_attn_nb(const AttnArgs& a, hipStream_t s) {
  const int tiles = a.rows * a.n_kv_heads * a.tiles, units = tiles * a.splits;
  if (a.waves == 0)
    hipLaunchKernelGGL((k_attn_top<NB, PAGED>), dim3(a.rows * a.n_kv_heads * (a.tiles / kTopTiles) * a.splits),
                       dim3(256), 0, s, a);
  const dim3 chunks(a.rows * a.n_kv_heads * (a.tiles / (kChunkWaves * chunk_tiles(NB))) * a.splits);
  if (a.waves == 0 && a.cap <= kAttnKeys * kFoldSteps)
    hipLaunchKernelGGL((k_attn_chunk<NB, PAGED, false>), chunks, dim3(64 * kChunkWaves), 0, s, a);
  else if (a.waves == 0)
    hipLaunchKernelGGL((k_attn_chunk<NB, PAGED, true>), chunks, dim3(64 * kChunkWaves), 0, s, a);
  else if (a.waves == 1 && a.is_short)
    hipLaunchKernelGGL((k_attn<NB, PAGED, 1, true>), dim3((units + 3) / 4), dim3(256), 0, s, a);
  else if (a.waves == 1)
    hipLaunchKernelGGL((k_attn<NB, PAGED, 1, false>), dim3((units + 3) / 4), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_attn<NB, PAGED, 4, false>), dim3(units), dim3(256), 0, s, a);
  if (a.splits > kManySplits)
    hipLaunchKernelGGL((k_attn_join<NB, true>), dim3(tiles, a.queries), dim3(256), 0, s, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL((k_attn_join<NB, false>), dim3(tiles), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <bool PAGED>
hipError_t launch_attn_kernel(const AttnArgs& a, int d_head, hipStream_t s) {
  switch (d_head) {
    case 16: return launch_attn_nb<1, PAGED>(a, s);
    case 32: return launch_attn_nb<2, PAGED>(a, s);
    case 48: return launch_attn_nb<3, PAGED>(a, s);
    case 64: return launch_attn_nb<4, PAGED>(a, s);
    case 80: return launch_attn_nb<5, PAGED>(a, s);
    case 96: return launch_attn_nb<6, PAGED>(a, s);
    case 112: return launch_attn_nb<7, PAGED>(a, s);
    case 128: return launch_attn_nb<8, PAGED>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace mnmt
