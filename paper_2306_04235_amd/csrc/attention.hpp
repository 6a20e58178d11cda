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
// One pass: scores are taken relative to the largest so far, an int32 that starts
// the products' accumulators at its negative for nothing.  Where a step brings a
// larger one, the sums so far are folded into fp32 and rescaled; the other steps
// (after a row's first keys, most) add integers only.
#pragma once

#include <climits>

#include "blocks.hpp"
#include "cache.hpp"

namespace mnmt {

constexpr int kAttnKeys = 64;         // keys per step of a wave
constexpr int kNoReference = -(1 << 22);  // below every score (|s| <= 127^2 128 < 2^21)
constexpr int kFoldSteps = 1024;      // steps after which the int32 sums are folded: 65536 * 2^14 < 2^31
constexpr float kLog2One = 22.99f;    // log2 of the fixed-point 1, below 0x7F7F7F, the largest number with digits in range
constexpr float kDigits = 8388608.f + 32896.f;
constexpr uint32_t kDigitBits = 0x4B008080u;  // its bits: p = 0

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
__device__ __forceinline__ int live_splits(const AttnArgs& a, int tile, int keys) {
  return tile < a.tiles ? min(a.splits, max(1, (keys + a.chunk - 1) / a.chunk)) : 1;
}

// Where a lane finds its keys and values: pages, values [token / 16][dh][16].
template <int NB>
struct PagedKeys {
  const AttnArgs& a;
  const int32_t* table;
  size_t koff, voff;
  int last, gk, gv, page_k, page_v;
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

template <int NB, bool PAGED, int WK>
__global__ __launch_bounds__(256, 2) void k_attn(AttnArgs a) {
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
    const int keys = tile_keys(a, w, tile), live = live_splits(a, tile, keys);
    if (split >= live) continue;
    const int kbegin = split * a.chunk, kend = split == live - 1 ? keys : kbegin + a.chunk;
    const int all_see = w.seen(a, 16 * tile / a.group);  // keys that every query of the tile sees
    // the lane's query
    const int m = 16 * tile + col, token = m / a.group;
    const bool real = token < w.n;
    const int mine = real ? w.seen(a, token) : INT_MAX;
    const size_t qrow = (size_t)w.first + (real ? token : 0);
    const int qhead = head * a.group + (real ? m - token * a.group : 0);
    v4i qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 64 * s + 16 * g;
      qf[s] = c < dh && real ? *(const v4i*)(a.q + qrow * a.ldq + (size_t)qhead * dh + c) : v4i{0, 0, 0, 0};
    }
    v4i acc[3][NB];
    float f[NB][4], sum = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[b][i] = 0.f;
        acc[0][b][i] = acc[1][b][i] = acc[2][b][i] = 0;
      }
    int ref = kNoReference, steps = 0;
    bool folded = false;
    auto fold = [&] {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[b][i] = fmaf(65536.f, (float)acc[0][b][i], f[b][i]);
          f[b][i] = fmaf(256.f, (float)acc[1][b][i], f[b][i]);
          f[b][i] += (float)acc[2][b][i];
          acc[0][b][i] = acc[1][b][i] = acc[2][b][i] = 0;
        }
    };
    // key rows of the lane in a step: 16 (l / 4 mod 4) + 4 j + l mod 4; slices past the head read its first bytes (their queries are 0)
    int slice[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) slice[s] = 64 * s + 16 * g < dh ? 64 * s + 16 * g : 0;
    PagedKeys<NB> at(a, PAGED ? row : 0, head, lane, kend);
    const int8_t* kbase = PAGED ? nullptr : a.k + (size_t)row * a.batch + (size_t)head * dh;
    const int8_t* vbase = PAGED ? nullptr : a.v + (size_t)row * a.batch + (size_t)head * dh;
    int8_t* stage = lds + wave * kWave;
    int key = kbegin + (WK == 1 ? 0 : kAttnKeys * wave);
    if (PAGED && key < kend) at.look(key);
    for (; key < kend; key += kAttnKeys * WK) {
      v4i kf[4][KS], vf[NB];
      bool there = true;
      if constexpr (PAGED) {
        const int8_t* kp = at.keys_of(key);
        const int8_t* vp = at.values_of(key);
        there = at.there();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int s = 0; s < KS; ++s) kf[j][s] = *(const v4i*)(kp + 4 * j * dh + slice[s]);
#pragma unroll
        for (int b = 0; b < NB; ++b) vf[b] = *(const v4i*)(vp + 256 * b);
        at.look(min(key + kAttnKeys * WK, kend - 1));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int8_t* kp = kbase + (size_t)min(key + 16 * ((lane >> 2) & 3) + 4 * j + (lane & 3), kend - 1) * a.ld;
#pragma unroll
          for (int s = 0; s < KS; ++s) kf[j][s] = *(const v4i*)(kp + slice[s]);
        }
        // values: a lane takes 4 keys (4 (l mod 16) ..) and 16 columns, and
        // stores dwords of 4 keys; chunks of 16 keys are swapped about by
        // column so that neither side meets bank conflicts
        v4i vr[4][KS];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int8_t* vp = vbase + (size_t)min(key + 4 * col + i, kend - 1) * a.ld;
#pragma unroll
          for (int s = 0; s < KS; ++s) vr[i][s] = *(const v4i*)(vp + slice[s]);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (64 * s + 16 * g < dh) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t x[4] = {(uint32_t)vr[0][s][c], (uint32_t)vr[1][s][c], (uint32_t)vr[2][s][c],
                                     (uint32_t)vr[3][s][c]};
              uint32_t y[4];
              transpose4(x, y[0], y[1], y[2], y[3]);
              // column 64 s + 16 g + 4 c + b: chunk (col / 4) ^ c ^ g
#pragma unroll
              for (int b = 0; b < 4; ++b)
                *(uint32_t*)(stage + (64 * s + 16 * g + 4 * c + b) * 64 + 16 * ((col >> 2) ^ c ^ g) + 4 * (col & 3)) = y[b];
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
      // scores less the reference: the lane's query, keys key + 16 g + 4 j + i
      v4i d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] = mfma16(kf[j][0], qf[0], v4i{-ref, -ref, -ref, -ref});
#pragma unroll
        for (int s = 1; s < KS; ++s) d[j] = mfma16(kf[j][s], qf[s], d[j]);
      }
      const int k0 = key + 16 * g, last = min(mine, kend);
      const bool masked = key + kAttnKeys > min(all_see, kend) || __any(!there);
      if (masked) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!there || k0 + 4 * j + i >= last) d[j][i] = INT_MIN / 2;
      }
      int top = max(max(d[0][0], d[0][1]), d[0][2]);
      top = max(top, d[0][3]);
#pragma unroll
      for (int j = 1; j < 4; ++j) {
        top = max(max(top, d[j][0]), d[j][1]);
        top = max(max(top, d[j][2]), d[j][3]);
      }
      top = quad_max(top);
      ++steps;
      if (__any(top > 0) || steps == kFoldSteps) {
        const int up = max(top, 0);
        if (steps > 1 || folded) {
          const float scale = __builtin_amdgcn_exp2f(-(float)up * a.c2);
          fold();
          folded = true;
          steps = 1;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[b][i] *= scale;
          sum *= scale;
        }
        ref += up;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][i] -= up;  // (masked places stay far below)
      }
      uint32_t total = 0;
      v4i pa, pb, pc;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = __float_as_uint(__builtin_amdgcn_exp2f(fmaf((float)d[j][i], a.c2, kLog2One)) + kDigits);
          if (masked && (!there || k0 + 4 * j + i >= last)) x[i] = kDigitBits;
          total += x[i];
        }
        const uint32_t lo0 = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), lo1 = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);
        const uint32_t hi0 = __builtin_amdgcn_perm(x[1], x[0], 0x0c0c0602u), hi1 = __builtin_amdgcn_perm(x[3], x[2], 0x0c0c0602u);
        pc[j] = (int)(__builtin_amdgcn_perm(lo1, lo0, 0x05040100u) ^ 0x80808080u);
        pb[j] = (int)(__builtin_amdgcn_perm(lo1, lo0, 0x07060302u) ^ 0x80808080u);
        pa[j] = (int)__builtin_amdgcn_perm(hi1, hi0, 0x05040100u);
      }
      sum += (float)(total - 16u * kDigitBits);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        acc[0][b] = mfma16(vf[b], pa, acc[0][b]);
        acc[1][b] = mfma16(vf[b], pb, acc[1][b]);
        acc[2][b] = mfma16(vf[b], pc, acc[2][b]);
      }
    }
    fold();
    sum = quad_sum(sum);
    // f: columns 16 b + 4 g + i of the lane's query
    float* part = a.part + ((size_t)(row * a.n_kv_heads + head) * a.tiles + tile) * a.splits * (16 * (dh + 2)) +
                  (size_t)split * (16 * (dh + 2));
    if constexpr (WK == 1) {
      if (live == 1) {
        if (real) {
          const float inv = sum > 0.f ? a.c_pv / sum : 0.f;
          const size_t o = qrow * a.ldo + (size_t)qhead * dh + 4 * g;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if (a.kind == MNMT_ATTN_F32) {
              *(float4*)((float*)a.out + o + 16 * b) =
                  make_float4(f[b][0] * inv, f[b][1] * inv, f[b][2] * inv, f[b][3] * inv);
            } else {
              char4 c = make_char4(code_of(f[b][0] * inv), code_of(f[b][1] * inv), code_of(f[b][2] * inv),
                                   code_of(f[b][3] * inv));
              *(char4*)((int8_t*)a.out + o + 16 * b) = c;
            }
          }
        }
      } else {
        if (g == 0) {
          part[16 * dh + col] = sum;
          part[16 * dh + 16 + col] = (float)ref;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
          *(float4*)(part + col * dh + 16 * b + 4 * g) = make_float4(f[b][0], f[b][1], f[b][2], f[b][3]);
      }
    } else {
      // join the four waves' sums, each relative to its own reference
      float* mine_f = (float*)(lds + wave * kWave);
      if (g == 0) {
        mine_f[col] = sum;
        mine_f[16 + col] = (float)ref;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *(float4*)(mine_f + 32 + col * (dh + 4) + 16 * b + 4 * g) = make_float4(f[b][0], f[b][1], f[b][2], f[b][3]);
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * dh / 4; i += 256) {
        const int q = i / (dh / 4), c = 4 * (i % (dh / 4));
        float top = (float)kNoReference, wsum = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int v = 0; v < 4; ++v) top = fmaxf(top, ((const float*)(lds + v * kWave))[16 + q]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float* src = (const float*)(lds + v * kWave);
          const float scale = __builtin_amdgcn_exp2f((src[16 + q] - top) * a.c2);
          const float4 x = *(const float4*)(src + 32 + q * (dh + 4) + c);
          wsum = fmaf(scale, src[q], wsum);
          y.x = fmaf(scale, x.x, y.x);
          y.y = fmaf(scale, x.y, y.y);
          y.z = fmaf(scale, x.z, y.z);
          y.w = fmaf(scale, x.w, y.w);
        }
        if (live == 1) {
          const int mq = 16 * tile + q, tq = mq / a.group;
          if (tq < w.n) {
            const float inv = wsum > 0.f ? a.c_pv / wsum : 0.f;
            const size_t o = ((size_t)w.first + tq) * a.ldo + (size_t)(head * a.group + mq - tq * a.group) * dh + c;
            if (a.kind == MNMT_ATTN_F32)
              *(float4*)((float*)a.out + o) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
            else
              *(char4*)((int8_t*)a.out + o) =
                  make_char4(code_of(y.x * inv), code_of(y.y * inv), code_of(y.z * inv), code_of(y.w * inv));
          }
        } else {
          if (c == 0) {
            part[16 * dh + q] = wsum;
            part[16 * dh + 16 + q] = top;
          }
          *(float4*)(part + q * dh + c) = y;
        }
      }
      __syncthreads();
    }
  }
}

// Joins the key ranges of a query tile; one block per tile.
template <int NB>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  constexpr int dh = 16 * NB;
  const int per_row = a.n_kv_heads * a.tiles;
  const int row = blockIdx.x / per_row, head = blockIdx.x % per_row / a.tiles, tile = blockIdx.x % a.tiles;
  const AttnRow w = attn_row(a, row);
  if (16 * tile >= w.n * a.group) return;
  const int live = live_splits(a, tile, tile_keys(a, w, tile));
  if (live == 1) return;
  const float* part = a.part + (size_t)blockIdx.x * a.splits * (16 * (dh + 2));
  for (int i = threadIdx.x; i < 16 * dh / 4; i += 256) {
    const int q = i / (dh / 4), c = 4 * (i % (dh / 4)), mq = 16 * tile + q, tq = mq / a.group;
    if (tq >= w.n) continue;
    float top = (float)kNoReference, wsum = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < live; ++s) top = fmaxf(top, part[(size_t)s * (16 * (dh + 2)) + 16 * dh + 16 + q]);
    for (int s = 0; s < live; ++s) {
      const float* src = part + (size_t)s * (16 * (dh + 2));
      const float scale = __builtin_amdgcn_exp2f((src[16 * dh + 16 + q] - top) * a.c2);
      const float4 x = *(const float4*)(src + q * dh + c);
      wsum = fmaf(scale, src[16 * dh + q], wsum);
      y.x = fmaf(scale, x.x, y.x);
      y.y = fmaf(scale, x.y, y.y);
      y.z = fmaf(scale, x.z, y.z);
      y.w = fmaf(scale, x.w, y.w);
    }
    const float inv = wsum > 0.f ? a.c_pv / wsum : 0.f;
    const size_t o = ((size_t)w.first + tq) * a.ldo + (size_t)(head * a.group + mq - tq * a.group) * dh + c;
    if (a.kind == MNMT_ATTN_F32)
      *(float4*)((float*)a.out + o) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
    else
      *(char4*)((int8_t*)a.out + o) =
          make_char4(code_of(y.x * inv), code_of(y.y * inv), code_of(y.z * inv), code_of(y.w * inv));
  }
}

template <int NB, bool PAGED>
hipError_t launch_attn_nb(const AttnArgs& a, int waves, hipStream_t s) {
  const int tiles = a.rows * a.n_kv_heads * a.tiles, units = tiles * a.splits;
  if (waves == 1)
    hipLaunchKernelGGL((k_attn<NB, PAGED, 1>), dim3((units + 3) / 4), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_attn<NB, PAGED, 4>), dim3(units), dim3(256), 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((k_attn_join<NB>), dim3(tiles), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <bool PAGED>
hipError_t launch_attn_kernel(const AttnArgs& a, int d_head, int waves, hipStream_t s) {
  switch (d_head) {
    case 16: return launch_attn_nb<1, PAGED>(a, waves, s);
    case 32: return launch_attn_nb<2, PAGED>(a, waves, s);
    case 48: return launch_attn_nb<3, PAGED>(a, waves, s);
    case 64: return launch_attn_nb<4, PAGED>(a, waves, s);
    case 80: return launch_attn_nb<5, PAGED>(a, waves, s);
    case 96: return launch_attn_nb<6, PAGED>(a, waves, s);
    case 112: return launch_attn_nb<7, PAGED>(a, waves, s);
    case 128: return launch_attn_nb<8, PAGED>(a, waves, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace mnmt
