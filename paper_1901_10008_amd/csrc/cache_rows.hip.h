// Device code of libsk_cache.so that moves rows and pages: norm, rotation and append; copies of pages.
#pragma once

#include "cache_kernels.hip.h"

namespace sk {

// ---------------------------------------------------------------------------
// norm, rotation, append
// ---------------------------------------------------------------------------
struct AppendArgs {
  const AttnDev *problems;
  const uint32_t *first;  // first workgroup of each problem
  int32_t n;
};

// The last index i of [0, n) with first[i] <= x, 64 candidates at a time (first[0] <= x, not decreasing; x the same in all lanes).
template <class T>
__device__ __forceinline__ int32_t last_not_above(const T *first, int32_t n, int64_t x, int lane) {
  int32_t lo = 0;
  while (n > 1) {
    const int32_t step = (n + 63) / 64, i = lo + lane * step;
    const bool le = lane * step < n && (int64_t)(*(const T SK_GLOBAL *)(uintptr_t)(first + i)) <= x;
    const int32_t hit = max(1, (int32_t)__popcll(__ballot(le))) - 1;
    lo += hit * step;
    n = min(step, n - hit * step);
  }
  return lo;
}

template <int DT>
__device__ __forceinline__ void append_row(const AttnDev &P, int32_t row, int32_t part, int lane) {
  const int32_t seq = last_not_above(P.first_row, P.sequences, row, lane);
  const int32_t a = load_i32(P.first_row + seq), b = load_i32(P.first_row + seq + 1);
  if (row < a || row >= b) return;
  const int64_t capacity = (int64_t)P.columns << P.page_shift;
  const int64_t length = min((int64_t)max(load_i32(P.lengths + seq), 0), capacity);
  const int64_t pos = length - (min(b, P.rows) - a) + (row - a);
  const bool in_cache = pos >= 0 && pos < capacity;
  const int32_t page = in_cache ? load_i32(P.table + (int64_t)seq * P.columns + (pos >> P.page_shift)) : -1;
  const bool there = (uint32_t)page < (uint32_t)P.num_pages;
  const int64_t slot = (int64_t)page * P.page_stride + (pos & ((1 << P.page_shift) - 1)) * P.token_stride;
  const int half = P.rotary / 2;
  const int64_t angle = min(max(pos, (int64_t)0), (int64_t)max(P.positions - 1, 0)) * half;

  const int lph = P.lanes_per_head, e0 = (lane & (lph - 1)) * 8, heads = P.q_heads + 2 * P.kv_heads;
  const int at_once = 64 / lph;
  const char *x_row = (const char *)P.qkv + 2 * (int64_t)row * P.qkv_row;
  for (int t = 0; t < P.turns; ++t) {
    const int head = (part * P.turns + t) * at_once + lane / lph;
    const bool ok = head < heads && e0 < P.dim;
    const char *xp = x_row + 2 * ((int64_t)head * P.dim + e0);
    u32x4 raw = load16(ok ? (const void *)xp : (const void *)g_zeros);
    const int kind = head < P.q_heads ? 0 : head < P.q_heads + P.kv_heads ? 1 : 2;
    if (kind < 2) {
      const void *w = kind == 0 ? P.q_weight : P.k_weight;
      float y[8];
      unpack8<DT>(raw, y);
      float scale = 1.f;
      if (w) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += y[i] * y[i];
        for (int d = 1; d < lph; d *= 2) sum += __shfl_xor(sum, d);
        scale = 1.f / sqrtf(sum / (float)P.dim + P.eps);
        float f[8];
        unpack8<DT>(load16(e0 < P.dim ? (const void *)((const char *)w + 2 * e0) : (const void *)g_zeros), f);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= scale * f[i];
      }
      if (ok && e0 < P.rotary) {
        if (P.neighbours) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (e0 + 2 * i >= P.rotary) break;
            const float co = P.cos[angle + e0 / 2 + i], si = P.sin[angle + e0 / 2 + i], u = y[2 * i], v = y[2 * i + 1];
            y[2 * i] = u * co - v * si;
            y[2 * i + 1] = v * co + u * si;
          }
        } else {
          // the other element of a pair, normalised like this one
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = e0 + i;
            if (e >= P.rotary) break;
            const bool low = e < half;
            const int other = low ? e + half : e - half, at = low ? e : other;
            const float co = P.cos[angle + at], si = P.sin[angle + at];
            float z = elem<DT>(*(const uint16_t SK_GLOBAL *)(uintptr_t)(xp + 2 * (other - e0)));
            if (w) z *= scale * elem<DT>(*(const uint16_t SK_GLOBAL *)(uintptr_t)((const char *)w + 2 * other));
            y[i] = low ? y[i] * co - z * si : y[i] * co + z * si;
          }
        }
      }
      raw = u32x4{pack2<DT>(y[0], y[1]), pack2<DT>(y[2], y[3]), pack2<DT>(y[4], y[5]), pack2<DT>(y[6], y[7])};
    }
    if (!ok) continue;
    if (kind == 0)
      store16((char *)P.q + 2 * ((int64_t)row * P.q_row + (int64_t)head * P.q_head + e0), raw);
    else if (there)
      store16((char *)(kind == 1 ? P.k : P.v) + 2 * (slot + (int64_t)(head - P.q_heads - (kind == 1 ? 0 : P.kv_heads)) * P.head_stride + e0), raw);
  }
}

__global__ void __launch_bounds__(CACHE_THREADS) sk_append(AppendArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t problem = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, lane));
  const AttnDev &P = a.problems[problem];
  const int64_t n = ((int64_t)blockIdx.x - a.first[problem]) * 4 + wave;
  const int64_t row = n / P.parts;
  if (row >= P.rows) return;
  if (P.dtype == SK_BF16)
    append_row<SK_BF16>(P, (int32_t)row, (int32_t)(n % P.parts), lane);
  else
    append_row<SK_F16>(P, (int32_t)row, (int32_t)(n % P.parts), lane);
}

// ---------------------------------------------------------------------------
// copies of pages
// ---------------------------------------------------------------------------
// A workgroup copies a chunk of a page of an array; those behind the copies bring changed rows of the page table, read from host
// memory.
__global__ void __launch_bounds__(CACHE_THREADS) sk_copy_pages(CopyArgs a) {
  const int64_t per_move = a.chunks * a.n_arrays;
  const int64_t copies = per_move * a.n_moves;
  if ((int64_t)blockIdx.x < copies) {
    const int32_t move = (int32_t)(blockIdx.x / per_move), rest = (int32_t)(blockIdx.x % per_move);
    const int32_t array = (int32_t)(rest / a.chunks);
    const int64_t begin = (int64_t)(rest % a.chunks) * COPY_CHUNK, bytes = a.arrays[array].bytes, end = min(bytes, begin + COPY_CHUNK);
    const char *src = a.arrays[array].base + bytes * a.moves[move].from;
    char *dst = a.arrays[array].base + bytes * a.moves[move].to;
    int64_t i = begin + 16 * (int64_t)threadIdx.x;
    constexpr int64_t STEP = 16 * CACHE_THREADS;
    for (; i + 3 * STEP < end; i += 4 * STEP) {
      u32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = load16(src + i + j * STEP);
#pragma unroll
      for (int j = 0; j < 4; ++j) store16(dst + i + j * STEP, v[j]);
    }
    for (; i < end; i += STEP) store16(dst + i, load16(src + i));
  } else {
    const int32_t r = (int32_t)(blockIdx.x - copies);
    if (r >= a.n_rows) return;
    const int32_t row = a.rows[r];
    for (int32_t i = threadIdx.x; i < a.columns; i += CACHE_THREADS) a.table[(int64_t)row * a.columns + i] = a.rows[a.n_rows + (int64_t)r * a.columns + i];
  }
}

}  // namespace sk
