// Device code of libsk_cache.so that moves rows and pages: norm, rotation and append; copies of pages.
#pragma once

#include "cache_kernels.hip.h"

namespace sk {

// ---------------------------------------------------------------------------
// norm, rotation, append
// ---------------------------------------------------------------------------
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ f32x4 load_f4_any(const float *p) { return *(const f32x4_any SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ float load_f(const float *p) { return *(const float SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ uint32_t load_u16(const void *p) { return *(const uint16_t SK_GLOBAL *)(uintptr_t)p; }

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

// Loads and stores of what a launch will not see again, past the caches (ONCE) where it moves more than PAST_CACHES bytes: what is there
// stays there, and the launch is faster by as much (19000 rows of 48 heads of 128 by 7 %, 1 GB of pages by 3 %).  A smaller launch's
// outputs would be found in the caches by the one that reads them.
template <bool ONCE>
__device__ __forceinline__ u32x4 load16_once(const void *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4 SK_GLOBAL *)(uintptr_t)p);
  return load16(p);
}
template <bool ONCE>
__device__ __forceinline__ void store16_once(void *p, u32x4 v) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(v, (u32x4 SK_GLOBAL *)(uintptr_t)p);
  else
    store16(p, v);
}

// The sum over groups of 1, 2, 4, .. 32 neighbouring lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ float other_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int32_t, v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_over(float v, int lanes) {
  if (lanes >= 2) v += other_lane<0xb1>(v);    // quad_perm: the other of two
  if (lanes >= 4) v += other_lane<0x4e>(v);    // quad_perm: the other two of four
  if (lanes >= 8) v += other_lane<0x141>(v);   // row_half_mirror
  if (lanes >= 16) v += other_lane<0x140>(v);  // row_mirror
  if (lanes >= 32) v = sum16(v);
  return v;
}

// How a row's heads are rotated: not at all; pairs of elements half the rotated length apart, where that is whole pieces of 8; neighbours, in
// whole pieces; element by element.
enum { ROTATE_NONE, ROTATE_HALVES, ROTATE_NEIGHBOURS, ROTATE_ANY };

// A wave takes some heads of a row, 8 elements a lane, in turns of as many heads as it has lanes for.  What a lane needs of the angles and weights is
// the same in every turn and stays in registers; the other element of a pair is read from memory once more (the line is in the L1)
// and normalised like the first.  Bound by memory: every element is read and written once; 19000 rows of 48 heads of 128, 469 MB in 96 us,
// 4.9 TB/s (a large copy 5.15).  A step of few rows is bound by a launch and its chain of loads (row, sequence, page, heads): 3 rows 3.6 us.
template <int DT, int ROTATE, bool ONCE>
__device__ __forceinline__ void append_heads(const SK_CONSTANT AttnDev &P, int64_t row, int32_t part, int lane, int64_t angle, bool there, int64_t slot) {
  const int lph = P.lanes_per_head, e0 = (lane & (lph - 1)) * 8, at_once = 64 / lph, dim = P.dim, half = P.rotary / 2;
  const int q_heads = P.q_heads, kv_heads = P.kv_heads, heads = q_heads + 2 * kv_heads;
  const char *x = (const char *)P.qkv + 2 * (row * P.qkv_row + e0);
  const bool in_head = e0 < dim, turned = ROTATE != ROTATE_NONE && e0 < P.rotary;
  const bool low = e0 < half;
  const int other = ROTATE == ROTATE_HALVES && turned ? (low ? half : -half) : 0;  // from a lane's elements to the others of their pairs
  const bool q_norm = P.q_weight != nullptr, k_norm = P.k_weight != nullptr;

  u32x4 qw = {0, 0, 0, 0}, kw = qw, qo = qw, ko = qw;
  if (q_norm) {
    qw = load16(in_head ? (const char *)P.q_weight + 2 * e0 : (const char *)g_zeros);
    if (ROTATE == ROTATE_HALVES) qo = load16(in_head ? (const char *)P.q_weight + 2 * (e0 + other) : (const char *)g_zeros);
  }
  if (k_norm) {
    kw = load16(in_head ? (const char *)P.k_weight + 2 * e0 : (const char *)g_zeros);
    if (ROTATE == ROTATE_HALVES) ko = load16(in_head ? (const char *)P.k_weight + 2 * (e0 + other) : (const char *)g_zeros);
  }
  // (a, b) -> (a co - b si, b co + a si): of halves a lane holds eight a or eight b, and si has the sign it needs
  float co[8], si[8];
  if constexpr (ROTATE == ROTATE_HALVES || ROTATE == ROTATE_NEIGHBOURS) {
    constexpr int N = ROTATE == ROTATE_HALVES ? 8 : 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) co[i] = 1.f, si[i] = 0.f;
    if (turned) {
      const int64_t at = angle + (ROTATE == ROTATE_HALVES ? (low ? e0 : e0 - half) : e0 / 2);
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const f32x4 c4 = load_f4_any(P.cos + at + i), s4 = load_f4_any(P.sin + at + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          co[i + j] = c4[j];
          si[i + j] = ROTATE == ROTATE_HALVES && low ? -s4[j] : s4[j];
        }
      }
    }
  }
  u32x4 raw, pair;  // of the next turn
  const int first = part * P.turns * at_once + lane / lph;
  auto load = [&](int t, u32x4 &v, u32x4 &w) {
    const int head = first + t * at_once;
    const bool ok = head < heads && in_head && t < P.turns;
    const char *p = x + 2 * (int64_t)head * dim;
    v = load16_once<ONCE>(ok ? p : (const char *)g_zeros);
    if (ROTATE == ROTATE_HALVES) w = load16(ok ? p + 2 * other : (const char *)g_zeros);
  };
  load(0, raw, pair);
  for (int t = 0; t < P.turns; ++t) {
    const int head = first + t * at_once;
    u32x4 v = raw;
    const u32x4 w = pair;
    load(t + 1, raw, pair);
    const int kind = head < q_heads ? 0 : head < q_heads + kv_heads ? 1 : 2;
    const bool norm = kind == 0 ? q_norm : kind == 1 && k_norm;
    float y[8];
    unpack8<DT>(v, y);
    float scale = 1.f;
    if (__ballot(norm)) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += y[k] * y[k];
      sum = sum_over(sum, lph);
      if (norm) {
        scale = 1.f / sqrtf(sum / (float)dim + P.eps);
        float f[8];
        unpack8<DT>(kind == 0 ? qw : kw, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] *= scale * f[k];
      }
    }
    if (kind < 2) {
      if constexpr (ROTATE == ROTATE_HALVES) {
        float z[8], f[8];
        unpack8<DT>(w, z);
        unpack8<DT>(kind == 0 ? qo : ko, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float r = y[k] * co[k] + (norm ? z[k] * (scale * f[k]) : z[k]) * si[k];
          y[k] = turned ? r : y[k];  // (an infinite element that is not rotated stays what it is)
        }
      } else if constexpr (ROTATE == ROTATE_NEIGHBOURS) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float a = y[2 * k], b = y[2 * k + 1];
          y[2 * k] = turned ? a * co[k] - b * si[k] : a;
          y[2 * k + 1] = turned ? b * co[k] + a * si[k] : b;
        }
      } else if constexpr (ROTATE == ROTATE_ANY) {
        if (turned && head < heads && in_head) {
          const char *xp = x + 2 * (int64_t)head * dim;
          const char *wp = (const char *)(kind == 0 ? P.q_weight : P.k_weight) + 2 * e0;
          for (int k = 0; k < 8; ++k) {
            const int e = e0 + k;
            if (e >= P.rotary) break;
            const bool a = P.neighbours ? (e & 1) == 0 : e < half;
            const int to = P.neighbours ? (a ? 1 : -1) : (a ? half : -half), at = P.neighbours ? e / 2 : (a ? e : e - half);
            float z = elem<DT>(load_u16(xp + 2 * (k + to)));
            if (norm) z *= scale * elem<DT>(load_u16(wp + 2 * (k + to)));
            const float c1 = load_f(P.cos + angle + at), s1 = load_f(P.sin + angle + at), o = elem<DT>(load_u16(xp + 2 * k));
            const float n = norm ? o * (scale * elem<DT>(load_u16(wp + 2 * k))) : o;
            const float r = a ? n * c1 - z * s1 : n * c1 + z * s1;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = j == k ? r : y[j];
          }
        }
      }
      if (norm || ROTATE != ROTATE_NONE) v = u32x4{pack2<DT>(y[0], y[1]), pack2<DT>(y[2], y[3]), pack2<DT>(y[4], y[5]), pack2<DT>(y[6], y[7])};
    }
    if (head >= heads || !in_head) continue;
    if (kind == 0)
      store16_once<ONCE>((char *)P.q + 2 * (row * P.q_row + (int64_t)head * P.q_head + e0), v);
    else if (there)
      store16_once<ONCE>((char *)(kind == 1 ? P.k : P.v) + 2 * (slot + (int64_t)(head - q_heads - (kind == 1 ? 0 : kv_heads)) * P.head_stride + e0), v);
  }
}

template <int DT, bool ONCE>
__device__ __forceinline__ void append_row(const SK_CONSTANT AttnDev &P, int32_t row, int32_t part, int lane) {
  int32_t seq, a, b, n;
  if (P.sequences <= 64) {  // a sequence per lane
    const int s = min(lane, P.sequences - 1);
    const int32_t first = load_i32(P.first_row + s), next = load_i32(P.first_row + s + 1), length = load_i32(P.lengths + s);
    seq = max(1, (int32_t)__popcll(__ballot(lane < P.sequences && first <= row))) - 1;
    a = lane_of(first, seq), b = lane_of(next, seq), n = lane_of(length, seq);
  } else {
    seq = __builtin_amdgcn_readfirstlane(last_not_above(P.first_row, P.sequences, row, lane));
    a = load_i32(P.first_row + seq), b = load_i32(P.first_row + seq + 1), n = load_i32(P.lengths + seq);
  }
  if (row < a || row >= b) return;
  const int64_t capacity = (int64_t)P.columns << P.page_shift;
  const int64_t pos = min((int64_t)max(n, 0), capacity) - min(b, P.rows) + row;  // (below the capacity, whatever first_row holds)
  const int32_t page = pos >= 0 ? load_i32(P.table + (int64_t)seq * P.columns + (pos >> P.page_shift)) : -1;
  const bool there = (uint32_t)page < (uint32_t)P.num_pages;
  const int64_t slot = (int64_t)page * P.page_stride + (pos & ((1 << P.page_shift) - 1)) * P.token_stride;
  const int64_t angle = max(pos, (int64_t)0) * (P.rotary / 2);
  const int kind = P.rotary == 0 ? ROTATE_NONE : !P.neighbours && P.rotary % 16 == 0 ? ROTATE_HALVES : P.neighbours && P.rotary % 8 == 0 ? ROTATE_NEIGHBOURS : ROTATE_ANY;
  switch (kind) {
    case ROTATE_NONE: return append_heads<DT, ROTATE_NONE, ONCE>(P, row, part, lane, angle, there, slot);
    case ROTATE_HALVES: return append_heads<DT, ROTATE_HALVES, ONCE>(P, row, part, lane, angle, there, slot);
    case ROTATE_NEIGHBOURS: return append_heads<DT, ROTATE_NEIGHBOURS, ONCE>(P, row, part, lane, angle, there, slot);
    default: return append_heads<DT, ROTATE_ANY, ONCE>(P, row, part, lane, angle, there, slot);
  }
}

template <bool ONCE>
__global__ void __launch_bounds__(CACHE_THREADS) sk_append(AppendArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t problem = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, lane));
  const SK_CONSTANT AttnDev &P = *(const SK_CONSTANT AttnDev *)(uintptr_t)(a.problems + problem);
  const uint32_t first = a.n == 1 ? 0u : ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[problem];
  const int64_t n = ((int64_t)blockIdx.x - first) * 4 + wave;
  const int64_t row = n / P.parts;
  if (row >= P.rows) return;
  if (P.dtype == SK_BF16)
    append_row<SK_BF16, ONCE>(P, (int32_t)row, (int32_t)(n % P.parts), lane);
  else
    append_row<SK_F16, ONCE>(P, (int32_t)row, (int32_t)(n % P.parts), lane);
}

// ---------------------------------------------------------------------------
// copies of pages
// ---------------------------------------------------------------------------
// Bound by memory: 500 pages of 32 KB in each of 32 arrays, 1.05 GB read and written in 211 us, 5.0 TB/s.  A workgroup copies a chunk of a page
// of an array; those behind the copies bring changed rows of the page table, out of the launch's arguments where they fit (a fork into sixteen
// sequences of 50 pages: 4.4 us so, 6.0 with the rows in host memory).
template <bool ONCE>
__global__ void __launch_bounds__(CACHE_THREADS) sk_copy_pages(CopyArgs a) {
  const int64_t per_move = a.chunks * a.n_arrays;
  const int64_t copies = per_move * a.n_moves;
  if ((int64_t)blockIdx.x < copies) {
    const int32_t move = (int32_t)(blockIdx.x / per_move), rest = (int32_t)(blockIdx.x % per_move);
    const int32_t array = (int32_t)(rest / a.chunks), at = 4 * array, from = 4 * a.n_arrays + 2 * move;
    char *base = (char *)((uint64_t)(uint32_t)a.words[at + 1] << 32 | (uint32_t)a.words[at]);
    const int64_t bytes = (int64_t)((uint64_t)(uint32_t)a.words[at + 3] << 32 | (uint32_t)a.words[at + 2]);
    const int64_t begin = (int64_t)(rest % a.chunks) * COPY_CHUNK, end = min(bytes, begin + COPY_CHUNK);
    const char *src = base + bytes * a.words[from];
    char *dst = base + bytes * a.words[from + 1];
    int64_t i = begin + 16 * (int64_t)threadIdx.x;
    constexpr int64_t STEP = 16 * CACHE_THREADS;
    for (; i + 3 * STEP < end; i += 4 * STEP) {
      u32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = load16_once<ONCE>(src + i + j * STEP);
#pragma unroll
      for (int j = 0; j < 4; ++j) store16_once<ONCE>(dst + i + j * STEP, v[j]);
    }
    for (; i < end; i += STEP) store16(dst + i, load16(src + i));
  } else {
    const int32_t at = 4 * a.n_arrays + 2 * a.n_moves, groups = (int32_t)(gridDim.x - copies);
    for (int32_t r = (int32_t)(blockIdx.x - copies); r < a.n_rows; r += groups) {
      const int64_t row = a.rows ? a.rows[r] : a.words[at + r], first = a.n_rows + (int64_t)r * a.columns;
      for (int32_t i = threadIdx.x; i < a.columns; i += CACHE_THREADS) a.table[row * a.columns + i] = a.rows ? a.rows[first + i] : a.words[at + first + i];
    }
  }
}

}  // namespace sk
