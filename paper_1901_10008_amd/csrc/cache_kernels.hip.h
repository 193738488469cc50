// Device code of libsk_cache.so (gfx950 / CDNA4 only): attention over paged caches, and what its kernels share with cache_rows.hip.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"

#if defined(__HIP_DEVICE_COMPILE__) && !defined(__gfx950__)
#error "written for gfx950"
#endif

namespace sk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// (pointers out of descriptors: said to be global, so that loads are not flat ones)
#define SK_GLOBAL __attribute__((address_space(1)))
__device__ __forceinline__ u32x4 load16(const void *p) { return *(const u32x4 SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ f32x4 load_f4(const void *p) { return *(const f32x4 SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ int32_t load_i32(const int32_t *p) { return *(const int32_t SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ void store16(void *p, u32x4 v) { *(u32x4 SK_GLOBAL *)(uintptr_t)p = v; }
__device__ __forceinline__ void store8(void *p, u32x2 v) { *(u32x2 SK_GLOBAL *)(uintptr_t)p = v; }

// What a lane reads that must count as zeros: its address is replaced, so that no load stands under a branch.
__device__ __attribute__((aligned(16))) const uint32_t g_zeros[4] = {0u, 0u, 0u, 0u};

template <int DT>
__device__ __forceinline__ float elem(uint32_t bits) {
  if constexpr (DT == SK_BF16) return __builtin_bit_cast(float, bits << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <int DT>
__device__ __forceinline__ void unpack8(const u32x4 &v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = elem<DT>(v[i] & 0xffffu);
    x[2 * i + 1] = elem<DT>(v[i] >> 16);
  }
}
// Two values rounded to nearest even, the first in the low half.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  if constexpr (DT == SK_BF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  }
}
template <int DT>
__device__ __forceinline__ void mma16(const u32x4 &a, const u32x4 &b, f32x4 &c) {
  if constexpr (DT == SK_BF16)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ void mma32(const u32x4 &a, const u32x4 &b, f32x16 &c) {
  if constexpr (DT == SK_BF16)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// The transposing LDS read: each group of 16 lanes reads four rows of 16 16-bit elements, lane i of the group elements
// 4 (i % 4) .. + 3 of row i / 4, and gets column i: four elements, one per row.
__device__ __forceinline__ u32x2 read_transposed(const unsigned char *p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(unsigned char *)p));
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Partial results that another workgroup reads, maybe behind another L2: written through to memory and read from there
// (device scope).
__device__ __forceinline__ void store_shared(float *p, f32x2 v) {
  __hip_atomic_store((unsigned long long *)p, __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_shared(const float *p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// ---------------------------------------------------------------------------
// which unit of work a workgroup takes
// ---------------------------------------------------------------------------
// The lengths are in device memory, so the units (a block of rows of a key-value head of a sequence, and a slice of its
// keys) are counted on the device: every workgroup looks at all sequences of the launch and finds its own unit from the sums
// before it.  Units of many rows come first, those of late rows (which see the most) before those of early ones; key-value heads
// vary fastest, so that with eight of them each has a die (and its L2) of its own.
struct Unit {
  int32_t problem, seq;
  int32_t head, block;          // key-value head, block of rows
  int32_t split, splits;
  uint32_t slot;                // this workgroup's place in the workspace
  uint32_t first_slot;          // of the unit's first slice: also its arrival counter
  bool many, any;
};

// A sequence in this step: rows and lengths cut to the bounds that the grid was made for.
struct Step {
  int32_t first, fresh, length, behind;  // first row, rows to compute, tokens, position of the first new token
};
__device__ __forceinline__ Step step_of(const int32_t *length, const int32_t *first, int32_t rows, int32_t max_new, int64_t capacity) {
  const int32_t a = load_i32(first), b = load_i32(first + 1), n = load_i32(length);
  Step s;
  s.first = min(max(a, 0), rows);
  const int32_t all = min(max(b, s.first), rows) - s.first;
  s.length = (int32_t)min((int64_t)max(n, 0), capacity);
  s.behind = s.length - all;
  s.fresh = min(all, max_new);
  return s;
}
// The keys that rows at positions p0 .. p1 see: blocks of KEYS from 0 on that hold sinks, then blocks from `low` on.
struct Span {
  int32_t low, sink_blocks, blocks;
};
template <int KEYS>
__device__ __forceinline__ Span span_of(int32_t p0, int32_t p1, int32_t window, int32_t sinks) {
  Span s;
  s.low = window ? max(0, (int32_t)max((int64_t)p0 - window + 1, (int64_t)0)) & ~(KEYS - 1) : 0;
  s.sink_blocks = window ? (int32_t)(((int64_t)min(sinks, s.low) + KEYS - 1) / KEYS) : 0;
  s.blocks = p1 < 0 ? 0 : s.sink_blocks + (p1 - s.low) / KEYS + 1;
  if (p1 < 0) s.sink_blocks = 0;
  return s;
}

struct Count {
  int32_t units, blocks;  // blocks of keys of an average unit
  bool many;
};
__device__ __forceinline__ Count count_units(const Step &s, int32_t kv_heads, int32_t group, int32_t window, int32_t sinks) {
  Count c;
  const int64_t rows = (int64_t)s.fresh * group;
  c.many = rows > MOST_FEW;
  const int32_t per = c.many ? ROWS_MANY : ROWS_FEW;
  const int32_t row_blocks = (int32_t)((rows + per - 1) / per);
  c.units = row_blocks * kv_heads;
  const int32_t tokens = (per + group - 1) / group, last = s.behind + s.fresh - 1;
  if (c.many) {
    const Span a = span_of<KEYS_MANY>(s.behind, min(s.behind + tokens - 1, last), window, sinks);
    const Span b = span_of<KEYS_MANY>(max(last - tokens + 1, s.behind), last, window, sinks);
    c.blocks = (a.blocks + b.blocks + 1) / 2;
  } else {
    c.blocks = span_of<KEYS_FEW>(s.behind, last, window, sinks).blocks;
  }
  return c;
}

struct FindScratch {
  int64_t total[2][4];  // blocks of keys over all units (many, few), per wave
  int32_t units[2][4];
  int32_t items[2][4];
  Unit unit;
};

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ int32_t wave_sum(int32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ int32_t wave_scan(int32_t v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

struct AttnArgs {
  const AttnDev *problems;
  const AttnSeq *seqs;
  int32_t sequences;
  uint32_t grid_many, grid_few;
  float *ws_many, *ws_few;
  uint32_t *arrivals;  // grid_many + grid_few, zero between launches
};

// How many blocks of keys a slice takes so that all slices fit `grid` workgroups: ceil(blocks / that) over the units adds up to
// total / that + units at most.  No unit is split where the units alone do not leave room.
__device__ __forceinline__ int32_t blocks_per_slice(int64_t total, int64_t units, int64_t grid, int32_t least) {
  if (units >= grid) return 0x7fffffff;
  const int64_t per = (total + (grid - units) - 1) / (grid - units);
  return (int32_t)min(max(per, (int64_t)least), (int64_t)0x7fffffff);
}
__device__ __forceinline__ int32_t splits_of(int32_t blocks, int32_t per) {
  return min(max((int32_t)(((int64_t)blocks + per - 1) / per), 1), MOST_SPLITS);
}
constexpr int LEAST_FEW = 4;   // a block of keys for each wave
constexpr int LEAST_MANY = 4;  // 256 keys

__device__ __forceinline__ void find_unit(const AttnArgs &a, FindScratch *f) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.sequences + CACHE_THREADS - 1) / CACHE_THREADS;
  const int s0 = tid * per, s1 = min(s0 + per, a.sequences);
  auto look = [&](int s) {
    const AttnSeq q = a.seqs[s];
    return count_units(step_of(q.length, q.first, q.rows, q.max_new, q.capacity), q.kv_heads, q.group, q.window, q.sinks);
  };
  int64_t total_many = 0, total_few = 0;
  int32_t units_many = 0, units_few = 0;
  Count mine = {};  // (the only one, with at most CACHE_THREADS sequences)
  for (int s = s0; s < s1; ++s) {
    mine = look(s);
    (mine.many ? total_many : total_few) += (int64_t)mine.units * mine.blocks;
    (mine.many ? units_many : units_few) += mine.units;
  }
  total_many = wave_sum64(total_many);
  total_few = wave_sum64(total_few);
  const int32_t um = wave_sum(units_many), uf = wave_sum(units_few);
  if (lane == 0) {
    f->total[0][wave] = total_many;
    f->total[1][wave] = total_few;
    f->units[0][wave] = um;
    f->units[1][wave] = uf;
  }
  if (tid == 0) f->unit.any = false;
  __syncthreads();
  int64_t total[2] = {0, 0}, units[2] = {0, 0};
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      total[k] += f->total[k][w];
      units[k] += f->units[k][w];
    }
  const int32_t per_many = blocks_per_slice(total[0], units[0], a.grid_many, LEAST_MANY);
  const int32_t per_few = blocks_per_slice(total[1], units[1], a.grid_few, LEAST_FEW);
  int32_t items_many = 0, items_few = 0;
  for (int s = s0; s < s1; ++s) {
    const Count c = per == 1 ? mine : look(s);
    (c.many ? items_many : items_few) += c.units * splits_of(c.blocks, c.many ? per_many : per_few);
  }
  const int32_t scan_many = wave_scan(items_many, lane), scan_few = wave_scan(items_few, lane);
  if (lane == 63) {
    f->items[0][wave] = scan_many;
    f->items[1][wave] = scan_few;
  }
  __syncthreads();
  // workgroups below grid_many take units of many rows, the others those of few
  const bool many = blockIdx.x < a.grid_many;
  const int k = many ? 0 : 1;
  const int32_t item = (int32_t)(many ? blockIdx.x : blockIdx.x - a.grid_many);
  int32_t before = (many ? scan_many - items_many : scan_few - items_few);
  for (int w = 0; w < wave; ++w) before += f->items[k][w];
  if (item >= before && item < before + (many ? items_many : items_few)) {
    int32_t at = before;
    for (int s = s0; s < s1; ++s) {
      const Count c = per == 1 ? mine : look(s);
      if (c.many != many) continue;
      const int32_t splits = splits_of(c.blocks, many ? per_many : per_few);
      const int32_t n = c.units * splits;
      if (item < at + n) {
        const AttnSeq q = a.seqs[s];
        const int32_t i = item - at, rest = i / q.kv_heads;
        Unit u;
        u.problem = q.problem;
        u.seq = q.seq;
        u.head = i % q.kv_heads;
        u.split = rest % splits;
        u.splits = splits;
        u.block = c.units / q.kv_heads - 1 - rest / splits;
        u.slot = (uint32_t)item;
        u.first_slot = (uint32_t)(item - u.split * q.kv_heads);
        u.many = many;
        u.any = true;
        f->unit = u;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
}

// The slices of a unit but the last to arrive leave; true for that one.  Every wave's partial results have gone through to memory
// (device-scope stores, waited for) before one thread counts the workgroup in, so a relaxed count is enough on this hardware; the
// last one reads them with device-scope loads.  It also sets the count back for the next launch.
__device__ __forceinline__ bool last_to_arrive(uint32_t *arrivals, int32_t splits, uint32_t *flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t n = __hip_atomic_fetch_add(arrivals, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = n;
    if (n + 1 == (uint32_t)splits) __hip_atomic_store(arrivals, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *flag + 1 == (uint32_t)splits;
}

// ---------------------------------------------------------------------------
// pages
// ---------------------------------------------------------------------------
// Sixteen consecutive keys from a multiple of 16 on lie in one page.  Page numbers are read through the scalar cache (nothing writes the
// table while the kernel runs), a step ahead of the keys and values that need them.
#define SK_CONSTANT __attribute__((address_space(4)))
struct Pages {
  const int32_t *row;
  int32_t shift, num_pages, columns;
  int64_t page_stride, token_stride;
  __device__ __forceinline__ int32_t page_of(int32_t key) const {  // (key the same in all lanes)
    const int32_t c = key >> shift;
    return c < columns ? ((const SK_CONSTANT int32_t *)(uintptr_t)row)[c] : -1;
  }
  __device__ __forceinline__ bool there(int32_t page) const { return (uint32_t)page < (uint32_t)num_pages; }
  // element offset of a key in a page that is there
  __device__ __forceinline__ int64_t offset(int32_t page, int32_t key) const {
    return (int64_t)page * page_stride + (int64_t)(key & ((1 << shift) - 1)) * token_stride;
  }
};

// The softmax of a row, piece after piece: with m the maximum so far and l = sum exp2(s - m), a piece with maximum m' makes
// M = max(m, m'), l = l exp2(m - M) + sum exp2(s - M), and the outputs so far are scaled by the same exp2(m - M).  A row that
// has seen nothing has m = -inf; exp2 is then taken relative to 0, so that it stays at l = 0.
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }

// Whether the token at position p sees key j.
__device__ __forceinline__ bool sees(int32_t p, int32_t j, int32_t window, int32_t sinks) {
  return j <= p && (window == 0 || p - j < window || j < sinks);
}

// ---------------------------------------------------------------------------
// few rows: 16 rows, keys shared among the waves
// ---------------------------------------------------------------------------
// A row of LDS that holds a key's values: a power of two of bytes; pairs of 16-byte pieces turned over with the row, so that the rows of
// a transposing read (four or eight of them, 32 or 64 bytes of each) lie in different banks.
template <int DP>
struct ValueRows {
  static constexpr int BYTES = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;
  static __device__ __forceinline__ int at(int row, int byte) {
    const int turn = BYTES == 128 ? (row >> 1) & 3 : row & 7;
    return row * BYTES + (byte ^ (turn << 5));
  }
};

template <int DT, int DP>
__device__ __forceinline__ void attend_few(const AttnArgs &a, const AttnDev &P, const Unit &u, unsigned char *lds, uint32_t *flag) {
  constexpr int KS = DP / 32, NB = DP / 16, PR = DP / 8, VI = PR / 2;  // VI pieces of values per lane and block of keys
  using VR = ValueRows<DP>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const Step st = step_of(P.lengths + u.seq, P.first_row + u.seq, P.rows, P.max_new, (int64_t)P.columns << P.page_shift);
  const int32_t all_rows = st.fresh * P.group, row0 = u.block * ROWS_FEW, rows = min(ROWS_FEW, all_rows - row0);
  const int32_t p0 = st.behind + row0 / P.group, p1 = st.behind + (row0 + rows - 1) / P.group;
  const Span span = span_of<KEYS_FEW>(p0, p1, P.window, P.sinks);
  const int32_t b0 = (int32_t)((int64_t)span.blocks * u.split / u.splits), b1 = (int32_t)((int64_t)span.blocks * (u.split + 1) / u.splits);

  const int32_t my_row = row0 + min(c, rows - 1);
  const int32_t my_token = my_row / P.group, my_head = u.head * P.group + my_row % P.group;
  const int32_t my_pos = c < rows ? st.behind + my_token : -1;
  const char *q = (const char *)P.q + 2 * ((int64_t)(st.first + my_token) * P.q_row + (int64_t)my_head * P.q_head);
  u32x4 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int e = 32 * s + 8 * g;
    qf[s] = load16(c < rows && e < P.dim ? (const void *)(q + 2 * e) : (const void *)g_zeros);
  }
  const Pages pages{P.table + (int64_t)u.seq * P.columns, P.page_shift, P.num_pages, P.columns, P.page_stride, P.token_stride};
  const char *kh = (const char *)P.k + 2 * (int64_t)u.head * P.head_stride, *vh = (const char *)P.v + 2 * (int64_t)u.head * P.head_stride;
  auto key_of = [&](int32_t b) { return b < span.sink_blocks ? b * KEYS_FEW : span.low + (b - span.sink_blocks) * KEYS_FEW; };

  unsigned char *mine = lds + wave * (KEYS_FEW * VR::BYTES);
  f32x4 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;

  u32x4 kf[2][KS], vf[VI];
  int32_t page[2];  // of the block that is loaded next
  auto look = [&](int32_t b) {
    const int32_t key0 = key_of(min(b, b1 - 1));
    page[0] = pages.page_of(key0);
    page[1] = pages.page_of(key0 + 16);
  };
  auto load = [&](int32_t b) -> uint32_t {  // which halves are there
    const int32_t key0 = key_of(b);
    uint32_t present = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int32_t key = key0 + 16 * half;
      const bool there = pages.there(page[half]);
      const int64_t off = pages.offset(page[half], key);
      present |= there ? 1u << half : 0u;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int e = 32 * s + 8 * g;
        kf[half][s] = load16(there && e < P.dim ? (const void *)(kh + 2 * (off + c * P.token_stride + e)) : (const void *)g_zeros);
      }
#pragma unroll
      for (int i = 0; i < VI / 2; ++i) {
        const int n = (i + half * (VI / 2)) * 64 + lane, row = n / PR, e = n % PR * 8;
        const int32_t j = key0 + row;
        // values that no row sees are not read: what lies there may be anything
        const bool ok = there && e < P.dim && j <= p1 && (P.window == 0 || p0 - j < P.window || j < P.sinks);
        vf[i + half * (VI / 2)] = load16(ok ? (const void *)(vh + 2 * (off + (row & 15) * P.token_stride + e)) : (const void *)g_zeros);
      }
    }
    return present;
  };
  uint32_t present = 0;
  if (b0 + wave < b1) {
    look(b0 + wave);
    present = load(b0 + wave);
    look(b0 + wave + 4);
  }
  for (int32_t b = b0 + wave; b < b1; b += 4) {
    const int32_t key0 = key_of(b);
    const uint32_t now = present;
    f32x4 s[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      s[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) mma16<DT>(kf[half][k], qf[k], s[half]);
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int n = i * 64 + lane, row = n / PR, e = n % PR * 8;
      *(u32x4 *)(mine + VR::at(row, 2 * e)) = vf[i];
    }
    if (b + 4 < b1) {
      present = load(b + 4);
      look(b + 8);
    }
    // lane (g, c) has the scores of row c and keys key0 + 16 half + 4 g + i
    float top = -__builtin_inff();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t j = key0 + 16 * half + 4 * g + i;
        s[half][i] = (now >> half & 1) && sees(my_pos, j, P.window, P.sinks) ? s[half][i] * P.scale_log2 : -__builtin_inff();
        top = fmaxf(top, s[half][i]);
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float next = fmaxf(m, top), base = base_of(next), keep = exp2_fast(m - base);
    m = next;
    float sum = 0.f;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[half][i] = exp2_fast(s[half][i] - base);
        sum += s[half][i];
      }
    l = l * keep + sum;
    const u32x4 pf = {pack2<DT>(s[0][0], s[0][1]), pack2<DT>(s[0][2], s[0][3]), pack2<DT>(s[1][0], s[1][1]), pack2<DT>(s[1][2], s[1][3])};
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int byte = 2 * (16 * i + 4 * (c & 3)), row = 4 * g + (c >> 2);
      const u32x2 lo = read_transposed(mine + VR::at(row, byte)), hi = read_transposed(mine + VR::at(row + 16, byte));
      o[i] *= keep;
      mma16<DT>(u32x4{lo.x, lo.y, hi.x, hi.y}, pf, o[i]);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the waves' results together: [wave][row] maximum and sum, [wave][row][element] outputs relative to the common maximum
  float *stats = (float *)(lds + 4 * KEYS_FEW * VR::BYTES);
  if (g == 0) {
    stats[wave * 32 + c] = m;
    stats[wave * 32 + 16 + c] = l;
  }
  __syncthreads();
  float top = -__builtin_inff();
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, stats[w * 32 + c]);
  const float part = exp2_fast(m - base_of(top));
  static_assert(KEYS_FEW * VR::BYTES >= ROWS_FEW * DP * 4, "a wave's outputs fit its values' place");
  float *out = (float *)mine;
#pragma unroll
  for (int i = 0; i < NB; ++i) *(f32x4 *)(out + c * DP + 16 * i + 4 * g) = o[i] * part;
  __syncthreads();
  float *ws = a.ws_few + (int64_t)u.slot * part_floats(ROWS_FEW, DP);
  for (int n = tid; n < rows * (DP / 4); n += CACHE_THREADS) {
    const int r = n / (DP / 4), e = n % (DP / 4) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    float big = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      v += *(const f32x4 *)((const float *)(lds + w * (KEYS_FEW * VR::BYTES)) + r * DP + e);
      big = fmaxf(big, stats[w * 32 + r]);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += stats[w * 32 + 16 + r] * exp2_fast(stats[w * 32 + r] - base_of(big));
    if (u.splits == 1) {
      const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
      const int32_t row = row0 + r;
      char *dst = (char *)P.out + 2 * ((int64_t)(st.first + row / P.group) * P.out_row + (int64_t)(u.head * P.group + row % P.group) * P.out_head + e);
      if (e < P.dim) store8(dst, u32x2{pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv)});
    } else {
      store_shared(ws + r * DP + e, f32x2{v.x, v.y});
      store_shared(ws + r * DP + e + 2, f32x2{v.z, v.w});
      if (e == 0) store_shared(ws + ROWS_FEW * DP + 2 * r, f32x2{big, sum});
    }
  }
  if (u.splits == 1) return;
  if (!last_to_arrive(a.arrivals + a.grid_many + u.first_slot, u.splits, flag)) return;
  // the slices in order: the result does not depend on who came last
  const float *ws0 = a.ws_few + (int64_t)u.first_slot * part_floats(ROWS_FEW, DP);
  const int64_t step = (int64_t)P.kv_heads * part_floats(ROWS_FEW, DP);
  for (int n = tid; n < rows * (DP / 4); n += CACHE_THREADS) {
    const int r = n / (DP / 4), e = n % (DP / 4) * 4;
    float big = -__builtin_inff(), sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < u.splits; ++s) {
      const float *w = ws0 + s * step;
      const f32x2 ms = load_shared(w + ROWS_FEW * DP + 2 * r), x = load_shared(w + r * DP + e), y = load_shared(w + r * DP + e + 2);
      const float next = fmaxf(big, ms.x), keep = exp2_fast(big - base_of(next)), mul = exp2_fast(ms.x - base_of(next));
      sum = sum * keep + ms.y * mul;
      v = v * keep + f32x4{x.x, x.y, y.x, y.y} * mul;
      big = next;
    }
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
    const int32_t row = row0 + r;
    char *dst = (char *)P.out + 2 * ((int64_t)(st.first + row / P.group) * P.out_row + (int64_t)(u.head * P.group + row % P.group) * P.out_head + e);
    if (e < P.dim) store8(dst, u32x2{pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv)});
  }
}

// ---------------------------------------------------------------------------
// many rows: 128 rows, 32 for each wave, keys through LDS
// ---------------------------------------------------------------------------
// A row of LDS that holds a key: its 16-byte pieces turned over with the row, so that 16 lanes that read one piece of 16 rows meet 16
// different groups of four banks.
template <int DP>
struct KeyRows {
  static constexpr int BYTES = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;
  static __device__ __forceinline__ int at(int row, int byte) {
    const int turn = BYTES == 128 ? (row >> 1) & 7 : row & 15;
    return row * BYTES + (byte ^ (turn << 4));
  }
};

template <int DT, int DP>
__device__ __forceinline__ void attend_many(const AttnArgs &a, const AttnDev &P, const Unit &u, unsigned char *lds, uint32_t *flag) {
  constexpr int KS = DP / 16, NB = DP / 32, PR = DP / 8, LI = KEYS_MANY * PR / CACHE_THREADS;  // LI pieces per thread and tile, keys and values each
  using KR = KeyRows<DP>;
  using VR = ValueRows<DP>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, c = lane & 31;
  const Step st = step_of(P.lengths + u.seq, P.first_row + u.seq, P.rows, P.max_new, (int64_t)P.columns << P.page_shift);
  const int32_t all_rows = st.fresh * P.group, row0 = u.block * ROWS_MANY, rows = min(ROWS_MANY, all_rows - row0);
  const int32_t p0 = st.behind + row0 / P.group, p1 = st.behind + (row0 + rows - 1) / P.group;
  const Span span = span_of<KEYS_MANY>(p0, p1, P.window, P.sinks);
  const int32_t b0 = (int32_t)((int64_t)span.blocks * u.split / u.splits), b1 = (int32_t)((int64_t)span.blocks * (u.split + 1) / u.splits);

  const int32_t in_block = wave * 32 + c;
  const bool row_ok = in_block < rows;
  const int32_t my_row = row0 + min(in_block, rows - 1);
  const int32_t my_token = my_row / P.group, my_head = u.head * P.group + my_row % P.group;
  const int32_t my_pos = row_ok ? st.behind + my_token : -1;
  // positions of the wave's rows (uniform)
  const bool wave_ok = wave * 32 < rows;
  const int32_t w0 = st.behind + (row0 + min(wave * 32, rows - 1)) / P.group, w1 = st.behind + (row0 + min(wave * 32 + 31, rows - 1)) / P.group;
  const char *q = (const char *)P.q + 2 * ((int64_t)(st.first + my_token) * P.q_row + (int64_t)my_head * P.q_head);
  u32x4 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int e = 16 * s + 8 * h;
    qf[s] = load16(row_ok && e < P.dim ? (const void *)(q + 2 * e) : (const void *)g_zeros);
  }
  const Pages pages{P.table + (int64_t)u.seq * P.columns, P.page_shift, P.num_pages, P.columns, P.page_stride, P.token_stride};
  const char *kh = (const char *)P.k + 2 * (int64_t)u.head * P.head_stride, *vh = (const char *)P.v + 2 * (int64_t)u.head * P.head_stride;
  auto key_of = [&](int32_t b) { return b < span.sink_blocks ? b * KEYS_MANY : span.low + (b - span.sink_blocks) * KEYS_MANY; };

  unsigned char *ks = lds, *vs = lds + KEYS_MANY * KR::BYTES;
  f32x16 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = -__builtin_inff(), l = 0.f;

  u32x4 kr[LI], vr[LI];
  int32_t page[4];  // of the tile that is loaded next
  auto look = [&](int32_t b) {
    const int32_t key0 = key_of(min(b, b1 - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) page[i] = pages.page_of(key0 + 16 * i);
  };
  auto load = [&](int32_t b) -> uint32_t {  // which of its blocks of 16 keys are there
    const int32_t key0 = key_of(b);
    uint32_t present = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) present |= pages.there(page[i]) ? 1u << i : 0u;
#pragma unroll
    for (int i = 0; i < LI; ++i) {
      const int n = i * CACHE_THREADS + tid, row = n / PR, e = n % PR * 8;
      const int block = (i * 4 + wave) * 4 / PR;  // the wave's pieces lie in one block of 16 keys
      const int32_t id = block == 0 ? page[0] : block == 1 ? page[1] : block == 2 ? page[2] : page[3];
      const int32_t j = key0 + row;
      const int64_t at = 2 * (pages.offset(id, key0 + 16 * block) + (row & 15) * P.token_stride + e);
      const bool there = pages.there(id) && e < P.dim;
      kr[i] = load16(there ? (const void *)(kh + at) : (const void *)g_zeros);
      // values that no row sees are not read: what lies there may be anything
      const bool seen = j <= p1 && (P.window == 0 || p0 - j < P.window || j < P.sinks);
      vr[i] = load16(there && seen ? (const void *)(vh + at) : (const void *)g_zeros);
    }
    return present;
  };
  uint32_t present = 0;
  if (b0 < b1) {
    look(b0);
    present = load(b0);
    look(b0 + 1);
  }
  for (int32_t b = b0; b < b1; ++b) {
    const int32_t key0 = key_of(b);
    const uint32_t now = present;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LI; ++i) {
      const int n = i * CACHE_THREADS + tid, row = n / PR, e = n % PR * 8;
      *(u32x4 *)(ks + KR::at(row, 2 * e)) = kr[i];
      *(u32x4 *)(vs + VR::at(row, 2 * e)) = vr[i];
    }
    __syncthreads();
    if (b + 1 < b1) {
      present = load(b + 1);
      look(b + 2);
    }
    // whether any row of the wave sees any of these keys
    const bool use = wave_ok && key0 <= w1 && (P.window == 0 || (int64_t)w0 - (key0 + KEYS_MANY - 1) < P.window || key0 < P.sinks);
    if (!use) continue;
    const bool whole = now == 15 && key0 + KEYS_MANY - 1 <= w0 && (P.window == 0 || (int64_t)w1 - key0 < P.window);
    f32x16 s[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s[half][j] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const u32x4 kf = *(const u32x4 *)(ks + KR::at(32 * half + c, 2 * (16 * k + 8 * h)));
        mma32<DT>(kf, qf[k], s[half]);
      }
    }
    // lane (h, c) has the scores of row c and keys key0 + 32 half + 8 (i / 4) + 4 h + i % 4
    float top = -__builtin_inff();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[half][i] *= P.scale_log2;
        if (!whole) {
          const int32_t j = key0 + 32 * half + 8 * (i / 4) + 4 * h + i % 4;
          s[half][i] = (now >> (2 * half + i / 8) & 1) && sees(my_pos, j, P.window, P.sinks) ? s[half][i] : -__builtin_inff();
        }
        top = fmaxf(top, s[half][i]);
      }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float next = fmaxf(m, top), base = base_of(next), keep = exp2_fast(m - base);
    m = next;
    float sum = 0.f;
    u32x4 pf[4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[half][i] = exp2_fast(s[half][i] - base);
        sum += s[half][i];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
        pf[2 * half + t] = u32x4{pack2<DT>(s[half][8 * t], s[half][8 * t + 1]), pack2<DT>(s[half][8 * t + 2], s[half][8 * t + 3]),
                                 pack2<DT>(s[half][8 * t + 4], s[half][8 * t + 5]), pack2<DT>(s[half][8 * t + 6], s[half][8 * t + 7])};
    }
    l = l * keep + sum;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      o[i] *= keep;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int row = 16 * t + 4 * h + ((lane & 15) >> 2), byte = 2 * (32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3));
        const u32x2 lo = read_transposed(vs + VR::at(row, byte)), hi = read_transposed(vs + VR::at(row + 8, byte));
        mma32<DT>(u32x4{lo.x, lo.y, hi.x, hi.y}, pf[t], o[i]);
      }
    }
  }
  l += __shfl_xor(l, 32);

  if (u.splits > 1) {
    // partial results as they stand in the registers: [wave][register pair][lane], then maximum and sum of each row
    float *ws = a.ws_many + (int64_t)u.slot * part_floats(ROWS_MANY, DP);
    if (wave_ok) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) store_shared(ws + ((wave * NB + i) * 8 + j) * 128 + 2 * lane, f32x2{o[i][2 * j], o[i][2 * j + 1]});
      if (h == 0) store_shared(ws + ROWS_MANY * DP + 2 * in_block, f32x2{m, l});
    }
    if (!last_to_arrive(a.arrivals + u.first_slot, u.splits, flag)) return;
    if (!wave_ok) return;
    const float *ws0 = a.ws_many + (int64_t)u.first_slot * part_floats(ROWS_MANY, DP);
    const int64_t step = (int64_t)P.kv_heads * part_floats(ROWS_MANY, DP);
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    for (int s = 0; s < u.splits; ++s) {
      const float *w = ws0 + s * step;
      const f32x2 ms = load_shared(w + ROWS_MANY * DP + 2 * in_block);
      const float next = fmaxf(m, ms.x), keep = exp2_fast(m - base_of(next)), mul = exp2_fast(ms.x - base_of(next));
      l = l * keep + ms.y * mul;
      m = next;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const f32x2 x = load_shared(w + ((wave * NB + i) * 8 + j) * 128 + 2 * lane);
          o[i][2 * j] = o[i][2 * j] * keep + x.x * mul;
          o[i][2 * j + 1] = o[i][2 * j + 1] * keep + x.y * mul;
        }
    }
  }
  if (!row_ok) return;
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
  char *dst = (char *)P.out + 2 * ((int64_t)(st.first + my_token) * P.out_row + (int64_t)my_head * P.out_head);
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int e = 32 * i + 8 * b + 4 * h;
      if (e < P.dim)
        store8(dst + 2 * e, u32x2{pack2<DT>(o[i][4 * b] * inv, o[i][4 * b + 1] * inv), pack2<DT>(o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv)});
    }
}

template <int DT, int DP>
__global__ void __launch_bounds__(CACHE_THREADS, DP <= 128 ? 2 : 1) sk_attend(AttnArgs a) {
  constexpr int FEW = 4 * KEYS_FEW * ValueRows<DP>::BYTES + 4 * 2 * ROWS_FEW * 4, MANY = KEYS_MANY * (KeyRows<DP>::BYTES + ValueRows<DP>::BYTES);
  __shared__ __attribute__((aligned(16))) unsigned char lds[FEW > MANY ? FEW : MANY];
  __shared__ FindScratch found;
  __shared__ uint32_t flag;
  find_unit(a, &found);
  if (!found.unit.any) return;
  const Unit u = found.unit;
  const AttnDev &P = a.problems[__builtin_amdgcn_readfirstlane(u.problem)];
  Unit v;  // the same in scalar registers
  v.problem = 0;
  v.seq = __builtin_amdgcn_readfirstlane(u.seq);
  v.head = __builtin_amdgcn_readfirstlane(u.head);
  v.block = __builtin_amdgcn_readfirstlane(u.block);
  v.split = __builtin_amdgcn_readfirstlane(u.split);
  v.splits = __builtin_amdgcn_readfirstlane(u.splits);
  v.slot = __builtin_amdgcn_readfirstlane(u.slot);
  v.first_slot = __builtin_amdgcn_readfirstlane(u.first_slot);
  v.many = v.any = true;
  if (__builtin_amdgcn_readfirstlane((int)u.many))
    attend_many<DT, DP>(a, P, v, lds, &flag);
  else
    attend_few<DT, DP>(a, P, v, lds, &flag);
}

}  // namespace sk
