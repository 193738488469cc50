// Device code of libsk_cache.so (gfx950 / CDNA4 only): attention over paged caches, and what its kernels share with cache_rows.hip.h.
#pragma once

#include "device.hip.h"

#include <type_traits>

#include "cache_internal.h"
#include "cache_units.h"

namespace sk {

// ---------------------------------------------------------------------------
// which unit of work a workgroup takes
// ---------------------------------------------------------------------------
// The lengths are in device memory, so the units (a block of rows of a key-value head of a sequence, and a slice of its
// keys) are counted on the device: every workgroup looks at all sequences of the launch and finds its own unit from the sums
// before it; workgroups beyond the last leave.  Units of many rows come first, those of late rows (which see the most) before those of early
// ones; key-value heads vary fastest, so that with eight of them each has a die (and its L2) of its own.

__device__ __forceinline__ Step step_of(const AttnSeq &q) { return step_of(q, load_i32(q.first), load_i32(q.first + 1), load_i32(q.length)); }

struct Unit {
  int32_t problem, seq;
  int32_t head, block;          // key-value head, block of rows
  int32_t split, splits;
  uint32_t slot;                // this workgroup's place in the workspace
  uint32_t first_slot;          // of the unit's first slice: also its arrival counter
  Step step;
  bool many, any;
};

struct AttnArgs {
  const AttnDev *problems;
  const AttnSeq *seqs;
  int32_t sequences;
  int32_t workgroups;  // that the card runs at a time
  uint32_t grid;       // workgroups of the launch
  uint32_t slots_many, slots_few;  // places of the workspace for slices of either kind
  float *ws_many, *ws_few;
  uint32_t *arrivals;  // slots_many, then as many as there are for few; zero between launches
};

// n / d for 0 <= n < 2^31.
__device__ __forceinline__ int32_t fast_div(int32_t n, FastDiv d) { return (int32_t)((uint64_t)(uint32_t)n * d.mul >> d.shift); }

struct FindScratch {
  int64_t work[4];  // per wave
  int32_t items[2][4], cut[2][4];
  Unit unit;
};

// Unit number i of a sequence's, whose slices have the places from `slot` on.
__device__ __forceinline__ Unit unit_of(const AttnSeq &q, const Step &s, const Count &c, int32_t splits, int32_t i, int32_t slot) {
  const int32_t rest = (int32_t)((uint32_t)i / (uint32_t)q.kv_heads), block = (int32_t)((uint32_t)rest / (uint32_t)splits);
  Unit u;
  u.problem = q.problem;
  u.seq = q.seq;
  u.head = i - rest * q.kv_heads;
  u.split = rest - block * splits;
  u.splits = splits;
  u.block = c.row_blocks - 1 - block;
  u.slot = (uint32_t)(slot + i);
  u.first_slot = (uint32_t)(slot + i - u.split * q.kv_heads);
  u.step = s;
  u.many = c.many;
  u.any = true;
  return u;
}
__device__ __forceinline__ Unit unit_in_lane(const Unit &u, int lane) {
  Unit r;
  r.problem = lane_of(u.problem, lane);
  r.seq = lane_of(u.seq, lane);
  r.head = lane_of(u.head, lane);
  r.block = lane_of(u.block, lane);
  r.split = lane_of(u.split, lane);
  r.splits = lane_of(u.splits, lane);
  r.slot = (uint32_t)lane_of((int32_t)u.slot, lane);
  r.first_slot = (uint32_t)lane_of((int32_t)u.first_slot, lane);
  r.step.first = lane_of(u.step.first, lane);
  r.step.fresh = lane_of(u.step.fresh, lane);
  r.step.length = lane_of(u.step.length, lane);
  r.step.behind = lane_of(u.step.behind, lane);
  r.many = lane_of((int32_t)u.many, lane) != 0;
  r.any = true;
  return r;
}

// The unit, or slice of one, that a workgroup takes: those of many rows first.  MANY: there may be such.
template <bool MANY, bool WIDE>
__device__ __forceinline__ Unit find_unit(const AttnArgs &a, FindScratch *f) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t item = (int32_t)blockIdx.x;
  if (a.sequences <= 64) {
    // a sequence per lane, every wave for itself
    AttnSeq q{};
    q.kv_heads = 1;
    Step s{};
    Count c{0, 0, 0, false};
    if (lane < a.sequences) {
      q = a.seqs[lane];
      s = step_of(q);
      c = count_units<MANY, WIDE>(s, q);
    }
    const int32_t units = lane_of(wave_scan(items_of(c, 1)), 63);
    const int64_t work = lane_of(wave_scan(work_of(c)), 63);
    int32_t most = even_share(work, a.workgroups), splits = splits_of(c, most);
    // Few units: slices as short as leaves all of them running at once.  (A slice costs its workgroup 5 us besides the keys: six caches of 50
    // to 120 thousand tokens take 7 and 5 % longer in two and four rounds of slices, 96 caches with a window of 1024 12 and 32 %.)
    for (int i = 0; i < 8 && units <= a.workgroups / 2 && lane_of(wave_scan(c.units * splits), 63) > a.workgroups; ++i) {
      most += most / 8 + 1;
      splits = splits_of(c, most);
    }
    // units and slices, and those of them that are slices, up to and with this lane's
    int32_t n_many, n_few, upto_many, upto_few, cut_many, cut_few;
    auto sums = [&]() {
      const int32_t n = items_of(c, splits);
      n_many = MANY && c.many ? n : 0, n_few = n - n_many;
      upto_many = MANY ? wave_scan(n_many) : 0, upto_few = wave_scan(n_few);
      cut_many = MANY ? wave_scan(splits > 1 ? n_many : 0) : 0, cut_few = wave_scan(splits > 1 ? n_few : 0);
    };
    sums();
    if (!slices_fit(lane_of(upto_many + upto_few, 63), lane_of(cut_many, 63), lane_of(cut_few, 63), a.grid, a.slots_many, a.slots_few)) {
      splits = 1;
      sums();
    }
    const int32_t all_many = MANY ? lane_of(upto_many, 63) : 0;
    const bool many = MANY && item < all_many;
    if (!many) item -= all_many;
    const int32_t upto = many ? upto_many : upto_few, mine = many ? n_many : n_few;
    const uint64_t hit = __ballot(item >= upto - mine && item < upto);
    Unit u{};
    u.any = hit != 0;
    if (!u.any) return u;
    const int who = __builtin_ctzll(hit);
    return unit_in_lane(unit_of(q, s, c, splits, item - (upto - mine), (many ? cut_many : cut_few) - mine), who);
  }
  // a run of sequences per thread
  const int per_thread = (a.sequences + CACHE_THREADS - 1) / CACHE_THREADS;
  const int s0 = tid * per_thread, s1 = min(s0 + per_thread, a.sequences);
  AttnSeq q{};
  Step s{};
  Count c{0, 0, 0, false};
  auto look = [&](int i) {
    q = a.seqs[i];
    s = step_of(q);
    c = count_units<MANY, WIDE>(s, q);
  };
  int64_t work = 0;
  for (int i = s0; i < s1; ++i) {
    look(i);
    work += work_of(c);
  }
  work = lane_of(wave_scan(work), 63);
  if (lane == 0) f->work[wave] = work;
  if (tid == 0) f->unit.any = false;
  __syncthreads();
  int32_t most = even_share(f->work[0] + f->work[1] + f->work[2] + f->work[3], a.workgroups);
  int32_t n[2], cut[2], upto[2], cut_upto[2];  // of many rows and of few
  for (int round = 0; round < 2; ++round) {
    n[0] = n[1] = cut[0] = cut[1] = 0;
    for (int i = s0; i < s1; ++i) {
      if (per_thread > 1) look(i);
      const int32_t splits = splits_of(c, most), here = items_of(c, splits), sliced = splits > 1 ? here : 0;
      n[0] += MANY && c.many ? here : 0, cut[0] += MANY && c.many ? sliced : 0;
      n[1] += MANY && c.many ? 0 : here, cut[1] += MANY && c.many ? 0 : sliced;
#pragma unroll
      for (int k = 0; k < 2; ++k) n[k] = min(n[k], MOST_ITEMS), cut[k] = min(cut[k], MOST_ITEMS);
    }
#pragma unroll
    for (int k = MANY ? 0 : 1; k < 2; ++k) {
      upto[k] = wave_scan(n[k]);
      cut_upto[k] = wave_scan(cut[k]);
      if (lane == 63) {
        f->items[k][wave] = min(upto[k], MOST_ITEMS);
        f->cut[k][wave] = min(cut_upto[k], MOST_ITEMS);
      }
    }
    __syncthreads();
    auto all = [](const int32_t (&w)[4]) { return w[0] + w[1] + w[2] + w[3]; };
    if (slices_fit((MANY ? all(f->items[0]) : 0) + all(f->items[1]), MANY ? all(f->cut[0]) : 0, all(f->cut[1]), a.grid, a.slots_many, a.slots_few)) break;
    most = 0x7ffffffe;
    __syncthreads();
  }
  const int32_t all_many = MANY ? f->items[0][0] + f->items[0][1] + f->items[0][2] + f->items[0][3] : 0;
  const bool many = MANY && item < all_many;
  if (!many) item -= all_many;
  const int32_t mine = many ? n[0] : n[1];
  int32_t before = (many ? upto[0] : upto[1]) - mine, slot = many ? cut_upto[0] - cut[0] : cut_upto[1] - cut[1];
  for (int w = 0; w < wave; ++w) {
    before += f->items[many ? 0 : 1][w];
    slot += f->cut[many ? 0 : 1][w];
  }
  if (item >= before && item < before + mine) {
    int32_t at = before;
    for (int i = s0; i < s1; ++i) {
      if (per_thread > 1) look(i);
      if (c.many != many) continue;
      const int32_t splits = splits_of(c, most), here = items_of(c, splits);
      if (item < at + here) {
        f->unit = unit_of(q, s, c, splits, item - at, slot);
        break;
      }
      at += here;
      slot += splits > 1 ? here : 0;
    }
  }
  __syncthreads();
  if (!f->unit.any) return f->unit;
  return unit_in_lane(f->unit, 0);
}

// ---------------------------------------------------------------------------
// pages
// ---------------------------------------------------------------------------
// Sixteen consecutive keys from a multiple of 16 on lie in one page.  Page numbers are read through the scalar cache (nothing writes the
// table while the kernel runs), a step ahead of the keys and values that need them; addresses are a scalar base for the sixteen keys and an
// offset per lane that never changes.
struct Pages {
  const int32_t *row;
  int32_t shift, num_pages, columns;
  int64_t page_stride, token_stride;
  __device__ __forceinline__ int32_t page_of(int32_t key) const {  // (key the same in all lanes)
    const int32_t c = column_of(key, shift, columns);
    return c >= 0 ? ((const SK_CONSTANT int32_t *)(uintptr_t)row)[c] : -1;
  }
  __device__ __forceinline__ bool there(int32_t page) const { return (uint32_t)page < (uint32_t)num_pages; }
  // Byte offset of a key.  Where its page is not there, of one in page 0, whose memory can be read: what is read there does not enter a result.
  __device__ __forceinline__ int64_t bytes(int32_t page, int32_t key) const {
    return 2 * ((int64_t)(there(page) ? page : 0) * page_stride + (int64_t)(key & ((1 << shift) - 1)) * token_stride);
  }
};

// The softmax of a row, piece after piece: weights are exp2(s - m) with a base m, l is their sum.  m is the maximum of the first piece
// that the row sees anything of; a later piece moves it (and l and the outputs so far are scaled by exp2(m - new m)) only where its
// maximum is more than RISE above it: until then weights of up to 2^RISE are as exact in 16 bits as those up to 1, and sums in fp32
// do not mind.  (With rows of random scores some row of 32 meets a new maximum in more than half of the steps of a prompt.)  A row that
// has seen nothing has m = -inf; exp2 is then taken relative to 0, so that it stays at l = 0.
constexpr float RISE = 8.f;
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }
// A weight is exp2(fma(score, scale, -base)), and the base a score times the scale, rounded: all weights of a row are off by the same factor, which
// the division by their sum takes out.  From scores of 2^24 on it is no small one (half a unit of the base in the exponent).  Where a row's
// base is beyond FAR scores are rounded to products first, as the base was: the difference is exact then, and no weight exceeds 2^RISE.
constexpr float FAR = 65536.f;
__device__ __forceinline__ bool any_far(float base) { return __builtin_expect(__ballot(fabsf(base) >= FAR) != 0, 0); }
__device__ __forceinline__ float rounded_difference(float score, float scale, float base) {
#pragma clang fp contract(off)
  const float product = score * scale;
  return product - base;
}
// Weights are rounded to 16 bits for the matrix units.  f16 has nothing below 2^-25: there they are 2^7 times as large (with RISE up to 2^15, and 65504
// is the largest number), so that weights down to 2^-32 of the base count, and are as exact as others down to 2^-21.  Sums are larger by as much.
template <int DT>
constexpr float LIFT = DT == SK_F16 ? 7.f : 0.f;
__device__ __forceinline__ float inverse(float sum) { return sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum); }  // (nothing seen: 0)

// Values that some rows of a unit see and others do not must not reach the others, whatever they are; finite ones do not (their
// weight is 0), but 0 * inf is NaN.  Where a step's keys are not seen by all rows alike, values that are not finite are taken out
// on the way into LDS and, if there were any, added to the rows that see them at the end.  A row that sees one ends up not finite.
template <int DT>
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {  // 0xffff in each half that is not finite
  constexpr uint32_t E = DT == SK_BF16 ? 0x7f80u : 0x7c00u;
  return ((w & E) == E ? 0xffffu : 0u) | ((w >> 16 & E) == E ? 0xffff0000u : 0u);
}
template <int DT>
__device__ __forceinline__ bool clean(u32x4 &v) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t odd = odd_halves<DT>(v[i]);
    any |= odd;
    v[i] &= ~odd;
  }
  return any != 0;
}
// The sum of what is not finite in four elements (at `v` in the cache's first page) of the values that a row sees in some blocks of keys.  Rare, so
// it reads them again from memory, key by key.
template <int DT, class K>
__device__ __forceinline__ f32x4 odd_sum(const Pages &pages, const char *v, int32_t b0, int32_t b1, int32_t step, const K &key_of, int32_t keys, int32_t pos,
                                         int32_t window, int32_t sinks) {
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int32_t b = b0; b < b1; b += step)
#pragma unroll 1
    for (int32_t i = 0, j = key_of(b); i < keys; ++i, j = key_behind(j, 1)) {
      const int32_t page = pages.page_of(j);
      if (!pages.there(page) || !sees(pos, j, window, sinks)) continue;
      const u32x2 w = *(const u32x2 SK_GLOBAL *)(uintptr_t)(v + pages.bytes(page, j));
      const uint32_t lo = w.x & odd_halves<DT>(w.x), hi = w.y & odd_halves<DT>(w.y);
      sum += f32x4{elem<DT>(lo & 0xffffu), elem<DT>(lo >> 16), elem<DT>(hi & 0xffffu), elem<DT>(hi >> 16)};
    }
  return sum;
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

// Nothing moves across.  Matrix instructions whose LDS operands are to be read a group ahead need it: left alone the scheduler puts every read
// right above its use, and a wave waits out the way to LDS and back each time.
__device__ __forceinline__ void fixed_order() { __builtin_amdgcn_sched_barrier(0); }

// N pieces of 16 bytes a lane from memory into LDS: lane i's arrive at lds_addr + 1024 n + 16 i.  The instruction's own offset counts on both
// sides, so the lanes' offsets are lowered by as much and the descriptor begins DMA_FRONT bytes in front.  What lies outside the descriptor
// arrives as zeros.  In one statement, opened with the wait states that scalar registers written by vector instructions want before a memory
// instruction reads them; the compiler does not know of the loads, so they are waited for by hand (wait_dma).
constexpr int DMA_FRONT = 3072;
constexpr uint32_t DMA_OUTSIDE = 0x80000000u;
template <int N>
__device__ __forceinline__ void dma(__amdgpu_buffer_rsrc_t desc, const uint32_t (&at)[N], uint32_t lds_addr) {
  static_assert(N == 2 || N == 4, "written out for these");
  if constexpr (N == 4)
    asm volatile("s_nop 4\n\t"
                 "buffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %1, %4, 0 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %2, %4, 0 offen offset:2048 lds\n\t"
                 "buffer_load_dwordx4 %3, %4, 0 offen offset:3072 lds"
                 :
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(desc), "{m0}"(lds_addr)
                 : "memory");
  else
    asm volatile("s_nop 4\n\t"
                 "buffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen offset:1024 lds"
                 :
                 : "v"(at[0]), "v"(at[1]), "s"(desc), "{m0}"(lds_addr)
                 : "memory");
}
// Until all but the last N loads are there.
template <int N>
__device__ __forceinline__ void wait_dma() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int DT>
__device__ __forceinline__ u32x4 load_query(const void *p, bool ok, bool negate) {
  u32x4 v = load16(ok ? p : (const void *)g_zeros);
  if (negate) v ^= 0x80008000u;
  return v;
}

// Sixteen rows (a group's query heads, of one token mostly) against a run of keys.  Scores of 32 keys and 16 rows as K Q^T, so that a lane holds
// scores of one row: its maximum and sum are one permutation across lanes 16 and one across 32 apart, and its weights are, as they stand, the
// right operand of V^T P.  Keys go from memory straight into the left operand's registers (no wave needs another's), a step ahead; values
// have to be turned round, so they go by direct loads into LDS that is the wave's own and come back by transposing reads: no barrier in the
// loop.  The four waves take steps in turn and add up through LDS at the end.  Bound by memory: keys and values are read once, and what
// matters is bytes in flight: three workgroups of four waves on a compute unit, each wave with 16 KB (heads of 128) on their way.  Six caches
// of 50 to 120 thousand tokens, 8 heads of 128: 1.6 GB in 278 us, 5.8 TB/s (a streaming read 6.6, a copy 5.2); 96 caches of up to 8000 tokens
// 71.6 us, 4.5 TB/s with the ends of units; one of 800 tokens 7.7 us a call, of which 2 are finding the unit and 2 the way of the first keys.
template <int DT, int DP>
__device__ __forceinline__ void attend_few(const AttnArgs &a, const SK_CONSTANT AttnDev &P, const Unit &u, unsigned char *lds, uint32_t *flag) {
  constexpr int64_t SLOT = part_floats(ROWS_FEW, DP <= 128 ? 128 : 256);
  using VR = ValueRows<DP>;
  constexpr int KS = DP / 32, NB = DP / 16, SLOTS = VR::BYTES / 16, VH = SLOTS / 4;  // VH KB of values per 16 keys
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const Step &st = u.step;
  const int32_t row0 = u.block * ROWS_FEW, rows = min(ROWS_FEW, st.fresh * P.group - row0);
  const FastDiv by_group = {P.by_group.mul, P.by_group.shift};
  const int32_t p0 = st.behind + fast_div(row0, by_group), p1 = st.behind + fast_div(row0 + rows - 1, by_group);
  const int32_t window = P.window, sinks = P.sinks, dim = P.dim;
  const Span span = span_of<KEYS_FEW>(p0, p1, window, sinks);
  const bool two_spans = window && sinks > span.low;  // a row may see two runs of keys in a block
  const int32_t b0 = slice_start(span.blocks, u.split, u.splits), b1 = slice_start(span.blocks, u.split + 1, u.splits);

  const Pages pages{P.table + (int64_t)u.seq * P.columns, P.page_shift, P.num_pages, P.columns, P.page_stride, P.token_stride};
  const char *kh = (const char *)P.k + 2 * (int64_t)u.head * P.head_stride, *vh = (const char *)P.v + 2 * (int64_t)u.head * P.head_stride;
  auto key_of = [&](int32_t b) { return block_key<KEYS_FEW>(span, b); };
  // Offsets of this lane's pieces of 16 keys.  Keys go into registers: pieces beyond the head's end are read from its start and count as zeros.
  // Values go into LDS (see dma), a wave's to a place of its own: there such pieces come as zeros.
  constexpr int VI = VH < 4 ? VH : 4;  // loads per statement
  uint32_t ko[KS], vo[VH];
#pragma unroll
  for (int s = 0; s < KS; ++s) ko[s] = 2u * (uint32_t)(c * P.token_stride + (32 * s + 8 * g < dim ? 32 * s + 8 * g : 0));
#pragma unroll
  for (int i = 0; i < VH; ++i) {
    const int key = i * (64 / SLOTS) + lane / SLOTS, e = (VR::at(key, lane % SLOTS * 16) - key * VR::BYTES) / 2;
    vo[i] = e < dim ? 2u * (uint32_t)(key * P.token_stride + e) + DMA_FRONT - 1024 * (i % 4) : DMA_OUTSIDE;
  }
  unsigned char *mine = lds + wave * (KEYS_FEW * VR::BYTES);
  const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * (KEYS_FEW * VR::BYTES);
  u32x4 kf[2][KS];
  int32_t page[2];  // of the block that is loaded next
  auto look = [&](int32_t b) {
    const int32_t key0 = key_of(min(b, b1 - 1));
    page[0] = pages.page_of(key0);
    page[1] = pages.page_of(key0 + 16);
  };
  // whether all keys of a block are seen by all rows
  auto all_see = [&](int32_t b, int32_t key0) { return all_see_block<KEYS_FEW>(span, b, key0, p0, p1, window); };
  auto load_keys = [&](int32_t b) {
    const int32_t key0 = key_of(b);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const char *kb = kh + pages.bytes(page[half], key0 + 16 * half);
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[half][s] = load16(kb + ko[s]);
    }
  };
  auto bring_values = [&](int32_t b, const int32_t (&of)[2]) {
    const int32_t key0 = key_of(b);
    const bool whole = all_see(b, key0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int64_t at = pages.bytes(of[half], key0 + 16 * half) - DMA_FRONT;
      const __amdgpu_buffer_rsrc_t values = __builtin_amdgcn_make_buffer_rsrc((void *)(vh + at), 0, pages.there(of[half]) ? (int)DMA_OUTSIDE : 0, 0x00020000);
#pragma unroll
      for (int i = 0; i < VH; i += VI) {
        uint32_t some[VI];
#pragma unroll
        for (int n = 0; n < VI; ++n) some[n] = vo[i + n];
        if (!whole) {
          // values that no row sees: what lies there may be anything
#pragma unroll
          for (int n = 0; n < VI; ++n) {
            const int32_t j = key0 + 16 * half + (i + n) * (64 / SLOTS) + lane / SLOTS;
            some[n] = some_see(span, b, j, p0, p1, window, sinks) ? some[n] : DMA_OUTSIDE;
          }
        }
        dma<VI>(values, some, to + (half * VH + i) * 1024);
      }
    }
  };
  int32_t here[2] = {-1, -1};  // pages of the block in hand
  if (b0 + wave < b1) {
    look(b0 + wave);
    here[0] = page[0], here[1] = page[1];
    load_keys(b0 + wave);
    bring_values(b0 + wave, here);
    look(b0 + wave + 4);
  }

  const int32_t my_row = row0 + min(c, rows - 1);
  const int32_t my_token = fast_div(my_row, by_group), my_head = u.head * P.group + my_row - my_token * P.group;
  const int32_t my_pos = c < rows ? st.behind + my_token : -1;
  const char *q = (const char *)P.q + 2 * ((int64_t)(st.first + my_token) * P.q_row + (int64_t)my_head * P.q_head);
  const float scale = fabsf(P.scale_log2);  // (its sign goes into the queries)
  u32x4 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = load_query<DT>(q + 2 * (32 * s + 8 * g), c < rows && 32 * s + 8 * g < dim, P.scale_log2 < 0.f);

  f32x4 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  bool cleaned = false;

  for (int32_t b = b0 + wave; b < b1; b += 4) {
    const int32_t key0 = key_of(b);
    const uint32_t now = (pages.there(here[0]) ? 1u : 0u) | (pages.there(here[1]) ? 2u : 0u);
    if (dim != DP) {
#pragma unroll
      for (int k = 0; k < KS; ++k)
        if (32 * k + 8 * g >= dim) kf[0][k] = kf[1][k] = u32x4{0u, 0u, 0u, 0u};
    }
    f32x4 s[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      s[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) mma16<DT>(kf[half][k], qf[k], s[half]);
    }
    const bool sink = b < span.sink_blocks, alike = all_see(b, key0), whole = now == 3 && alike;
    const bool more = b + 4 < b1;
    if (more) {
      here[0] = page[0], here[1] = page[1];
      load_keys(b + 4);
      fixed_order();  // (they are counted on below)
      look(b + 8);
    }
    // lane (g, c) has the scores of row c and keys key0 + 16 half + 4 g + i
    if (!whole) {
      if (now == 3 && !two_spans) {
        const uint32_t last = (uint32_t)((sink ? span.sinks - 1 : my_pos) - key0 - 4 * g), width = sink || window == 0 ? 0x7fffffffu : (uint32_t)window - 1;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[half][i] = last - (uint32_t)(16 * half + i) <= width ? s[half][i] : -__builtin_inff();
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int32_t j = key0 + 16 * half + 4 * g + i;
            const bool ok = ((now >> half & 1) != 0) & sees(sink ? 0x7fffffff : my_pos, j, sink ? 1 : window, sink ? span.sinks : sinks);
            s[half][i] = ok ? s[half][i] : -__builtin_inff();
          }
      }
    }
    float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    top = max32(max16(top)) * scale;
    if (__ballot(top > m + RISE)) {
      const float next = fmaxf(m, top), keep = exp2_fast(m - base_of(next));
      m = next;
      l *= keep;
#pragma unroll
      for (int i = 0; i < NB; ++i) o[i] *= keep;
    }
    const float base = base_of(m);
    if (any_far(base)) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[half][i] = rounded_difference(s[half][i], scale, base) + LIFT<DT>;
    } else {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[half][i] = fmaf(s[half][i], scale, LIFT<DT> - base);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[half][i] = exp2_fast(s[half][i]);
        l += s[half][i];
      }
    // this block's values: behind them only the next block's keys are out
    if (more)
      wait_dma<2 * KS>();
    else
      wait_dma<0>();
    if (!alike && !sink && p0 != p1) {
#pragma unroll
      for (int i = 0; i < 2 * VH; ++i) {
        u32x4 *p = (u32x4 *)(mine + i * 1024 + 16 * lane);
        u32x4 v = *p;
        if (clean<DT>(v)) {
          *p = v;
          cleaned = true;
        }
      }
    }
    const u32x4 pf = {pack2<DT>(s[0][0], s[0][1]), pack2<DT>(s[0][2], s[0][3]), pack2<DT>(s[1][0], s[1][1]), pack2<DT>(s[1][2], s[1][3])};
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int byte = 2 * (16 * i + 4 * (c & 3)), row = 4 * g + (c >> 2);
      const u32x2 lo = read_transposed(mine + VR::at(row, byte)), hi = read_transposed(mine + VR::at(row + 16, byte));
      mma16<DT>(u32x4{lo.x, lo.y, hi.x, hi.y}, pf, o[i]);
    }
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the reads are done before the next values take their place
      bring_values(b + 4, here);
    }
  }
  if (__builtin_expect(__ballot(cleaned) != 0, 0)) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (16 * i + 4 * g < P.dim) o[i] += odd_sum<DT>(pages, vh + 2 * (16 * i + 4 * g), b0 + wave, b1, 4, key_of, KEYS_FEW, my_pos, window, sinks);
  }
  l = sum32(sum16(l));

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
  float *ws = a.ws_few + (int64_t)u.slot * SLOT;
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
      const float inv = inverse(sum);
      const int32_t row = row0 + r;
      const int32_t token = fast_div(row, by_group);
      char *dst = (char *)P.out + 2 * ((int64_t)(st.first + token) * P.out_row + (int64_t)(u.head * P.group + row - token * P.group) * P.out_head + e);
      if (e < P.dim) store8(dst, u32x2{pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv)});
    } else {
      store_shared(ws + r * DP + e, f32x2{v.x, v.y});
      store_shared(ws + r * DP + e + 2, f32x2{v.z, v.w});
      if (e == 0) store_shared(ws + ROWS_FEW * DP + 2 * r, f32x2{big, sum});
    }
  }
  if (u.splits == 1) return;
  if (!last_to_arrive(a.arrivals + a.slots_many + u.first_slot, u.splits, flag)) return;
  // the slices in order: the result does not depend on who came last
  const float *ws0 = a.ws_few + (int64_t)u.first_slot * SLOT;
  const int64_t step = (int64_t)P.kv_heads * SLOT;
  for (int n = tid; n < rows * (DP / 4); n += CACHE_THREADS) {
    const int r = n / (DP / 4), e = n % (DP / 4) * 4;
    float big = -__builtin_inff(), sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    constexpr int AT_ONCE = 8;  // slices whose loads go out together (one by one each would be waited for)
    for (int s = 0; s < u.splits; s += AT_ONCE) {
      f32x2 ms[AT_ONCE], x[AT_ONCE], y[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const float *w = ws0 + min(s + i, u.splits - 1) * step;
        ms[i] = load_shared(w + ROWS_FEW * DP + 2 * r), x[i] = load_shared(w + r * DP + e), y[i] = load_shared(w + r * DP + e + 2);
      }
      fixed_order();
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        if (s + i >= u.splits) break;
        const float next = fmaxf(big, ms[i].x), keep = exp2_fast(big - base_of(next)), mul = exp2_fast(ms[i].x - base_of(next));
        sum = sum * keep + ms[i].y * mul;
        v = v * keep + f32x4{x[i].x, x[i].y, y[i].x, y[i].y} * mul;
        big = next;
      }
    }
    const float inv = inverse(sum);
    const int32_t row = row0 + r;
    const int32_t token = fast_div(row, by_group);
    char *dst = (char *)P.out + 2 * ((int64_t)(st.first + token) * P.out_row + (int64_t)(u.head * P.group + row - token * P.group) * P.out_head + e);
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
// And one that holds a key's values: 64 bytes turned over with the row, so that the four rows of which half a wave reads 64 bytes each
// (transposing) lie in different banks.
template <int DP>
struct TileValueRows {
  static constexpr int BYTES = KeyRows<DP>::BYTES;
  static __device__ __forceinline__ int at(int row, int byte) {
    const int turn = BYTES == 128 ? (row >> 1) & 1 : row & 3;
    return row * BYTES + (byte ^ (turn << 6));
  }
};
// Two tiles of keys and values in LDS in turn, behind them which blocks of 16 keys of each are there, and whether values were taken out.
template <int DP>
struct ManyLds {
  static constexpr int TILE = keys_many(DP) * (KeyRows<DP>::BYTES + TileValueRows<DP>::BYTES), PRESENT = 2 * TILE, ODD = PRESENT + 8, BYTES = ODD + 8;
};

// 128 rows, 32 for each wave, against tiles of 64 keys (32 for heads of 256) that all waves read from LDS; scores as K Q^T and outputs as V^T P, as
// above: a lane holds half the scores of one row, and P needs no trip through LDS.  Matrix instructions of 32x32x16, which need half the operand
// bytes a product of the 16x16x32 ones.  Tiles come by direct loads into the other of two places while one is used; pieces are turned over
// so that neither reads of keys nor the transposing reads of values meet in a bank (conflicts 0; 59 million without).  Operands are read from
// LDS two groups of four ahead.  Bound by what a wave can issue, and power: prompts of 7000 to 8100 tokens, 32 query heads of 128, 969 us,
// 996 TFLOP/s of the pairs that are seen (a large library product 1483): 360 instructions a tile, 32 of them matrix instructions, one in about five
// cycles; the matrix units are busy 48 % of the cycles, LDS 24 %.  Scores of the next tile beside the softmax of this one gave nothing.
constexpr int SETS = 3;  // groups of LDS operands in registers: one in use, two on their way

template <int DT, int DP>
__device__ __forceinline__ void attend_many(const AttnArgs &a, const SK_CONSTANT AttnDev &P, const Unit &u, unsigned char *lds, uint32_t *flag) {
  constexpr int64_t SLOT = part_floats(ROWS_MANY, DP <= 128 ? 128 : 256);
  using KR = KeyRows<DP>;
  using VR = TileValueRows<DP>;
  constexpr int KEYS = keys_many(DP), HALVES = KEYS / 32, KS = DP / 16, NB = DP / 32, TILE = ManyLds<DP>::TILE, VALUES = KEYS * KR::BYTES;
  // a wave brings NI KB of keys and as much of values: ROWS consecutive keys, which lie in one block of 16
  constexpr int NI = KEYS * KR::BYTES / 4096, SLOTS = KR::BYTES / 16, ROWS = KEYS / 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, c = lane & 31;
  const Step &st = u.step;
  const int32_t group = P.group, dim = P.dim, window = P.window, sinks = P.sinks;
  const int32_t row0 = u.block * ROWS_MANY, rows = min(ROWS_MANY, st.fresh * group - row0);
  const FastDiv by_group = {P.by_group.mul, P.by_group.shift};
  const int32_t p0 = st.behind + fast_div(row0, by_group), p1 = st.behind + fast_div(row0 + rows - 1, by_group);
  const Span span = span_of<KEYS>(p0, p1, window, sinks);
  const bool two_spans = window && sinks > span.low;  // a row may see two runs of keys in a tile
  const int32_t b0 = slice_start(span.blocks, u.split, u.splits), b1 = slice_start(span.blocks, u.split + 1, u.splits);

  const Pages pages{P.table + (int64_t)u.seq * P.columns, P.page_shift, P.num_pages, P.columns, P.page_stride, P.token_stride};
  const char *kh = (const char *)P.k + 2 * (int64_t)u.head * P.head_stride, *vh = (const char *)P.v + 2 * (int64_t)u.head * P.head_stride;
  auto key_of = [&](int32_t b) { return block_key<KEYS>(span, b); };
  // Where this lane's pieces come from, counted from the first of the block's 16 keys.  Pieces beyond the head's end come as zeros.
  const int32_t first_key = wave * ROWS, block = first_key / 16;  // of the wave, in a tile
  uint32_t ko[NI], vo[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int key = first_key + i * (64 / SLOTS) + lane / SLOTS, place = lane % SLOTS * 16;
    const int ke = (KR::at(key, place) - key * KR::BYTES) / 2, ve = (VR::at(key, place) - key * VR::BYTES) / 2;  // (turning over twice changes nothing)
    const uint32_t at = 2u * (uint32_t)((key & 15) * P.token_stride) + DMA_FRONT - 1024 * i;
    ko[i] = ke < dim ? at + 2 * ke : DMA_OUTSIDE;
    vo[i] = ve < dim ? at + 2 * ve : DMA_OUTSIDE;
  }
  // Tiles of whose keys every row of the unit sees all.  What is decided for the others tile by tile is settled for these.
  const WholeBlocks full = whole_blocks<KEYS>(span, p0, p1, window);
  auto all_see = [&](int32_t b) { return (uint32_t)(b - full.first) < full.n; };
  int32_t next_key = key_of(b0), page = -1;  // first key of the tile that is brought next, and the page of the wave's keys in it
  auto look = [&]() { page = pages.page_of(key_behind(next_key, 16 * block)); };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * NI * 1024;
  uint32_t gone = 0;  // places where the wave's keys are not there
  auto bring = [&](int32_t b, int place) {
    const int32_t key0 = next_key;
    const bool there = pages.there(page);
    const int64_t at = pages.bytes(page, key_behind(key0, 16 * block)) - DMA_FRONT;
    const uint32_t to = lds0 + place * TILE;
    const int records = there ? (int)DMA_OUTSIDE : 0;
    dma<NI>(__builtin_amdgcn_make_buffer_rsrc((void *)(kh + at), 0, records, 0x00020000), ko, to);
    const __amdgpu_buffer_rsrc_t values = __builtin_amdgcn_make_buffer_rsrc((void *)(vh + at), 0, records, 0x00020000);
    if (all_see(b)) {
      dma<NI>(values, vo, to + VALUES);
    } else {
      // values that no row sees: what lies there may be anything
      uint32_t some[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int32_t j = key_behind(key0, first_key + i * (64 / SLOTS) + lane / SLOTS);
        some[i] = some_see(span, b, j, p0, p1, window, sinks) ? vo[i] : DMA_OUTSIDE;
      }
      dma<NI>(values, some, to + VALUES);
    }
    if (there == ((gone >> place & 1) != 0)) {
      gone ^= 1u << place;
      lds[ManyLds<DP>::PRESENT + 4 * place + wave] = there;
    }
    next_key = next_block_key<KEYS>(span, b, key0);
  };
  // Behind bring(b): the wave's pieces are there; values that are not finite are taken out where rows differ in what they see.
  bool cleaned = false;
  auto arrived = [&](int32_t b, int place) {
    wait_dma<0>();
    if (!all_see(b) && b >= span.sink_blocks) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        u32x4 *p = (u32x4 *)(lds + place * TILE + VALUES + wave * NI * 1024 + i * 1024 + 16 * lane);
        u32x4 v = *p;
        if (clean<DT>(v)) {
          *p = v;
          cleaned = true;
        }
      }
    }
  };
  if (tid < 2) ((uint32_t *)(lds + ManyLds<DP>::PRESENT))[tid] = 0x01010101u;
  __syncthreads();
  if (b0 < b1) {
    look();
    bring(b0, 0);
    look();
  }

  const int32_t in_block = wave * 32 + c;
  const bool row_ok = in_block < rows;
  const int32_t my_row = row0 + min(in_block, rows - 1);
  const int32_t my_token = fast_div(my_row, by_group), my_head = u.head * group + my_row - my_token * group;
  const int32_t my_pos = row_ok ? st.behind + my_token : -1;
  // positions of the wave's rows (uniform)
  const bool wave_ok = wave * 32 < rows;
  const int32_t w0 = st.behind + fast_div(row0 + min(wave * 32, rows - 1), by_group), w1 = st.behind + fast_div(row0 + min(wave * 32 + 31, rows - 1), by_group);
  const char *q = (const char *)P.q + 2 * ((int64_t)(st.first + my_token) * P.q_row + (int64_t)my_head * P.q_head);
  const float scale = fabsf(P.scale_log2);  // (its sign goes into the queries)
  u32x4 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = load_query<DT>(q + 2 * (16 * s + 8 * h), row_ok && 16 * s + 8 * h < dim, P.scale_log2 < 0.f);

  f32x16 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = -__builtin_inff(), l = 0.f;
  // where this lane's operands stand in a tile
  const unsigned char *ka[KS], *va[NB];
#pragma unroll
  for (int k = 0; k < KS; ++k) ka[k] = lds + KR::at(c, 2 * (16 * k + 8 * h));
#pragma unroll
  for (int i = 0; i < NB; ++i) va[i] = lds + VALUES + VR::at(4 * h + ((lane & 15) >> 2), 2 * (32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)));

  uint32_t *odd = (uint32_t *)(lds + ManyLds<DP>::ODD);  // whether any thread took values out
  if (tid == 0) *odd = 0;
  if (b0 < b1) arrived(b0, 0);
  __syncthreads();
  int32_t this_key = key_of(b0);
  auto step = [&](int32_t b, auto which) {
    constexpr int PLACE = decltype(which)::value;
    if (b + 1 < b1) {  // into the other place, which all waves have left behind the last barrier
      bring(b + 1, 1 - PLACE);
      look();
    }
    const int32_t key0 = this_key;
    this_key = next_block_key<KEYS>(span, b, key0);
    // whether any row of the wave sees any of these keys, and whether all see all
    const bool sink = b < span.sink_blocks;
    bool use = true, all = true;
    if (!all_see(b)) {
      use = wave_ok && some_see_block<KEYS>(span, b, key0, w0, w1, window, sinks);
      all = all_see_block<KEYS>(span, b, key0, w0, w1, window);
    }
    if (use) {
      constexpr uint32_t ALL = 0x01010101u;
      const uint32_t now = __builtin_amdgcn_readfirstlane(*(const uint32_t *)(lds + ManyLds<DP>::PRESENT + 4 * PLACE));
      const bool whole = all && now == ALL;
      f32x16 s[HALVES];
#pragma unroll
      for (int half = 0; half < HALVES; ++half)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[half][j] = 0.f;
      {
        constexpr int N = HALVES * KS / 4;  // groups of four
        u32x4 kf[SETS][4];
        auto read = [&](int n) {
#pragma unroll
          for (int i = 0; i < 4; ++i) kf[n % SETS][i] = *(const u32x4 *)(ka[(4 * n + i) % KS] + PLACE * TILE + (4 * n + i) / KS * 32 * KR::BYTES);
        };
#pragma unroll
        for (int n = 0; n < SETS - 1 && n < N; ++n) read(n);
        fixed_order();
#pragma unroll
        for (int n = 0; n < N; ++n) {
          if (n + SETS - 1 < N) read(n + SETS - 1);
          fixed_order();
#pragma unroll
          for (int i = 0; i < 4; ++i) mma32<DT>(kf[n % SETS][i], qf[(4 * n + i) % KS], s[(4 * n + i) / KS]);
          fixed_order();
        }
      }
      // lane (h, c) has the scores of row c and keys key0 + 32 half + 8 (i / 4) + 4 h + i % 4
      if (!whole) {
        if (now == ALL && !two_spans) {
          // keys key0 + e up to `last`, and no more than `width` before it
          const uint32_t last = (uint32_t)((sink ? span.sinks - 1 : my_pos) - key0 - 4 * h), width = sink || window == 0 ? 0x7fffffffu : (uint32_t)window - 1;
#pragma unroll
          for (int half = 0; half < HALVES; ++half)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[half][i] = last - (uint32_t)(32 * half + 8 * (i / 4) + i % 4) <= width ? s[half][i] : -__builtin_inff();
        } else {
#pragma unroll
          for (int half = 0; half < HALVES; ++half)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int32_t key = 32 * half + 8 * (i / 4), j = key_behind(key0, key + 4 * h + i % 4);
              const bool ok = ((now >> (8 * (key / ROWS)) & 1) != 0) & sees(sink ? 0x7fffffff : my_pos, j, sink ? 1 : window, sink ? span.sinks : sinks);
              s[half][i] = ok ? s[half][i] : -__builtin_inff();
            }
        }
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int half = 0; half < HALVES; ++half)
#pragma unroll
        for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, s[half][i]), s[half][i + 1]);
      top = max32(top) * scale;
      if (__ballot(top > m + RISE)) {
        const float next = fmaxf(m, top), keep = exp2_fast(m - base_of(next));
        m = next;
        l *= keep;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] *= keep;
      }
      const float base = base_of(m);
      if (any_far(base)) {
#pragma unroll
        for (int half = 0; half < HALVES; ++half)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[half][i] = rounded_difference(s[half][i], scale, base) + LIFT<DT>;
      } else {
#pragma unroll
        for (int half = 0; half < HALVES; ++half)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[half][i] = fmaf(s[half][i], scale, LIFT<DT> - base);
      }
      u32x4 pf[2 * HALVES];
#pragma unroll
      for (int half = 0; half < HALVES; ++half) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[half][i] = exp2_fast(s[half][i]);
          l += s[half][i];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
          pf[2 * half + t] = u32x4{pack2<DT>(s[half][8 * t], s[half][8 * t + 1]), pack2<DT>(s[half][8 * t + 2], s[half][8 * t + 3]),
                                   pack2<DT>(s[half][8 * t + 4], s[half][8 * t + 5]), pack2<DT>(s[half][8 * t + 6], s[half][8 * t + 7])};
      }
      {
        constexpr int G = 2 * HALVES;  // of a block of 32 elements: all its keys
        u32x4 vf[SETS][G];
        auto read = [&](int i) {
#pragma unroll
          for (int t = 0; t < G; ++t) {
            const unsigned char *p = va[i] + PLACE * TILE + 16 * t * VR::BYTES;
            const u32x2 x = read_transposed(p), y = read_transposed(p + 8 * VR::BYTES);
            vf[i % SETS][t] = u32x4{x.x, x.y, y.x, y.y};
          }
        };
#pragma unroll
        for (int i = 0; i < SETS - 1 && i < NB; ++i) read(i);
        fixed_order();
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if (i + SETS - 1 < NB) read(i + SETS - 1);
          fixed_order();
#pragma unroll
          for (int t = 0; t < G; ++t) mma32<DT>(vf[i % SETS][t], pf[t], o[i]);
          fixed_order();
        }
      }
    }
    if (b + 1 < b1) arrived(b + 1, 1 - PLACE);
    __syncthreads();
  };
  for (int32_t b = b0; b < b1; b += 2) {
    step(b, std::integral_constant<int, 0>{});
    if (b + 1 < b1) step(b + 1, std::integral_constant<int, 1>{});
  }
  if (cleaned) *odd = 1;
  __syncthreads();
  if (__builtin_expect(*odd != 0, 0)) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (32 * i + 8 * k + 4 * h < dim) {
          const f32x4 x = odd_sum<DT>(pages, vh + 2 * (32 * i + 8 * k + 4 * h), b0, b1, 1, key_of, KEYS, my_pos, window, sinks);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][4 * k + e] += x[e];
        }
  }
  l = sum32(l);

  if (u.splits > 1) {
    // partial results as they stand in the registers: [wave][register pair][lane], then maximum and sum of each row
    float *ws = a.ws_many + (int64_t)u.slot * SLOT;
    if (wave_ok) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) store_shared(ws + ((wave * NB + i) * 8 + j) * 128 + 2 * lane, f32x2{o[i][2 * j], o[i][2 * j + 1]});
      if (h == 0) store_shared(ws + ROWS_MANY * DP + 2 * in_block, f32x2{m, l});
    }
    if (!last_to_arrive(a.arrivals + u.first_slot, u.splits, flag)) return;
    if (!wave_ok) return;
    const float *ws0 = a.ws_many + (int64_t)u.first_slot * SLOT;
    const int64_t step = (int64_t)P.kv_heads * SLOT;
    // maximum and sum first, then the outputs, slice after slice, the next one's loads out
    m = -__builtin_inff();
    l = 0.f;
    constexpr int AT_ONCE = 8;
    for (int s = 0; s < u.splits; s += AT_ONCE) {
      f32x2 ms[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) ms[i] = load_shared(ws0 + min(s + i, u.splits - 1) * step + ROWS_MANY * DP + 2 * in_block);
      fixed_order();
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        if (s + i >= u.splits) break;
        const float next = fmaxf(m, ms[i].x);
        l = l * exp2_fast(m - base_of(next)) + ms[i].y * exp2_fast(ms[i].x - base_of(next));
        m = next;
      }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    const float base = base_of(m);
    f32x2 x[NB][8];
    float ms[2];
    auto read_max = [&](int s) { return load_shared(ws0 + min(s, u.splits - 1) * step + ROWS_MANY * DP + 2 * in_block).x; };
    auto read = [&](int s, int i) {
      const float *w = ws0 + min(s, u.splits - 1) * step;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = load_shared(w + ((wave * NB + i) * 8 + j) * 128 + 2 * lane);
      fixed_order();
    };
    ms[0] = read_max(0);
#pragma unroll
    for (int i = 0; i < NB; ++i) read(0, i);
    for (int s = 0; s < u.splits; ++s) {
      ms[1] = read_max(s + 1);
      const float mul = exp2_fast(ms[0] - base);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[i][2 * j] += x[i][j].x * mul;
          o[i][2 * j + 1] += x[i][j].y * mul;
        }
        fixed_order();
        read(s + 1, i);
      }
      ms[0] = ms[1];
    }
  }
  if (!row_ok) return;
  const float inv = inverse(l);
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

// The kernels: heads of up to 128 elements of either type in one, so that the tenants of a plan share a launch; heads of up to 256, whose
// sums take twice the registers, in another.  A plan that can only have units of few rows has kernels of its own, of which more workgroups
// fit a compute unit.
template <bool MANY, bool WIDE>
struct AttendLds {
  static constexpr int DP = WIDE ? 256 : 128, FEW = 4 * KEYS_FEW * ValueRows<DP>::BYTES + 4 * 2 * ROWS_FEW * 4;
  static constexpr int BYTES = MANY && ManyLds<DP>::BYTES > FEW ? ManyLds<DP>::BYTES : FEW;
};

template <int DT, int DP, bool MANY>
__device__ __forceinline__ void attend(const AttnArgs &a, const SK_CONSTANT AttnDev &P, const Unit &u, unsigned char *lds, uint32_t *flag) {
  if (MANY && u.many)
    attend_many<DT, DP>(a, P, u, lds, flag);
  else
    attend_few<DT, DP>(a, P, u, lds, flag);
}

template <bool MANY, bool WIDE>
__global__ void __launch_bounds__(CACHE_THREADS, resident(WIDE, MANY)) sk_attend(AttnArgs a) {
  __shared__ __attribute__((aligned(256))) unsigned char lds[AttendLds<MANY, WIDE>::BYTES];
  __shared__ FindScratch found;
  __shared__ uint32_t flag;
  const Unit u = find_unit<MANY, WIDE>(a, &found);
  if (!u.any) return;
  // (read through the scalar cache where it is needed)
  const SK_CONSTANT AttnDev &P = *(const SK_CONSTANT AttnDev *)(uintptr_t)(a.problems + u.problem);
  if constexpr (WIDE) {
    if (P.dtype == SK_BF16)
      attend<SK_BF16, 256, MANY>(a, P, u, lds, &flag);
    else
      attend<SK_F16, 256, MANY>(a, P, u, lds, &flag);
  } else {
    const int kind = (P.dtype == SK_BF16 ? 0 : 3) + (P.dim <= 64 ? 0 : P.dim <= 96 ? 1 : 2);
    switch (kind) {
      case 0: return attend<SK_BF16, 64, MANY>(a, P, u, lds, &flag);
      case 1: return attend<SK_BF16, 96, MANY>(a, P, u, lds, &flag);
      case 2: return attend<SK_BF16, 128, MANY>(a, P, u, lds, &flag);
      case 3: return attend<SK_F16, 64, MANY>(a, P, u, lds, &flag);
      case 4: return attend<SK_F16, 96, MANY>(a, P, u, lds, &flag);
      default: return attend<SK_F16, 128, MANY>(a, P, u, lds, &flag);
    }
  }
}

}  // namespace sk
