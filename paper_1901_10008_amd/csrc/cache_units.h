// Arithmetic of attention's units of work that the kernels and the host's checks share: which keys a run of rows sees, in which blocks
// they are walked through, and where the page table has their pages; how many units a sequence has, and into how many slices they are cut.
#pragma once

#include <cstdint>

#include "cache_internal.h"

#if defined(__HIPCC__)
#define SK_BOTH __host__ __device__ __forceinline__
#else
#define SK_BOTH inline
#endif

namespace sk {

template <class T>
SK_BOTH T lesser(T a, T b) { return b < a ? b : a; }
template <class T>
SK_BOTH T larger(T a, T b) { return a < b ? b : a; }

// Keys are counted in 32 bits.  A sequence has less than 2^31 tokens, but the last block of one, and the block looked up behind it, may reach
// beyond: such keys are negative here.  No row sees one, and no table has a page for it.
SK_BOTH int32_t key_behind(int32_t key, int32_t n) { return (int32_t)((uint32_t)key + (uint32_t)n); }
// The column of the page table that has a key's page; -1: none has.
SK_BOTH int32_t column_of(int32_t key, int32_t shift, int32_t columns) {
  const uint32_t c = (uint32_t)key >> shift;
  return c < (uint32_t)columns ? (int32_t)c : -1;
}

// The keys that rows at positions p0 .. p1 see: blocks of KEYS from `low` on (a multiple of 16), ahead of them blocks from 0 on for the sinks below
// it.  The last of these may reach beyond `low`: of its keys only the first `sinks` of the span count.
struct Span {
  int32_t low, sinks, sink_blocks, blocks;
};
template <int KEYS>
SK_BOTH Span span_of(int32_t p0, int32_t p1, int32_t window, int32_t sinks) {
  Span s;
  s.low = window ? (p0 >= window ? p0 - window + 1 : 0) & ~15 : 0;
  s.sinks = lesser(sinks, s.low);
  s.sink_blocks = (int32_t)(((uint32_t)s.sinks + KEYS - 1) / KEYS);
  s.blocks = p1 < 0 ? 0 : s.sink_blocks + (p1 - s.low) / KEYS + 1;
  return s;
}
// First key of block b, and of the block behind one that begins at `key`.
template <int KEYS>
SK_BOTH int32_t block_key(const Span &s, int32_t b) { return b < s.sink_blocks ? b * KEYS : s.low + (b - s.sink_blocks) * KEYS; }
template <int KEYS>
SK_BOTH int32_t next_block_key(const Span &s, int32_t b, int32_t key) { return b + 1 == s.sink_blocks ? s.low : key_behind(key, KEYS); }

// Whether the token at position p sees key j.  (No branches: a mask per element.)
SK_BOTH bool sees(int32_t p, int32_t j, int32_t window, int32_t sinks) {
  return (j <= p) & ((window == 0) | ((int32_t)((uint32_t)p - (uint32_t)j) < window) | (j < sinks));
}
// Whether any of the rows at positions p0 .. p1 sees key j of block b.
SK_BOTH bool some_see(const Span &s, int32_t b, int32_t j, int32_t p0, int32_t p1, int32_t window, int32_t sinks) {
  return b < s.sink_blocks ? j < s.sinks : ((uint32_t)j <= (uint32_t)p1) & ((window == 0) | ((int32_t)((uint32_t)p0 - (uint32_t)j) < window) | (j < sinks));
}
// Whether all of them see all keys of block b, which begins at `key`; whether any sees any of them.
template <int KEYS>
SK_BOTH bool all_see_block(const Span &s, int32_t b, int32_t key, int32_t p0, int32_t p1, int32_t window) {
  return b < s.sink_blocks ? (uint32_t)key + KEYS <= (uint32_t)s.sinks : ((uint32_t)key + KEYS - 1 <= (uint32_t)larger(p0, 0)) & ((window == 0) | (p1 - key < window));
}
template <int KEYS>
SK_BOTH bool some_see_block(const Span &s, int32_t b, int32_t key, int32_t p0, int32_t p1, int32_t window, int32_t sinks) {
  return b < s.sink_blocks || (key <= p1 && (window == 0 || p0 - key - (KEYS - 1) < window || key < sinks));
}
// Blocks first .. first + n - 1 of those that rows p0 .. p1 need: all of them see all keys there (sinks apart).
struct WholeBlocks {
  int32_t first;
  uint32_t n;
};
template <int KEYS>
SK_BOTH WholeBlocks whole_blocks(const Span &s, int32_t p0, int32_t p1, int32_t window) {
  const int32_t f0 = s.sink_blocks + (window && p1 - window >= s.low ? (p1 - window - s.low) / KEYS + 1 : 0);
  const int32_t f1 = s.sink_blocks + (p0 - s.low >= KEYS - 1 ? (p0 - s.low - (KEYS - 1)) / KEYS + 1 : 0);
  return WholeBlocks{f0, (uint32_t)larger(f1 - f0, 0)};
}

// A sequence in this step: rows and lengths cut to the bounds that the grid was made for.
struct Step {
  int32_t first, fresh, length, behind;  // first row, rows to compute, tokens, position of the first new token
};
SK_BOTH Step step_of(const AttnSeq &q, int32_t first_row, int32_t next_row, int32_t length) {
  Step s;
  s.first = lesser(larger(first_row, 0), q.rows);
  const int32_t all = lesser(larger(next_row, s.first), q.rows) - s.first;
  s.length = (int32_t)lesser((int64_t)larger(length, 0), q.capacity);
  s.behind = s.length - all;
  s.fresh = lesser(all, q.max_new);
  return s;
}

struct Count {
  int32_t row_blocks, units, blocks;  // blocks of keys of an average unit
  bool many;
};
template <bool MANY, bool WIDE>
SK_BOTH Count count_units(const Step &s, const AttnSeq &q) {
  const int32_t kv_heads = q.kv_heads, group = q.group, window = q.window, sinks = q.sinks;
  Count c;
  const int64_t rows = (int64_t)s.fresh * group;
  const int32_t last = s.behind + s.fresh - 1;
  c.many = MANY && rows > q.most_few;
  if (c.many) {
    c.row_blocks = (int32_t)((rows + ROWS_MANY - 1) / ROWS_MANY);
    const int32_t tokens = (int32_t)((uint32_t)(ROWS_MANY + group - 1) / (uint32_t)group);
    constexpr int KEYS = keys_many(WIDE ? 256 : 128);
    const Span a = span_of<KEYS>(s.behind, lesser(s.behind + tokens - 1, last), window, sinks);
    const Span b = span_of<KEYS>(larger(last - tokens + 1, s.behind), last, window, sinks);
    c.blocks = (a.blocks + b.blocks + 1) / 2;
  } else {
    c.row_blocks = (int32_t)((rows + ROWS_FEW - 1) / ROWS_FEW);
    c.blocks = span_of<KEYS_FEW>(s.behind, last, window, sinks).blocks;
  }
  c.units = c.row_blocks * kv_heads;
  return c;
}

// n / d for 0 <= n < 2^52 and d > 0: the rounded quotient of the exact values does not reach the next whole number, which is 1 / d away or more.
// (Whole numbers of 64 bits take the compiler a hundred instructions more.)
SK_BOTH int64_t divide(int64_t n, int64_t d) { return (int64_t)((double)n / (double)d); }
// The first of `blocks` that slice number `split` of a unit takes.
SK_BOTH int32_t slice_start(int32_t blocks, int32_t split, int32_t splits) { return splits == 1 ? split * blocks : (int32_t)divide((int64_t)blocks * split, splits); }

// Units of many keys are cut into slices, so that few units fill the card and no unit is what the launch waits for.  A slice takes at most `most`
// blocks of keys of few rows, or a TILE_WORK-th as many tiles of many: a tile takes 2 us, a block 0.5 to 1.  Of sixteen launches
// that mix chunks and single tokens one is 5 % slower with a ratio of 2 and 2 % faster with 4, one 8 % faster with 2 and 10 % slower with 4; the
// others take the same time within 2 %.
constexpr int TILE_WORK = 3;
constexpr int LEAST = 4;  // a block for each wave; tiles
SK_BOTH int32_t splits_of(const Count &c, int32_t most) {
  const uint32_t per = larger(c.many ? ((uint32_t)most + TILE_WORK - 1) / TILE_WORK : (uint32_t)most, (uint32_t)LEAST);
  return (int32_t)lesser(((uint32_t)larger(c.blocks, 1) + per - 1) / per, (uint32_t)MOST_SPLITS);
}
SK_BOTH int64_t work_of(const Count &c) { return (int64_t)c.units * c.blocks * (c.many ? TILE_WORK : 1); }
// work: blocks of few rows and TILE_WORK times the tiles of many.  That many for each workgroup the card runs at a time: with it units and slices
// are no more than these workgroups and the units together, and the slices of units that are cut (each of more than `most`) no more than twice
// these workgroups.
SK_BOTH int32_t even_share(int64_t work, int64_t workgroups) { return (int32_t)lesser(divide(work + workgroups - 1, workgroups), (int64_t)0x7ffffffe); }
// Units and slices of a sequence.  All of a launch's are no more than its grid; where first_row decreases there can be any number, of which no more
// are counted than keeps sums of sequences within 32 bits.
constexpr int32_t MOST_ITEMS = 1 << 24;
static_assert(MOST_GRID < MOST_ITEMS, "every sum that counts can be told from one that does not");
SK_BOTH int32_t items_of(const Count &c, int32_t splits) { return (int32_t)lesser((int64_t)c.units * splits, (int64_t)MOST_ITEMS); }
// Whether a launch has a workgroup for every unit and slice, and a place of the workspace for every slice.  With a first_row that decreases it
// may not: then nothing is cut, since slices of which some have no workgroup would never be joined and leave their count of arrivals behind.
SK_BOTH bool slices_fit(int32_t items, int32_t cut_many, int32_t cut_few, uint32_t grid, uint32_t slots_many, uint32_t slots_few) {
  return (uint32_t)items <= grid && (uint32_t)cut_many <= slots_many && (uint32_t)cut_few <= slots_few;
}

}  // namespace sk
