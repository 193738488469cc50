// Arithmetic of attention's units of work that the kernels and the host's checks share: which keys a run of rows sees, in which blocks
// they are walked through, and where the page table has their pages.
#pragma once

#include <cstdint>

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

}  // namespace sk
