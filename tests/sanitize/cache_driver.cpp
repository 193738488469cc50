// Host code of the operators over paged caches (cache_plan.cpp, and the arithmetic of cache_units.h that the kernels share) on seeded random
// plans, steps and accounts, for a build with sanitizers.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>

#include "cache_internal.h"
#include "cache_units.h"

static void need(bool ok, const char *what) {
  if (!ok) {
    std::printf("cache_driver: %s\n", what);
    std::exit(1);
  }
}

static void plans(std::mt19937 &rng) {
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  for (int round = 0; round < 2000; ++round) {
    std::vector<sk_attn_problem> ps((size_t)pick(0, 6));
    uintptr_t at = (uintptr_t)1 << 40;
    for (sk_attn_problem &p : ps) {
      p = sk_attn_problem{};
      p.dtype = pick(0, 20) ? pick(1, 2) : pick(-1, 3);
      p.kv_heads = pick(1, 9);
      p.q_heads = p.kv_heads * pick(1, 17);
      p.head_dim = pick(0, 9) ? 8 * pick(1, 32) : pick(0, 300);
      p.page_tokens = 16 << pick(0, 4);
      p.num_pages = pick(1, 100000);
      p.sequences = pick(1, 300);
      p.pages_per_sequence = pick(1, 3000);
      p.rows = pick(1, 5000);
      p.max_new = pick(0, 1) ? 0 : pick(1, 6000);
      p.window = pick(0, 1) ? 0 : pick(1, 5000);
      p.sinks = pick(0, 9);
      p.k = (void *)at, p.v = (void *)at, p.page_table = p.lengths = p.first_row = (int32_t *)at;
      at += (uintptr_t)1 << 36;
      p.q = (void *)at;
      at += (uintptr_t)1 << 36;
      p.out = pick(0, 5) ? (void *)at : nullptr;
      at += (uintptr_t)1 << 36;
      p.qkv = pick(0, 3) ? (void *)at : nullptr;
      if (pick(0, 30) == 0) p.token_stride = 8 * pick(0, 100), p.kv_head_stride = 8 * pick(0, 1000), p.page_stride = 8 * pick(0, 100000);
    }
    sk::AttnPlanHost h;
    std::string err;
    const sk_status st = sk::plan_attn(ps.data(), (int32_t)ps.size(), 256, pick(0, 2) ? 0 : pick(1, 2000), h, err);
    need((st == SK_OK) == err.empty(), "an error without a text, or a text without an error");
    if (st != SK_OK) continue;
    need(h.problems.size() == ps.size() && h.append_first.size() == ps.size() + 1, "sizes");
    int64_t seqs = 0;
    for (size_t i = 0; i < ps.size(); ++i) {
      const sk::AttnDev &d = h.problems[i];
      if (d.out) seqs += d.sequences;
      const int64_t per_row = (int64_t)d.parts * d.turns * (64 / d.lanes_per_head);
      need(per_row >= d.q_heads + 2 * d.kv_heads, "append leaves heads out");
      if (d.qkv) need(((int64_t)h.append_first[i + 1] - h.append_first[i]) * 4 >= (int64_t)d.rows * d.parts, "append leaves rows out");
    }
    need((int64_t)h.seqs.size() == seqs, "sequences");
    // units of the largest steps that the bounds allow fit the grids
    for (const sk::AttnGroup &g : h.groups) {
      int64_t few = 0, many = 0;
      for (int64_t s = g.first_seq; s < g.first_seq + g.sequences; ++s) {
        const sk::AttnSeq &q = h.seqs[(size_t)s];
        few += (int64_t)q.kv_heads * ((std::min<int64_t>((int64_t)q.group * q.max_new, q.most_few) + sk::ROWS_FEW - 1) / sk::ROWS_FEW);
        if ((int64_t)q.max_new * q.group > q.most_few && q.seq == 0) many += (int64_t)q.kv_heads * (((int64_t)q.rows * q.group + sk::ROWS_MANY - 1) / sk::ROWS_MANY);
      }
      need(g.grid >= std::max(few, many), "units without a workgroup");
      need(h.counters >= g.slots_few + g.slots_many, "counters");
      need(g.slots_few + g.slots_many <= 4 * g.workgroups, "more places than slices");
      need(h.workspace_floats >= g.slots_few * sk::part_floats(sk::ROWS_FEW, g.wide ? 256 : 128) + g.slots_many * sk::part_floats(sk::ROWS_MANY, g.wide ? 256 : 128), "workspace");
    }
  }
}

static void accounts(std::mt19937 &rng) {
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  for (int round = 0; round < 60; ++round) {
    const int pages = pick(1, 80), page = pick(1, 20), seqs = pick(1, 9), columns = pick(1, 12);
    sk::PageAccount a(pages, page, seqs, columns);
    // what lies in the pages: the copies move it, writes renew it
    std::vector<int> content((size_t)pages, 0);
    std::vector<std::vector<int>> want((size_t)seqs);  // per sequence: content of each of its pages
    int next = 0;
    for (int step = 0; step < 300; ++step) {
      std::string err;
      const int what = pick(0, 9);
      if (what == 0) {
        a.compact();
      } else if (what <= 2) {
        const int32_t from = pick(0, seqs - 1), to = pick(0, seqs - 1);
        if (a.fork(from, &to, 1, err) == SK_OK) want[(size_t)to] = want[(size_t)from];
      } else {
        std::vector<int32_t> ids, tokens;
        for (int s = 0; s < seqs; ++s)
          if (pick(0, 2) == 0) ids.push_back(s), tokens.push_back(pick(0, 1) ? std::min(a.tokens(s) + pick(0, 3), page * columns) : pick(0, page * columns));
        const std::vector<std::vector<int>> before = want;
        std::vector<int32_t> had;
        for (int32_t s : ids) had.push_back(a.tokens(s));
        if (a.resize(ids.data(), tokens.data(), (int32_t)ids.size(), err) == SK_OK)
          for (size_t i = 0; i < ids.size(); ++i) want[(size_t)ids[i]].resize((size_t)((tokens[i] + page - 1) / page), -1);
      }
      if (pick(0, 2) == 0) {
        for (const auto &w : a.waves()) {
          std::set<int32_t> read, written;
          for (const sk::PageMove &m : w) {
            read.insert(m.from);
            need(written.insert(m.to).second, "a page written twice in a wave");
          }
          for (int32_t p : written) need(!read.count(p), "a page read and written in a wave");
          for (const sk::PageMove &m : w) content[(size_t)m.to] = content[(size_t)m.from];
        }
        a.applied();
        need(a.pending() == 0 && a.dirty_rows().empty(), "something pending behind applied()");
        // pages new since the last time are written now, by those that hold them
        for (int s = 0; s < seqs; ++s)
          for (size_t c = 0; c < want[(size_t)s].size(); ++c) {
            int &x = content[(size_t)a.row(s)[c]];
            if (want[(size_t)s][c] == -1) {
              x = ++next;
              for (int t = 0; t < seqs; ++t)  // forked before it was written
                for (size_t d = 0; d < want[(size_t)t].size(); ++d)
                  if (a.row(t)[d] == a.row(s)[c]) want[(size_t)t][d] = x;
            }
            need(x == want[(size_t)s][c], "a page's content got lost");
          }
      }
      std::set<int32_t> used;
      for (int s = 0; s < seqs; ++s)
        for (int c = 0; c < columns; ++c)
          if (a.row(s)[c] >= 0) used.insert(a.row(s)[c]);
      need((int)used.size() == pages - a.free_pages(), "free pages");
    }
  }
}

// The blocks of keys of a run of rows against the definition, in 64 bits: sequences of any length that a plan takes, the longest among them.
template <int KEYS>
static void blocks_of_keys(std::mt19937 &rng) {
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)((((uint64_t)rng() << 32) | rng()) % (uint64_t)(hi - lo + 1)); };
  for (int round = 0; round < 4000; ++round) {
    const int shift = (int)pick(4, 16);
    const int64_t most = ((int64_t)1 << 31 >> shift) - 1, columns = pick(0, 2) ? pick(std::max<int64_t>(1, most - 5), most) : pick(1, std::min<int64_t>(most, 100));
    const int64_t capacity = columns << shift;
    const int64_t p1 = pick(0, 3) ? pick(std::max<int64_t>(0, capacity - 200), capacity - 1) : pick(0, capacity - 1), p0 = p1 - pick(0, 127);
    const int32_t window = (int32_t)(pick(0, 1) ? 0 : pick(0, 3) ? pick(1, 300) : pick(1, 0x7fffffff)), sinks = (int32_t)(pick(0, 1) ? pick(0, 70) : pick(0, 5) ? 0 : 0x7fffffff);
    const sk::Span s = sk::span_of<KEYS>((int32_t)p0, (int32_t)p1, window, sinks);
    auto row_sees = [&](int64_t p, int64_t j) { return j <= p && (window == 0 || p - j < window || j < sinks); };
    need(s.low >= 0 && s.low % 16 == 0 && s.sink_blocks >= 0 && s.blocks > s.sink_blocks, "span");
    for (int64_t j = std::max<int64_t>(0, p0); j <= p1; ++j) need(j >= s.low, "a key left out");
    const int64_t first_seen = window ? std::max<int64_t>(0, p0 - window + 1) : 0;
    need(s.low <= first_seen && (s.low == first_seen || s.low + 15 >= first_seen), "low");
    need((int64_t)s.low + (int64_t)(s.blocks - s.sink_blocks) * KEYS > p1 && (int64_t)s.sink_blocks * KEYS >= s.sinks, "blocks");
    const sk::WholeBlocks whole = sk::whole_blocks<KEYS>(s, (int32_t)p0, (int32_t)p1, window);
    std::set<int32_t> some;
    for (int i = 0; i < 3; ++i) some.insert({i, s.blocks - 1 - i, s.sink_blocks + i, s.sink_blocks - 1 - i, (int32_t)pick(0, s.blocks - 1)});
    for (int32_t b : some) {
      if (b < 0 || b >= s.blocks) continue;
      const bool sink = b < s.sink_blocks;
      const int64_t key = sink ? (int64_t)b * KEYS : s.low + (int64_t)(b - s.sink_blocks) * KEYS;
      need(sk::block_key<KEYS>(s, b) == key, "a block's key");
      // the block behind this one, which is looked up ahead, whether the rows need it or not
      const int64_t behind = b + 1 == s.sink_blocks ? s.low : key + KEYS;
      for (int i = 0; i < KEYS; i += 16) {
        const int32_t c = sk::column_of(sk::key_behind(sk::next_block_key<KEYS>(s, b, (int32_t)key), i), shift, (int32_t)columns);
        need(c == (behind + i < capacity ? (behind + i) >> shift : -1), "a column outside the table");
      }
      bool all = true, any = false, all_there = true;
      for (int i = 0; i < KEYS; ++i) {
        const int64_t j = key + i;
        bool every = j < capacity, one = false;
        for (int64_t p : {p0, p1, std::min(p0 + 1, p1), std::max(p1 - 1, p0), (p0 + p1) / 2}) {
          const bool here = sink ? j < s.sinks : row_sees(p, j);
          need(!sink || j >= s.sinks || row_sees(p, j), "a sink that a row does not see");
          every = every && here, one = one || here;
          if (j < capacity && p >= 0) need(sk::sees((int32_t)p, (int32_t)j, window, sinks) == row_sees(p, j), "sees");
        }
        need(sk::some_see(s, b, sk::key_behind((int32_t)key, i), (int32_t)p0, (int32_t)p1, window, sinks) >= one, "a value left out");
        if (j >= capacity && !sink) need(!sk::some_see(s, b, sk::key_behind((int32_t)key, i), (int32_t)p0, (int32_t)p1, window, sinks), "a value that nobody sees");
        all = all && every, any = any || one, all_there = all_there && j < capacity;
      }
      need(!sk::all_see_block<KEYS>(s, b, (int32_t)key, (int32_t)p0, (int32_t)p1, window) || all, "a block that not all see");
      need(!all || sinks || sk::all_see_block<KEYS>(s, b, (int32_t)key, (int32_t)p0, (int32_t)p1, window), "a block that all see");
      need(!any || sk::some_see_block<KEYS>(s, b, (int32_t)key, (int32_t)p0, (int32_t)p1, window, sinks), "a block that some see");
      need((uint32_t)(b - whole.first) >= whole.n || (all && all_there), "whole blocks");
    }
  }
}

// What every workgroup of a launch of sequences finds, from the lengths and rows that the device has: units and slices in the order of the
// sequences, those of many rows first.
struct Found {
  int64_t items, cut_many, cut_few;
  bool fits;
  struct Seq {
    int64_t first_item;
    int32_t units, splits;
  };
  std::vector<Seq> seqs;
};
template <bool MANY, bool WIDE>
static Found find(const std::vector<sk::AttnSeq> &seqs, const std::vector<int32_t> &first, const std::vector<int32_t> &length, const sk::AttnGroup &g) {
  std::vector<sk::Count> counts;
  int64_t work = 0, units = 0;
  for (size_t s = 0; s < seqs.size(); ++s) {
    counts.push_back(sk::count_units<MANY, WIDE>(sk::step_of(seqs[s], first[s], first[s + 1], length[s]), seqs[s]));
    work += sk::work_of(counts.back());
    units += counts.back().units;
  }
  int32_t most = sk::even_share(work, g.workgroups);
  auto items = [&]() {
    int64_t n = 0;
    for (const sk::Count &c : counts) n += (int64_t)c.units * sk::splits_of(c, most);
    return n;
  };
  for (int i = 0; i < 8 && seqs.size() <= 64 && units <= g.workgroups / 2 && items() > g.workgroups; ++i) most += most / 8 + 1;
  Found f{};
  for (int pass = 0; pass < 2; ++pass)
    for (const sk::Count &c : counts) {
      const int32_t splits = sk::splits_of(c, most);
      const int64_t n = (int64_t)c.units * splits;
      if (pass == 0) (c.many ? f.cut_many : f.cut_few) += splits > 1 ? n : 0;
      if (c.many != (pass == 0)) continue;
      f.seqs.push_back(Found::Seq{f.items, c.units, splits});
      f.items += n;
    }
  auto sum32 = [](int64_t n) { return (int32_t)std::min<int64_t>(n, (int64_t)1 << 30); };
  f.fits = sk::slices_fit(sum32(f.items), sum32(f.cut_many), sum32(f.cut_few), (uint32_t)g.grid, (uint32_t)g.slots_many, (uint32_t)g.slots_few);
  return f;
}

// Steps with rows in order always fit what their plan's launch has; of steps with rows in any order, those that do not are told.
static void steps(std::mt19937 &rng) {
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  int caught = 0, sliced = 0;
  for (int round = 0; round < 6000; ++round) {
    sk_attn_problem p{};
    p.dtype = 1;
    p.kv_heads = pick(1, 8);
    p.q_heads = p.kv_heads * pick(1, 8);
    p.head_dim = 8 * pick(1, 32);
    p.page_tokens = 16;
    p.num_pages = 10;
    p.sequences = pick(0, 3) ? pick(1, 64) : pick(65, 400);
    p.pages_per_sequence = pick(0, 1) ? pick(1, 100) : pick(100, 20000);
    p.rows = pick(0, 1) ? pick(1, 400) : pick(400, 4000);
    p.max_new = pick(0, 1) ? 0 : pick(1, 300);
    p.window = pick(0, 2) ? 0 : pick(1, 5000);
    p.sinks = pick(0, 9);
    const uintptr_t at = (uintptr_t)1 << 40;
    p.k = p.v = p.q = (void *)at, p.page_table = p.lengths = p.first_row = (int32_t *)at, p.out = (void *)(at << 1);
    sk::AttnPlanHost h;
    std::string err;
    need(sk::plan_attn(&p, 1, 256, pick(0, 1) ? 0 : pick(1, 700), h, err) == SK_OK && h.groups.size() == 1, "a plan of one problem");
    const sk::AttnGroup &g = h.groups[0];
    std::vector<int32_t> length, first{0};
    const int32_t capacity = p.pages_per_sequence * p.page_tokens;
    for (int s = 0; s < p.sequences; ++s) length.push_back(pick(0, 2) ? pick(0, capacity) : pick(0, 1) ? capacity : pick(0, 100));
    const bool in_order = round % 2;
    const bool alternate = round % 4 == 0;  // every second sequence has all rows
    for (int s = 1; s <= p.sequences; ++s) first.push_back(alternate ? s % 2 * p.rows : pick(0, 4) ? pick(0, p.rows) : pick(-5, p.rows + 5));
    if (in_order) std::sort(first.begin(), first.end());
    const Found f = g.wide ? (g.many ? find<true, true>(h.seqs, first, length, g) : find<false, true>(h.seqs, first, length, g))
                           : (g.many ? find<true, false>(h.seqs, first, length, g) : find<false, false>(h.seqs, first, length, g));
    need(!in_order || f.fits, "a step in order that does not fit its launch");
    bool straddles = false;  // a sequence that is cut, of whose slices only some have a workgroup
    for (const Found::Seq &s : f.seqs) straddles = straddles || (s.splits > 1 && s.first_item < g.grid && s.first_item + (int64_t)s.units * s.splits > g.grid);
    need(!straddles || !f.fits, "slices without a workgroup");
    caught += straddles;
    sliced += in_order && f.cut_many + f.cut_few > 0;
  }
  need(caught > 20 && sliced > 500, "steps that show nothing");
}

static void copies() {
  for (int64_t chunks = 1; chunks * sk::COPY_CHUNK <= sk::COPY_PAGE; chunks += 1 + chunks / 7) {
    const sk::CopyBatch b = sk::copy_batch(chunks);
    need(b.arrays >= 1 && b.arrays <= sk::COPY_ARRAYS && b.moves >= 1 && b.moves <= sk::COPY_MOVES, "a batch that a launch's arguments do not hold");
    need(chunks * b.arrays * b.moves + sk::ROW_GROUPS <= sk::MOST_GRID, "a batch that a launch's grid does not hold");
    need(b.moves == sk::COPY_MOVES || chunks * b.arrays * (b.moves + 1) + sk::ROW_GROUPS > sk::MOST_GRID, "a batch smaller than need be");
  }
}

int main() {
  std::mt19937 rng(7);
  plans(rng);
  blocks_of_keys<32>(rng);
  blocks_of_keys<64>(rng);
  accounts(rng);
  steps(rng);
  copies();
  std::printf("cache_driver: ok\n");
  return 0;
}
