// The account of pages (cache_plan.cpp) with host allocations that fail: a program of its own, since it replaces the operators new and delete.
#include <cstdio>
#include <cstdlib>
#include <new>
#include <random>

#include "cache_internal.h"

static long g_left = -1;  // allocations that succeed before all others fail; < 0: all succeed
void *operator new(size_t n) {
  if (g_left == 0) throw std::bad_alloc();
  if (g_left > 0) --g_left;
  void *p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

static void need(bool ok, const char *what) {
  if (!ok) {
    std::printf("cache_memory_driver: %s\n", what);
    std::exit(1);
  }
}

// Calls that run out of host memory change nothing.
struct State {
  std::vector<int32_t> tokens, rows, moves;
  int32_t free_pages;
  bool operator==(const State &o) const { return tokens == o.tokens && rows == o.rows && moves == o.moves && free_pages == o.free_pages; }
};
static State state_of(const sk::PageAccount &a) {
  State s;
  for (int i = 0; i < a.sequences(); ++i) {
    s.tokens.push_back(a.tokens(i));
    s.rows.insert(s.rows.end(), a.row(i), a.row(i) + a.columns());
  }
  for (const auto &w : a.waves()) {
    s.moves.push_back(-1);
    for (const sk::PageMove &m : w) s.moves.push_back(m.from), s.moves.push_back(m.to);
  }
  s.free_pages = a.free_pages();
  return s;
}
static void out_of_memory(std::mt19937 &rng) {
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  int failed = 0;
  for (int round = 0; round < 300; ++round) {
    const int seqs = pick(2, 9), page = 4, columns = 6;
    sk::PageAccount a(pick(10, 60), page, seqs, columns);
    std::string err;
    for (int step = 0; step < 40; ++step) {
      std::vector<int32_t> ids, tokens;
      for (int s = 0; s < seqs; ++s)
        if (pick(0, 1)) ids.push_back(s), tokens.push_back(pick(0, 2) ? std::min(a.tokens(s) + pick(0, 3), page * columns) : pick(0, page * columns));
      const int32_t from = pick(0, seqs - 1), to = pick(0, seqs - 1);
      const int what = pick(0, 3);
      auto call = [&]() { return what == 0 ? a.compact() : what == 1 ? a.fork(from, &to, 1, err) : a.resize(ids.data(), tokens.data(), (int32_t)ids.size(), err); };
      if (pick(0, 9) == 0) a.applied();
      const State before = state_of(a);
      bool done = false;
      for (long left = 0; !done; ++left) {
        g_left = left;
        try {
          call();
          done = true;
        } catch (const std::bad_alloc &) {
        }
        g_left = -1;
        if (!done) {
          ++failed;
          need(state_of(a) == before, "a call without memory has changed the account");
        }
      }
    }
  }
  need(failed > 1000, "calls that need no memory");
}

int main() {
  std::mt19937 rng(11);
  out_of_memory(rng);
  std::printf("cache_memory_driver: ok\n");
  return 0;
}
