// Plans of libsk_layer.so (layer_plan.cpp) on seeded random problems: every unit of a plan has a workgroup, every place of its workspace room.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "layer_internal.h"
#include "layer_units.h"

static void need(bool ok, const char *what) {
  if (!ok) {
    std::printf("layer_driver: %s\n", what);
    std::exit(1);
  }
}

static std::mt19937_64 g_random(1);
static int64_t between(int64_t lo, int64_t hi) { return lo + (int64_t)(g_random() % (uint64_t)(hi - lo + 1)); }
static void *address(int i) { return (void *)(((uintptr_t)i + 1) << 44); }

// An array of a workspace: it begins behind the end of the one before, and ends inside.
struct Walk {
  size_t end = 0, all;
  explicit Walk(size_t bytes) : all(bytes) {}
  template <class T>
  void next(const T *p, int64_t count) {
    const size_t at = (size_t)(uintptr_t)p;
    need(at % sizeof(T) == 0 || sizeof(T) > 16, "an array is not aligned");
    need(at >= end, "arrays of a workspace overlap");
    end = at + (size_t)count * sizeof(T);
    need(end <= all, "an array ends behind its workspace");
  }
};

static void norms() {
  const int n = (int)between(0, 60);
  std::vector<sk_norm_problem> problems;
  for (int i = 0; i < n; ++i) {
    sk_norm_problem p{};
    p.dtype = (int32_t)between(0, 2), p.residual_dtype = between(0, 1) ? p.dtype : (int32_t)SK_F32;
    p.rows = (int32_t)between(1, 5000), p.dim = (int32_t)between(1, 32768);
    p.block = p.residual = address(0);
    p.residual_out = address(2 * i + 1), p.next = address(2 * i + 2);
    problems.push_back(p);
  }
  sk::NormPlanHost out;
  std::string err;
  need(sk::plan_norm(problems.data(), n, out, err) == SK_OK, err.c_str());
  int seen = 0;
  for (const sk::NormLaunch &l : out.launches) {
    need(l.n >= 1 && l.n <= sk::NORM_PROBLEMS, "problems of a launch");
    for (int i = 0; i < sk::NORM_PROBLEMS; ++i) {
      if (i >= l.n) {
        need(l.table.first[i] == 0xffffffffu, "a place without a problem can be found");
        continue;
      }
      const sk::NormDev &d = l.table.problems[i];
      need(d.dim <= sk::norm_most_dim(l.form), "a row longer than its form takes");
      const int64_t end = i + 1 < l.n ? l.table.first[i + 1] : l.grid, groups = end - l.table.first[i];
      const int64_t of = sk::norm_rows_of(l.form);
        need(groups == (d.rows + of - 1) / of, "workgroups of a problem");
      ++seen;
    }
  }
  need(seen == n, "every problem once");
}

static void moes() {
  const int n = (int)between(0, 5);
  std::vector<sk_moe_problem> problems;
  for (int i = 0; i < n; ++i) {
    sk_moe_problem p{};
    p.dtype = (int32_t)between(1, 2), p.router_dtype = between(0, 1) ? p.dtype : (int32_t)SK_F32;
    p.rows = (int32_t)(between(0, 1) ? between(1, 40) : between(1, 3000)), p.dim = 8 * (int32_t)between(1, 300), p.experts = (int32_t)between(1, 512);
    p.top_k = (int32_t)between(1, std::min(32, p.experts)), p.ffn = 8 * (int32_t)between(1, 300), p.shared_ffn = between(0, 1) ? 8 * (int32_t)between(1, 200) : 0;
    p.x = p.router = p.up = p.down = p.shared_up = p.shared_down = address(0);
    if (between(0, 1)) p.gate = p.shared_gate = address(0);
    if (!p.shared_ffn) p.shared_gate = nullptr;
    p.out = address(3 * i + 1), p.expert_ids = (int32_t *)address(3 * i + 2), p.expert_weights = (float *)address(3 * i + 3);
    problems.push_back(p);
  }
  const int32_t workgroups = between(0, 1) ? (int32_t)between(1, 3000) : 0;
  sk::MoePlanHost out;
  std::string err;
  need(sk::plan_moe(problems.data(), n, 256, workgroups, out, err) == SK_OK, err.c_str());
  Walk work(out.workspace), counters(out.counters);
  size_t at = 0;
  for (int i = 0; i < n; ++i) {
    const sk_moe_problem &p = problems[(size_t)i];
    int64_t rows = 0;
    for (; rows < p.rows; ++at) {
      need(at < out.parts.size(), "parts");
      const sk::MoeDev &d = out.parts[at];
      need(d.row0 == rows && d.rows >= 1 && d.rows <= sk::MOE_ROWS, "rows of a part");
      rows += d.rows;
      const int64_t pairs = (int64_t)d.rows * d.top_k, places = pairs + (d.shared_ffn ? d.rows : 0);
      // the most groups that any choice can give: every expert has a pair, and one (or some) all others
      int64_t most = std::min<int64_t>(d.experts, pairs);
      most += (pairs - most) / sk::MOE_GROUP + (d.shared_ffn ? (d.rows + sk::MOE_GROUP - 1) / sk::MOE_GROUP : 0);
      need(d.most_groups >= most, "groups");
      const int64_t blocks = (d.rows + sk::ROUTE_ROWS - 1) / sk::ROUTE_ROWS;
      need(out.route_first[at + 1] - out.route_first[at] == blocks * ((d.experts + d.route_experts - 1) / d.route_experts), "units of the router");
      need(d.h_part >= 2 * std::max(d.ffn, d.shared_ffn) && d.h_part % 128 == 0 && d.h_stride == sk::H_PARTS * d.h_part, "strides of the workspace");
      need(d.y_stride == d.dim, "strides of the sums");
      need((int64_t)(out.add_first[at + 1] - out.add_first[at]) * 4 * sk::ADD_COLUMNS >= (int64_t)d.rows * d.dim, "units of the sums");
      need(d.count == out.counts + at, "counts");
      counters.next(d.routed, blocks * sk::COUNTER_STEP), counters.next(d.blocks_routed, sk::COUNTER_STEP);
      work.next(d.logits, (int64_t)d.rows * d.experts), work.next(d.ids, pairs), work.next(d.weights, pairs), work.next(d.row_of, pairs), work.next(d.place_at, pairs);
      work.next(d.groups, d.most_groups), work.next(d.first_begin, d.most_groups), work.next(d.second_begin, d.most_groups), work.next(d.h, places * d.h_stride), work.next(d.y, places * d.y_stride);
    }
    need(rows == p.rows, "all rows once");
  }
  need(at == out.parts.size(), "no other parts");
  for (const int64_t w : {out.up_workgroups, out.down_workgroups}) need(w >= 1 && (!workgroups || w <= workgroups), "workgroups");
  work.next(out.counts, (int64_t)out.parts.size());
}

// The shares of random work: every tile in one share, in their order.
static int32_t group_at(const std::vector<int64_t> &begin, int64_t at) {
  int32_t g = 0;
  while (g + 1 < (int32_t)begin.size() && begin[(size_t)g + 1] <= at) ++g;
  return g;
}
static void shares() {
  struct Group {
    int64_t each;
    int32_t tiles;
  };
  struct Part {
    std::vector<Group> groups;
    std::vector<int64_t> begin;
    int64_t work = 0;
  };
  std::vector<Part> parts((size_t)between(1, 4));
  int64_t total = 0;
  for (Part &p : parts) {
    const int32_t w = (int32_t)between(1, 2);
    for (int64_t n = between(0, between(0, 1) ? 3 : 90); n > 0; --n) {
      const int32_t mode = sk::moe::mode_of((int32_t)between(1, 32)), rows = (int32_t)between(1, between(0, 1) ? 300 : 20000);
      const Group g{sk::moe::cost((int32_t)between(1, between(0, 1) ? 300 : 9000), w, (int32_t)between(1, 2), mode), sk::moe::tiles_of(rows, w, mode)};
      need((int64_t)g.tiles * sk::moe::rows_of_tile(w, mode) >= rows && (int64_t)(g.tiles - 1) * sk::moe::rows_of_tile(w, mode) < rows, "tiles");
      p.groups.push_back(g);
      p.begin.push_back(p.work);
      p.work += g.each * g.tiles;
    }
    total += p.work;
  }
  const int64_t workgroups = between(1, between(0, 1) ? 20 : 1500);
  std::vector<std::pair<int32_t, int32_t>> seen(parts.size(), {0, 0});  // the next (group, tile)
  for (int64_t w = 0; w < workgroups; ++w) {
    const sk::moe::Share s = sk::moe::share_of(total, workgroups, w);
    int64_t offset = 0;
    for (size_t i = 0; i < parts.size(); ++i) {
      const Part &p = parts[i];
      if (offset < s.end && s.begin < offset + p.work && p.work > 0) {
        std::pair<int32_t, int32_t> ends[2];
        for (int e = 0; e < 2; ++e) {
          const int64_t at = e ? s.end - offset : std::max<int64_t>(s.begin - offset, 0);
          int32_t g = group_at(p.begin, at);
          int32_t t = sk::moe::tile_from(at, p.begin[(size_t)g], p.groups[(size_t)g].each, p.groups[(size_t)g].tiles);
          if (t == p.groups[(size_t)g].tiles) ++g, t = 0;
          ends[e] = {g, t};
        }
        if (ends[0] < ends[1]) {
          need(ends[0] == seen[i], "a tile is left out or done twice");
          seen[i] = ends[1];
        }
      }
      offset += p.work;
    }
  }
  for (size_t i = 0; i < parts.size(); ++i) need(seen[i] == std::make_pair((int32_t)parts[i].groups.size(), 0), "all tiles");
}

static void verifications() {
  const int n = (int)between(0, between(0, 3) ? 5 : 40);
  std::vector<sk_verify_problem> problems;
  for (int i = 0; i < n; ++i) {
    sk_verify_problem p{};
    p.dtype = (int32_t)between(0, 2), p.sequences = (int32_t)between(1, 100), p.rows = (int32_t)between(1, 600), p.vocab = (int32_t)between(1, between(0, 1) ? 200 : 200000);
    p.first_row = p.drafted = (const int32_t *)address(0), p.logits = address(0), p.accept_random = p.sample_random = (const float *)address(0);
    if (between(0, 1)) p.draft_logits = address(0);
    p.tokens = (int32_t *)address(2 * i + 1), p.accepted = (int32_t *)address(2 * i + 2);
    problems.push_back(p);
  }
  sk::VerifyPlanHost out;
  std::string err;
  need(sk::plan_verify(problems.data(), n, out, err) == SK_OK, err.c_str());
  Walk work(out.workspace), counters(out.counters);
  int seen = 0;
  for (const sk::VerifyLaunch &l : out.launches) {
    need(l.n >= 1 && l.n <= sk::VERIFY_PROBLEMS, "problems of a launch");
    for (int i = 0; i < sk::VERIFY_PROBLEMS; ++i) {
      if (i >= l.n) {
        need(l.table.stat_first[i] == 0xffffffffu && l.table.sum_first[i] == 0xffffffffu, "a place without a problem can be found");
        continue;
      }
      const sk::VerifyDev &d = l.table.problems[i];
      need(d.rows == problems[(size_t)seen].rows && d.vocab == problems[(size_t)seen].vocab, "problems in their order");
      need(d.pieces >= 1 && d.pieces <= 8 && (int64_t)d.chunks * d.pieces * 512 >= d.vocab && ((int64_t)d.chunks - 1) * d.pieces * 512 < d.vocab, "chunks");
      need((i + 1 < l.n ? l.table.stat_first[i + 1] : l.stat_grid) - l.table.stat_first[i] == ((int64_t)d.rows * (d.draft_logits ? 2 : 1) * d.chunks + 3) / 4, "units of the rows");
      need((i + 1 < l.n ? l.table.sum_first[i + 1] : l.sum_grid) - l.table.sum_first[i] == (int64_t)d.sequences * ((d.chunks + sk::VERIFY_CHUNKS - 1) / sk::VERIFY_CHUNKS), "units of the sequences");
      counters.next(d.arrived, (int64_t)d.sequences * sk::COUNTER_STEP);
      work.next(d.stats, (int64_t)d.rows * 2 * d.chunks), work.next(d.sums, (int64_t)d.sequences * d.chunks);
      ++seen;
    }
  }
  need(seen == n, "every problem once");
}

int main() {
  for (int i = 0; i < 400; ++i) norms(), moes(), shares(), verifications();
  std::printf("layer_driver: ok\n");
  return 0;
}
