// Plans of libsk_layer.so (layer_plan.cpp) on seeded random problems: every unit of a plan has a workgroup, every place of its workspace room.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "layer_internal.h"

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
  need(sk::plan_norm(problems.data(), n, 256, out, err) == SK_OK, err.c_str());
  int seen = 0;
  for (const sk::NormLaunch &l : out.launches) {
    need(l.n >= 1 && l.n <= sk::NORM_PROBLEMS, "problems of a launch");
    for (int i = 0; i < sk::NORM_PROBLEMS; ++i) {
      if (i >= l.n) {
        need(l.args.first[i] == 0xffffffffu, "a place without a problem can be found");
        continue;
      }
      const sk::NormDev &d = l.args.problems[i];
      need(d.dim <= sk::norm_most_dim(l.form), "a row longer than its form takes");
      const int64_t end = i + 1 < l.n ? l.args.first[i + 1] : l.grid, groups = end - l.args.first[i];
      need(l.form == sk::NORM_WAVE ? groups * 4 >= d.rows && (groups - 1) * 4 < d.rows : groups == d.rows, "workgroups of a problem");
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
  sk::MoePlanHost out;
  std::string err;
  need(sk::plan_moe(problems.data(), n, 256, out, err) == SK_OK, err.c_str());
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
      // the most groups that any choice can give: experts that are full but for one group each
      int64_t most = 0, left = pairs;
      for (int e = 0; e < d.experts && left > 0; ++e) most += 1, left -= 1;
      most += left / sk::MOE_GROUP;
      need(d.most_groups >= std::min(most, pairs), "groups");
      const int64_t blocks = (d.rows + sk::ROUTE_ROWS - 1) / sk::ROUTE_ROWS, shared = d.shared_ffn ? (d.rows + sk::MOE_GROUP - 1) / sk::MOE_GROUP : 0;
      need((int64_t)d.up_tiles * d.up_rows >= d.ffn && (int64_t)d.down_tiles * d.down_rows >= d.dim && (int64_t)d.shared_tiles * d.up_rows >= d.shared_ffn, "tiles");
      need(out.route_first[at + 1] - out.route_first[at] == blocks * ((d.experts + sk::ROUTE_EXPERTS - 1) / sk::ROUTE_EXPERTS), "units of the router");
      need(out.up_first[at + 1] - out.up_first[at] == (uint64_t)(d.most_groups * (int64_t)d.up_tiles + shared * d.shared_tiles), "units of up");
      need(out.down_first[at + 1] - out.down_first[at] == (uint64_t)((d.most_groups + shared) * d.down_tiles), "units of down");
      need(d.h_stride >= 2 * std::max(d.ffn, d.shared_ffn) && d.h_stride % 128 == 0 && d.part_stride >= d.dim, "strides of the workspace");
      counters.next(d.routed, blocks), counters.next(d.blocks_routed, 1), counters.next(d.summed, d.down_tiles);
      work.next(d.logits, (int64_t)d.rows * d.experts), work.next(d.ids, pairs), work.next(d.places, pairs), work.next(d.weights, pairs), work.next(d.row_of, pairs);
      work.next(d.groups, d.most_groups), work.next(d.n_groups, 1), work.next(d.h, places * d.h_stride), work.next(d.part, places * d.part_stride);
    }
    need(rows == p.rows, "all rows once");
  }
  need(at == out.parts.size(), "no other parts");
}

static void verifications() {
  const int n = (int)between(0, 5);
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
  need(sk::plan_verify(problems.data(), n, 256, out, err) == SK_OK, err.c_str());
  need((int)out.problems.size() == n, "problems");
  Walk work(out.workspace), counters(out.counters);
  for (int i = 0; i < n; ++i) {
    const sk::VerifyDev &d = out.problems[(size_t)i];
    need(d.pieces >= 1 && d.pieces <= 4 && (int64_t)d.chunks * d.pieces * 2048 >= d.vocab && ((int64_t)d.chunks - 1) * d.pieces * 2048 < d.vocab, "chunks");
    need(out.stat_first[i + 1] - out.stat_first[i] == (uint64_t)d.rows * (d.draft_logits ? 2 : 1) * d.chunks, "units of the rows");
    need(out.sum_first[i + 1] - out.sum_first[i] == (uint64_t)d.sequences * d.chunks, "units of the sequences");
    counters.next(d.arrived, d.sequences);
    work.next(d.stats, (int64_t)d.rows * 2 * d.chunks), work.next(d.sums, (int64_t)d.sequences * d.chunks);
  }
}

int main() {
  for (int i = 0; i < 400; ++i) norms(), moes(), verifications();
  std::printf("layer_driver: ok\n");
  return 0;
}
