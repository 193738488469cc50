// Host side of libsk_layer.so without HIP calls: checks, grids, layout of workspaces.
#include <algorithm>
#include <cmath>
#include <utility>

#include "layer_internal.h"

namespace sk {

namespace {

sk_status refuse(std::string &err, sk_status st, const std::string &msg) {
  err = msg;
  return st;
}

bool known(int32_t dtype) { return dtype == SK_F32 || dtype == SK_BF16 || dtype == SK_F16; }
bool multiple(const void *p, int64_t of) { return (uintptr_t)p % (uintptr_t)of == 0; }

// The outputs of a plan, as spans of addresses.
struct Spans {
  std::vector<std::pair<uintptr_t, uintptr_t>> list;
  bool far = false;  // one does not fit the address space
  void add(const void *p, int64_t rows, int64_t stride, int64_t dim, int64_t size) {
    if (!p) return;
    const __int128 bytes = ((__int128)(rows - 1) * stride + dim) * size;
    if (bytes + (__int128)(uintptr_t)p > ((__int128)1 << 63)) far = true;
    else list.emplace_back((uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes);
  }
  bool overlap() {
    std::sort(list.begin(), list.end());
    for (size_t i = 1; i < list.size(); ++i)
      if (list[i].first < list[i - 1].second) return true;
    return false;
  }
};

// The inputs of a plan whose outputs must not touch them: rows of `dim` bytes, `stride` bytes apart.
struct Inputs {
  struct Rows {
    uintptr_t at;
    uint64_t rows, stride, dim;
  };
  std::vector<Rows> list;
  void add(const void *p, int64_t rows, int64_t stride, int64_t dim) {
    if (p) list.push_back(Rows{(uintptr_t)p, (uint64_t)rows, (uint64_t)stride, (uint64_t)dim});
  }
  void add(const void *p, int64_t bytes) { add(p, 1, 0, bytes); }
  // Whether one of them has a byte of an output (spans that are sorted, and do not overlap).  What lies between rows is not read.
  bool touch(const Spans &outputs) const {
    for (const Rows &r : list) {
      const uintptr_t end = r.at + (r.rows - 1) * r.stride + r.dim;
      auto it = std::upper_bound(outputs.list.begin(), outputs.list.end(), r.at, [](uintptr_t at, const std::pair<uintptr_t, uintptr_t> &o) { return at < o.second; });
      for (; it != outputs.list.end() && it->first < end; ++it) {
        // the first row that ends behind the output's beginning
        const uint64_t behind = it->first < r.at + r.dim ? 0 : r.stride ? (it->first - r.at - r.dim) / r.stride + 1 : r.rows;
        if (behind < r.rows && r.at + behind * r.stride < it->second) return true;
      }
    }
    return false;
  }
};

// A row stride as given, or packed.  false: it is negative, or rows would overlap (`one_for_all`: rows may share).
bool stride_of(int64_t given, int64_t dim, int64_t rows, int64_t &stride) {
  stride = given ? given : dim;
  return stride >= dim || (rows == 1 && stride >= 0);
}

template <class P, class F>
sk_status each(const P *problems, int32_t n, std::string &err, F f) {
  if (n < 0 || (n > 0 && !problems)) return refuse(err, SK_ERR_INVALID_ARG, "problems is null or n is negative");
  for (int32_t i = 0; i < n; ++i) {
    const sk_status st = f(problems[i]);
    if (st != SK_OK) {
      err = "problem " + std::to_string(i) + ": " + err;
      return st;
    }
  }
  return SK_OK;
}

// Places in a workspace.
struct Layout {
  size_t bytes = 0;
  template <class T>
  void take(T *&p, int64_t count, size_t align = 256) {
    bytes = (bytes + align - 1) / align * align;
    p = (T *)(uintptr_t)bytes;
    bytes += (size_t)count * sizeof(T);
  }
};

}  // namespace

// ---- norms -----------------------------------------------------------------------------------------------------------------

// From that many rows on a row gets no more than a wave or two, so that all of a workgroup's lanes have something of a row and more rows are on their way:
// 768 x 8000 20.2 us against 29.8 with a workgroup of four waves for each, 64 x 50000 13.2 against 76.  Below it they are alike, or the workgroups of
// four better (1536 x 1100: 8.0 us against 9.2).
constexpr int32_t NORM_MANY_ROWS = 2048;
// Problems of up to that many rows in all go together in the form of the longest of them: a launch costs more than idle threads.
constexpr int64_t NORM_STEP_ROWS = 1024;

sk_status plan_norm(const sk_norm_problem *problems, int32_t n, NormPlanHost &out, std::string &err) {
  Spans written;
  struct Item {
    NormForm form;
    NormDev dev;
    int64_t groups;
  };
  std::vector<Item> items;
  double bytes = 0.0;
  int64_t all_rows = 0;
  const sk_status st = each(problems, n, err, [&](const sk_norm_problem &p) -> sk_status {
    if (!known(p.dtype)) return refuse(err, SK_ERR_UNSUPPORTED, "dtype must be SK_F32, SK_BF16 or SK_F16");
    if (p.residual_dtype != p.dtype && p.residual_dtype != SK_F32) return refuse(err, SK_ERR_UNSUPPORTED, "residual_dtype must be dtype or SK_F32");
    if (p.rows < 1 || p.dim < 1) return refuse(err, SK_ERR_INVALID_ARG, "a size is less than 1");
    if (p.dim > norm_most_dim(NORM_LONG)) return refuse(err, SK_ERR_UNSUPPORTED, "rows of more than 32768 elements");
    if (p.kind != SK_NORM_RMS && p.kind != SK_NORM_LAYER) return refuse(err, SK_ERR_INVALID_ARG, "no such kind");
    if ((p.post != 0 && p.post != 1) || (p.gate_rows != 0 && p.gate_rows != 1) || p.reserved != 0) return refuse(err, SK_ERR_INVALID_ARG, "post and gate_rows must be 0 or 1, reserved 0");
    if (p.gate_act < SK_ACT_NONE || p.gate_act > SK_ACT_RELU) return refuse(err, SK_ERR_INVALID_ARG, "no such gate_act");
    if (!(p.eps >= 0.f) || !std::isfinite(p.eps) || !std::isfinite(p.residual_scale) || !std::isfinite(p.block_scale))
      return refuse(err, SK_ERR_INVALID_ARG, "eps is negative, or eps or a scale is not finite");
    if (!p.block && !p.residual) return refuse(err, SK_ERR_INVALID_ARG, "neither block nor residual is given");
    if (!p.residual_out && !p.next) return refuse(err, SK_ERR_INVALID_ARG, "neither residual_out nor next is given");
    NormDev d{};
    const int64_t dim = p.dim, one = elem_size(p.dtype), res = elem_size(p.residual_dtype);
    d.n_rows = p.n_rows, d.block = p.block, d.gate = p.block ? p.gate : nullptr, d.residual = p.residual;
    d.post_weight = p.post_weight, d.post_bias = p.post_bias, d.pre_weight = p.pre_weight, d.pre_bias = p.pre_bias;
    d.residual_out = p.residual_out, d.next = p.next;
    if (!stride_of(p.block_stride, dim, p.rows, d.block_stride) || !stride_of(p.residual_stride, dim, p.rows, d.residual_stride) ||
        !stride_of(p.residual_out_stride, dim, p.rows, d.residual_out_stride) || !stride_of(p.next_stride, dim, p.rows, d.next_stride) ||
        !stride_of(p.gate_stride, dim, p.gate_rows ? p.rows : 1, d.gate_stride))
      return refuse(err, SK_ERR_INVALID_ARG, "a stride is less than a row");
    if (!p.gate_rows) d.gate_stride = 0;
    for (const void *q : {p.block, p.gate, p.post_weight, p.post_bias, p.pre_weight, p.pre_bias, (const void *)p.next})
      if (!multiple(q, one)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers must be multiples of their elements' size");
    if (!multiple(p.residual, res) || !multiple(p.residual_out, res) || !multiple(p.n_rows, 4)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers must be multiples of their elements' size");
    written.add(p.residual_out, p.rows, d.residual_out_stride, dim, res);
    written.add(p.next, p.rows, d.next_stride, dim, one);
    Spans reach;  // (read, but they have to fit as well)
    reach.add(p.block, p.rows, d.block_stride, dim, one), reach.add(p.residual, p.rows, d.residual_stride, dim, res), reach.add(p.gate, p.rows, d.gate_stride, dim, one);
    if (written.far || reach.far) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
    d.rows = p.rows, d.dim = p.dim, d.eps = p.eps;
    d.residual_scale = p.residual_scale != 0.f ? p.residual_scale : 1.f, d.block_scale = p.block_scale != 0.f ? p.block_scale : 1.f;
    d.dtype = (int8_t)p.dtype, d.residual_dtype = (int8_t)p.residual_dtype, d.kind = (int8_t)p.kind, d.post = (int8_t)p.post, d.act = (int8_t)p.gate_act;
    int form = p.rows >= NORM_MANY_ROWS && dim <= norm_most_dim(NORM_ROWS) ? NORM_SIXTEEN : NORM_GROUP;
    while (dim > norm_most_dim((NormForm)form)) ++form;
    const int64_t of = norm_rows_of((NormForm)form), groups = ((int64_t)p.rows + of - 1) / of;
    if (groups > norm_most_grid((NormForm)form)) return refuse(err, SK_ERR_UNSUPPORTED, "more rows than a launch's grid can hold");
    all_rows += p.rows;
    bytes += (double)p.rows * dim * (double)(one * ((p.block != nullptr) + (d.gate && p.gate_rows) + (p.next != nullptr)) + res * ((p.residual != nullptr) + (p.residual_out != nullptr)));
    items.push_back(Item{(NormForm)form, d, groups});
    return SK_OK;
  });
  if (st != SK_OK) return st;
  if (written.overlap()) return refuse(err, SK_ERR_OVERLAP, "ranges of residual_out and next overlap");
  if (all_rows <= NORM_STEP_ROWS) {
    NormForm longest = NORM_GROUP;
    for (const Item &it : items) longest = std::max(longest, it.form);
    for (Item &it : items) it.form = longest;  // (none of them has many rows)
  }
  for (int f = 0; f < NORM_FORMS; ++f) {
    NormLaunch *l = nullptr;
    for (const Item &it : items) {
      if (it.form != (NormForm)f) continue;
      if (!l || l->n == NORM_PROBLEMS || l->grid + it.groups > norm_most_grid((NormForm)f)) {
        out.launches.emplace_back();
        l = &out.launches.back();
        l->form = (NormForm)f, l->once = bytes > (double)PAST_CACHES, l->grid = 0, l->n = 0;
        for (uint32_t &first : l->table.first) first = 0xffffffffu;
      }
      l->table.problems[l->n] = it.dev;
      l->table.first[l->n++] = (uint32_t)l->grid;
      l->grid += it.groups;
    }
  }
  return SK_OK;
}

// ---- mixture of experts ----------------------------------------------------------------------------------------------------

// The router splits its sums where that gives no more workgroups than the card holds at a time: 8 experts of 4096 and 2 rows 7.5 us instead of 11.1,
// 60 of 2048 and 61 rows (480 workgroups) 11.0 instead of 12.5; but 33 of 1000 and 250 rows (1071) 15.7 instead of 13.7.
constexpr int64_t ROUTE_SPLIT_UNITS = 512;

sk_status plan_moe(const sk_moe_problem *problems, int32_t n, int32_t compute_units, int32_t workgroups, MoePlanHost &out, std::string &err) {
  Spans written;
  out.route_first.assign(1, 0u), out.add_first.assign(1, 0u);
  int64_t route = 0, add = 0, tiles = 0;
  Layout counters, work;
  const sk_status st = each(problems, n, err, [&](const sk_moe_problem &p) -> sk_status {
    if (p.dtype != SK_BF16 && p.dtype != SK_F16) return refuse(err, SK_ERR_UNSUPPORTED, "dtype must be SK_BF16 or SK_F16");
    if (p.router_dtype != p.dtype && p.router_dtype != SK_F32) return refuse(err, SK_ERR_UNSUPPORTED, "router_dtype must be dtype or SK_F32");
    if (p.rows < 1 || p.dim < 1 || p.experts < 1 || p.top_k < 1 || p.ffn < 1 || p.shared_ffn < 0) return refuse(err, SK_ERR_INVALID_ARG, "a size is less than 1");
    if (p.top_k > p.experts) return refuse(err, SK_ERR_INVALID_ARG, "top_k is larger than the number of experts");
    if (p.experts > MOE_EXPERTS || p.top_k > MOE_TOP) return refuse(err, SK_ERR_UNSUPPORTED, "more than 512 experts or 32 chosen");
    if (p.dim % 8 || p.ffn % 8 || p.shared_ffn % 8) return refuse(err, SK_ERR_UNSUPPORTED, "dim and widths must be multiples of 8");
    if (p.dim >= 1 << 21 || p.ffn > 1 << 24 || p.shared_ffn > 1 << 24) return refuse(err, SK_ERR_UNSUPPORTED, "dim of 2^21 and more, or a width of more than 2^24");
    if (p.act < SK_ACT_NONE || p.act > SK_ACT_RELU) return refuse(err, SK_ERR_INVALID_ARG, "no such act");
    if (p.scoring != SK_MOE_SOFTMAX && p.scoring != SK_MOE_SIGMOID) return refuse(err, SK_ERR_INVALID_ARG, "no such scoring");
    if ((p.normalize != 0 && p.normalize != 1) || !std::isfinite(p.scale)) return refuse(err, SK_ERR_INVALID_ARG, "normalize must be 0 or 1, scale finite");
    if (!p.x || !p.router || !p.up || !p.down || !p.out) return refuse(err, SK_ERR_INVALID_ARG, "null pointer");
    if (p.shared_ffn && (!p.shared_up || !p.shared_down || (p.gate != nullptr) != (p.shared_gate != nullptr)))
      return refuse(err, SK_ERR_INVALID_ARG, "the shared expert has no weights, or a gate where the experts have none, or none where they have one");
    const int64_t dim = p.dim, ffn = p.ffn, rs = elem_size(p.router_dtype);
    int64_t x, o, r, ur, dr;
    if (!stride_of(p.x_stride, dim, p.rows, x) || !stride_of(p.out_stride, dim, p.rows, o) || !stride_of(p.router_stride, dim, p.experts, r) || !stride_of(p.up_row_stride, dim, ffn, ur) ||
        !stride_of(p.down_row_stride, ffn, dim, dr))
      return refuse(err, SK_ERR_INVALID_ARG, "a stride is less than a row");
    for (int64_t s : {x, o, r, ur, dr})
      if (s >= (int64_t)1 << 40) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
    if (x >= 1 << 21 || ur >= 1 << 26 || dr >= 1 << 26) return refuse(err, SK_ERR_UNSUPPORTED, "rows of x 2^21 elements apart and more, or rows of weights 2^26");
    int64_t ue, de;
    if (!stride_of(p.up_expert_stride, (ffn - 1) * ur + dim, p.experts, ue) || !stride_of(p.down_expert_stride, (dim - 1) * dr + ffn, p.experts, de))
      return refuse(err, SK_ERR_INVALID_ARG, "a stride lets experts overlap");
    if (!p.up_expert_stride) ue = ffn * ur;
    if (!p.down_expert_stride) de = dim * dr;
    if (ue >= (int64_t)1 << 50 || de >= (int64_t)1 << 50) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
    for (int64_t s : {x, o, ur, dr, ue, de})
      if (s % 8) return refuse(err, SK_ERR_UNSUPPORTED, "strides must be multiples of 16 bytes");
    if (r * rs % 16) return refuse(err, SK_ERR_UNSUPPORTED, "strides must be multiples of 16 bytes");
    for (const void *q : {p.x, p.router, p.gate, p.up, p.down, p.shared_gate, p.shared_up, p.shared_down, (const void *)p.out})
      if (!multiple(q, 16)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers must be multiples of 16 bytes");
    for (const void *q : {(const void *)p.n_rows, (const void *)p.router_bias, (const void *)p.expert_ids, (const void *)p.expert_weights})
      if (!multiple(q, 4)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers to numbers must be multiples of 4 bytes");
    written.add(p.out, p.rows, o, dim, 2);
    written.add(p.expert_ids, p.rows, p.top_k, p.top_k, 4);
    written.add(p.expert_weights, p.rows, p.top_k, p.top_k, 4);
    if (written.far) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
    for (int64_t row0 = 0; row0 < p.rows; row0 += MOE_ROWS) {
      MoeDev d{};
      const int64_t rows = std::min<int64_t>(MOE_ROWS, p.rows - row0), pairs = rows * p.top_k;
      d.n_rows = p.n_rows;
      d.x = (const char *)p.x + 2 * row0 * x, d.out = (char *)p.out + 2 * row0 * o;
      d.router = (const char *)p.router, d.gate = (const char *)p.gate, d.up = (const char *)p.up, d.down = (const char *)p.down;
      d.shared_gate = (const char *)p.shared_gate, d.shared_up = (const char *)p.shared_up, d.shared_down = (const char *)p.shared_down;
      d.bias = p.router_bias;
      d.user_ids = p.expert_ids ? p.expert_ids + row0 * p.top_k : nullptr;
      d.user_weights = p.expert_weights ? p.expert_weights + row0 * p.top_k : nullptr;
      d.x_stride = 2 * x, d.out_stride = 2 * o, d.router_stride = rs * r, d.up_expert = 2 * ue, d.down_expert = 2 * de, d.up_row = 2 * ur, d.down_row = 2 * dr;
      d.row0 = (int32_t)row0, d.rows = (int32_t)rows, d.dim = p.dim, d.experts = p.experts, d.top_k = p.top_k, d.ffn = p.ffn, d.shared_ffn = p.shared_ffn;
      d.act = p.act, d.scoring = p.scoring, d.normalize = p.normalize, d.dtype = p.dtype, d.router_f32 = p.router_dtype == SK_F32;
      d.scale = p.scale != 0.f ? p.scale : 1.f;
      // every group but the last of an expert has MOE_GROUP rows
      const int64_t blocks = (rows + ROUTE_ROWS - 1) / ROUTE_ROWS, shared_groups = p.shared_ffn ? (rows + MOE_GROUP - 1) / MOE_GROUP : 0;
      const int64_t reached = std::min<int64_t>(p.experts, pairs), routed_groups = reached + (pairs - reached) / MOE_GROUP;
      d.most_groups = (int32_t)(routed_groups + shared_groups);
      d.route_experts = blocks * ((p.experts + 1) / 2) <= ROUTE_SPLIT_UNITS ? 2 : 8;
      route += blocks * ((p.experts + d.route_experts - 1) / d.route_experts);
      add += (rows * ((p.dim + ADD_COLUMNS - 1) / ADD_COLUMNS) + 3) / 4;
      if (route > MOST_GRID || add > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more units of work than a launch's grid can hold");
      out.route_first.push_back((uint32_t)route), out.add_first.push_back((uint32_t)add);
      tiles += std::max(d.most_groups * ((dim + 15) / 16), routed_groups * ((ffn + 15) / 16) + shared_groups * (((int64_t)p.shared_ffn + 15) / 16));
      counters.take(d.routed, blocks * COUNTER_STEP), counters.take(d.blocks_routed, 1 * COUNTER_STEP);
      work.take(d.logits, rows * p.experts), work.take(d.ids, pairs), work.take(d.weights, pairs), work.take(d.row_of, pairs), work.take(d.place_at, pairs);
      work.take(d.groups, d.most_groups), work.take(d.first_begin, d.most_groups), work.take(d.second_begin, d.most_groups);
      d.h_part = (std::max<int64_t>(ffn, p.shared_ffn) + 63) / 64 * 128, d.h_stride = H_PARTS * d.h_part;
      d.y_stride = dim;
      const int64_t places = pairs + (p.shared_ffn ? rows : 0);
      work.take(d.h, places * d.h_stride), work.take(d.y, places * d.y_stride);
      out.parts.push_back(d);
    }
    return SK_OK;
  });
  if (st != SK_OK) return st;
  if (written.overlap()) return refuse(err, SK_ERR_OVERLAP, "ranges of out, expert_ids and expert_weights overlap");
  work.take(out.counts, (int64_t)out.parts.size());
  for (size_t i = 0; i < out.parts.size(); ++i) out.parts[i].count = out.counts + i;
  // never more than there can be tiles
  auto cut = [&](int64_t resident) { return std::max<int64_t>(1, std::min<int64_t>(workgroups ? workgroups : resident * compute_units, tiles)); };
  out.up_workgroups = cut(MOE_UP_RESIDENT), out.down_workgroups = cut(MOE_DOWN_RESIDENT);
  out.counters = counters.bytes;
  out.workspace = work.bytes;
  return SK_OK;
}

// ---- verification ----------------------------------------------------------------------------------------------------------

// Waves that the rows of a problem are cut for, where its chunks can still grow.
constexpr int64_t VERIFY_WAVES = 6000;

sk_status plan_verify(const sk_verify_problem *problems, int32_t n, VerifyPlanHost &out, std::string &err) {
  Spans written;
  Inputs read;
  Layout counters, work;
  const sk_status st = each(problems, n, err, [&](const sk_verify_problem &p) -> sk_status {
    if (!known(p.dtype)) return refuse(err, SK_ERR_UNSUPPORTED, "dtype must be SK_F32, SK_BF16 or SK_F16");
    if (p.sequences < 1 || p.rows < 1 || p.vocab < 1) return refuse(err, SK_ERR_INVALID_ARG, "a size is less than 1");
    if (p.sequences > 1 << 20) return refuse(err, SK_ERR_UNSUPPORTED, "more than 2^20 sequences");
    if (p.vocab > 1 << 30) return refuse(err, SK_ERR_UNSUPPORTED, "a vocabulary of more than 2^30 tokens");
    if (p.reserved != 0) return refuse(err, SK_ERR_INVALID_ARG, "reserved is not 0");
    if (!p.first_row || !p.logits || !p.sample_random || !p.tokens || !p.accepted || (p.drafted && !p.accept_random)) return refuse(err, SK_ERR_INVALID_ARG, "null pointer");
    VerifyDev d{};
    const int64_t one = elem_size(p.dtype);
    if (!stride_of(p.logits_stride, p.vocab, p.rows, d.logits_stride) || !stride_of(p.draft_stride, p.vocab, p.rows, d.draft_stride))
      return refuse(err, SK_ERR_INVALID_ARG, "a stride is less than a row");
    for (const void *q : {p.logits, p.draft_logits})
      if (!multiple(q, one)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers must be multiples of their elements' size");
    for (const void *q : {(const void *)p.first_row, (const void *)p.drafted, (const void *)p.temperatures, (const void *)p.accept_random, (const void *)p.sample_random, (const void *)p.tokens,
                          (const void *)p.accepted})
      if (!multiple(q, 4)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers to numbers must be multiples of 4 bytes");
    Spans reach;
    reach.add(p.logits, p.rows, d.logits_stride, p.vocab, one), reach.add(p.draft_logits, p.rows, d.draft_stride, p.vocab, one);
    written.add(p.tokens, 1, 0, p.rows, 4), written.add(p.accepted, 1, 0, p.sequences, 4);
    if (written.far || reach.far) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
    d.logits_stride *= one, d.draft_stride *= one;
    read.add(p.logits, p.rows, d.logits_stride, p.vocab * one), read.add(p.first_row, 4 * ((int64_t)p.sequences + 1)), read.add(p.sample_random, 4 * (int64_t)p.sequences);
    read.add(p.temperatures, 4 * (int64_t)p.sequences);
    if (p.drafted) read.add(p.drafted, 4 * (int64_t)p.rows), read.add(p.accept_random, 4 * (int64_t)p.rows), read.add(p.draft_logits, p.rows, d.draft_stride, p.vocab * one);
    d.first_row = p.first_row, d.drafted = p.drafted, d.logits = (const char *)p.logits, d.draft_logits = p.drafted ? (const char *)p.draft_logits : nullptr;
    d.temperatures = p.temperatures, d.accept_random = p.accept_random, d.sample_random = p.sample_random, d.tokens = p.tokens, d.accepted = p.accepted;
    d.dtype = p.dtype, d.sequences = p.sequences, d.rows = p.rows, d.vocab = p.vocab, d.temperature = p.temperature;
    // larger chunks where there are enough of them (up to four pieces: a lane keeps its part in registers, and eight waves a SIMD take 24.4 -> 23.6 us), and
    // a row is longer than one (the kernels' chunks of several pieces are for rows of eight logits and more)
    const int64_t lines = (int64_t)p.rows * (d.draft_logits ? 2 : 1);
    d.pieces = 1;
    while (d.pieces < VERIFY_PIECES && p.vocab > 512 * d.pieces && lines * ((p.vocab + 1024 * d.pieces - 1) / (1024 * d.pieces)) >= VERIFY_WAVES) d.pieces *= 2;
    const int64_t chunk = 512 * (int64_t)d.pieces;
    d.chunks = (int32_t)((p.vocab + chunk - 1) / chunk);
    const int64_t stat = (lines * d.chunks + 3) / 4, sum = p.sequences * (((int64_t)d.chunks + VERIFY_CHUNKS - 1) / VERIFY_CHUNKS);
    if (stat > MOST_GRID || sum > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more units of work than a launch's grid can hold");
    counters.take(d.arrived, (int64_t)p.sequences * COUNTER_STEP);
    work.take(d.stats, (int64_t)p.rows * 2 * d.chunks), work.take(d.sums, (int64_t)p.sequences * d.chunks);
    VerifyLaunch *l = out.launches.empty() ? nullptr : &out.launches.back();
    if (!l || l->n == VERIFY_PROBLEMS || l->stat_grid + stat > MOST_GRID || l->sum_grid + sum > MOST_GRID) {
      out.launches.emplace_back();
      l = &out.launches.back();
      l->n = 0, l->stat_grid = l->sum_grid = 0;
      for (int i = 0; i < VERIFY_PROBLEMS; ++i) l->table.stat_first[i] = l->table.sum_first[i] = 0xffffffffu;
    }
    l->table.problems[l->n] = d;
    l->table.stat_first[l->n] = (uint32_t)l->stat_grid, l->table.sum_first[l->n++] = (uint32_t)l->sum_grid;
    l->stat_grid += stat, l->sum_grid += sum;
    return SK_OK;
  });
  if (st != SK_OK) return st;
  if (written.overlap()) return refuse(err, SK_ERR_OVERLAP, "ranges of tokens and accepted overlap");
  if (read.touch(written)) return refuse(err, SK_ERR_OVERLAP, "tokens or accepted touch an input");
  out.counters = counters.bytes;
  out.workspace = work.bytes;
  return SK_OK;
}

}  // namespace sk
