// Host side of libsk_cache.so without HIP calls: checks and grids of attention plans, the account of pages.
#include <algorithm>
#include <cmath>
#include <utility>

#include "cache_internal.h"

namespace sk {

namespace {

sk_status refuse(std::string &err, sk_status st, const std::string &msg) {
  err = msg;
  return st;
}

bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Last element, plus one, of an array of rows x heads x dim with these strides; < 0: it does not fit 62 bits.
int64_t extent(int64_t rows, int64_t row_stride, int64_t heads, int64_t head_stride, int64_t dim) {
  const __int128 e = (__int128)(rows - 1) * row_stride + (__int128)(heads - 1) * head_stride + dim;
  return e > ((__int128)1 << 62) ? -1 : (int64_t)e;
}

// Strides of rows (or tokens) and heads under which no two vectors of `dim` elements overlap: one of them holds a vector, the other
// all that the first runs over.
bool apart(int64_t outer_n, int64_t outer, int64_t inner_n, int64_t inner, int64_t dim) {
  auto nested = [dim](int64_t big, int64_t small_n, int64_t small) { return small >= dim && (__int128)big >= (__int128)(small_n - 1) * small + dim; };
  if (outer_n == 1) return inner_n == 1 || inner >= dim;
  if (inner_n == 1) return outer >= dim;
  return nested(outer, inner_n, inner) || nested(inner, outer_n, outer);
}

sk_status check_problem(const sk_attn_problem &p, AttnDev &d, std::string &err) {
  if (p.dtype != SK_BF16 && p.dtype != SK_F16) return refuse(err, SK_ERR_UNSUPPORTED, "dtype must be SK_BF16 or SK_F16");
  if (p.q_heads < 1 || p.kv_heads < 1 || p.head_dim < 1 || p.page_tokens < 1 || p.num_pages < 1 || p.sequences < 1 || p.pages_per_sequence < 1 || p.rows < 1)
    return refuse(err, SK_ERR_INVALID_ARG, "a size is less than 1");
  if (p.sequences > 1 << 20) return refuse(err, SK_ERR_UNSUPPORTED, "more than 2^20 sequences");
  if ((int64_t)p.q_heads + 2 * (int64_t)p.kv_heads > (int64_t)1 << 30) return refuse(err, SK_ERR_UNSUPPORTED, "more than 2^30 heads");
  if (p.max_new < 0 || p.window < 0 || p.sinks < 0 || p.rotary_dim < 0 || p.reserved != 0)
    return refuse(err, SK_ERR_INVALID_ARG, "max_new, window, sinks or rotary_dim is negative, or reserved is not 0");
  if (p.q_heads % p.kv_heads) return refuse(err, SK_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (p.head_dim % 8 || p.head_dim > 256) return refuse(err, SK_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 256");
  if (p.page_tokens < 16 || p.page_tokens > 65536 || (p.page_tokens & (p.page_tokens - 1)))
    return refuse(err, SK_ERR_UNSUPPORTED, "page_tokens must be a power of two from 16 to 65536");
  if ((int64_t)p.pages_per_sequence * p.page_tokens >= (int64_t)1 << 31) return refuse(err, SK_ERR_UNSUPPORTED, "a sequence of 2^31 tokens and more");
  if ((int64_t)p.rows * p.q_heads >= (int64_t)1 << 31) return refuse(err, SK_ERR_UNSUPPORTED, "2^31 query vectors and more");
  if (p.rotary_dim % 2 || p.rotary_dim > p.head_dim) return refuse(err, SK_ERR_INVALID_ARG, "rotary_dim must be even and at most head_dim");
  if (p.neighbours != 0 && p.neighbours != 1) return refuse(err, SK_ERR_INVALID_ARG, "neighbours must be 0 or 1");
  if (!(p.eps >= 0.f) || !std::isfinite(p.eps) || !std::isfinite(p.scale)) return refuse(err, SK_ERR_INVALID_ARG, "eps is negative, or eps or scale is not finite");
  if (!p.k || !p.v || !p.page_table || !p.lengths || !p.first_row || !p.q) return refuse(err, SK_ERR_INVALID_ARG, "null pointer");
  if (!p.qkv && !p.out) return refuse(err, SK_ERR_INVALID_ARG, "neither qkv nor out is given");
  for (int64_t s : {p.page_stride, p.kv_head_stride, p.token_stride, p.qkv_row_stride, p.q_row_stride, p.q_head_stride, p.out_row_stride, p.out_head_stride})
    if (s < 0) return refuse(err, SK_ERR_INVALID_ARG, "negative stride");
  const int64_t dim = p.head_dim;
  d = AttnDev{};
  d.qkv = p.qkv, d.q_weight = p.q_weight, d.k_weight = p.k_weight, d.cos = p.cos, d.sin = p.sin;
  d.q = p.q, d.out = p.out, d.k = p.k, d.v = p.v, d.table = p.page_table, d.lengths = p.lengths, d.first_row = p.first_row;
  const bool packed = !p.page_stride && !p.kv_head_stride && !p.token_stride;
  d.token_stride = packed ? dim : p.token_stride;
  d.head_stride = packed ? dim * p.page_tokens : p.kv_head_stride;
  d.page_stride = packed ? dim * p.page_tokens * p.kv_heads : p.page_stride;
  const int64_t heads_in = p.q_heads + 2 * (int64_t)p.kv_heads;
  d.qkv_row = p.qkv_row_stride ? p.qkv_row_stride : heads_in * dim;
  d.q_row = p.q_row_stride || p.q_head_stride ? p.q_row_stride : p.q_heads * dim;
  d.q_head = p.q_row_stride || p.q_head_stride ? p.q_head_stride : dim;
  d.out_row = p.out_row_stride || p.out_head_stride ? p.out_row_stride : p.q_heads * dim;
  d.out_head = p.out_row_stride || p.out_head_stride ? p.out_head_stride : dim;
  if (!apart(p.page_tokens, d.token_stride, p.kv_heads, d.head_stride, dim) ||
      (p.num_pages > 1 && d.page_stride < dim))
    return refuse(err, SK_ERR_INVALID_ARG, "the cache's strides let tokens or heads overlap");
  if (d.qkv_row < heads_in * dim) return refuse(err, SK_ERR_INVALID_ARG, "qkv_row_stride is less than a row");
  if (!apart(p.rows, d.q_row, p.q_heads, d.q_head, dim)) return refuse(err, SK_ERR_INVALID_ARG, "the strides of q let rows or heads overlap");
  if (p.out && !apart(p.rows, d.out_row, p.q_heads, d.out_head, dim)) return refuse(err, SK_ERR_INVALID_ARG, "the strides of out let rows or heads overlap");
  // a page as a whole (heads and tokens) lies before the next, or pages lie between the heads' or tokens' parts: then its vectors must still be apart
  const int64_t page_extent = extent(p.page_tokens, d.token_stride, p.kv_heads, d.head_stride, dim);
  if (page_extent < 0 || extent(p.num_pages, d.page_stride, 1, 0, page_extent) < 0) return refuse(err, SK_ERR_UNSUPPORTED, "the cache's strides reach too far");
  if (p.num_pages > 1 && d.page_stride < page_extent) {
    const __int128 all = (__int128)(p.num_pages - 1) * d.page_stride;
    const bool inside_heads = p.kv_heads > 1 && d.page_stride >= (__int128)(p.page_tokens - 1) * d.token_stride + dim && d.token_stride <= d.page_stride &&
                              d.head_stride >= all + (__int128)(p.page_tokens - 1) * d.token_stride + dim;
    if (!inside_heads) return refuse(err, SK_ERR_INVALID_ARG, "the cache's strides let pages overlap");
  }
  if (d.token_stride >= (int64_t)1 << 26) return refuse(err, SK_ERR_UNSUPPORTED, "token_stride of 2^26 elements and more");
  for (int64_t s : {d.page_stride, d.head_stride, d.token_stride, d.qkv_row, d.q_row, d.q_head, d.out_row, d.out_head})
    if (s % 8) return refuse(err, SK_ERR_UNSUPPORTED, "strides must be multiples of 16 bytes");
  for (const void *q : {(const void *)p.k, (const void *)p.v, p.qkv, p.q_weight, p.k_weight, (const void *)p.cos, (const void *)p.sin, (const void *)p.q, (const void *)p.out})
    if (!aligned(q)) return refuse(err, SK_ERR_UNSUPPORTED, "pointers must be multiples of 16 bytes");
  if (((uintptr_t)p.page_table | (uintptr_t)p.lengths | (uintptr_t)p.first_row) & 3) return refuse(err, SK_ERR_UNSUPPORTED, "pointers to numbers must be multiples of 4 bytes");
  for (int64_t e : {extent(p.rows, d.qkv_row, 1, 0, heads_in * dim), extent(p.rows, d.q_row, p.q_heads, d.q_head, dim), extent(p.rows, d.out_row, p.q_heads, d.out_head, dim)})
    if (e < 0) return refuse(err, SK_ERR_UNSUPPORTED, "a stride reaches too far");
  if (p.qkv && p.rotary_dim) {
    if (!p.cos || !p.sin) return refuse(err, SK_ERR_INVALID_ARG, "rotary_dim is given without cos and sin");
    if ((int64_t)p.positions < (int64_t)p.pages_per_sequence * p.page_tokens)
      return refuse(err, SK_ERR_INVALID_ARG, "cos and sin have fewer rows than a sequence can have tokens");
  }
  d.dtype = p.dtype, d.q_heads = p.q_heads, d.kv_heads = p.kv_heads, d.group = p.q_heads / p.kv_heads, d.dim = p.head_dim;
  d.by_group = fast_div_of((uint32_t)d.group);
  while ((1 << d.page_shift) < p.page_tokens) ++d.page_shift;
  d.num_pages = p.num_pages, d.columns = p.pages_per_sequence, d.sequences = p.sequences, d.rows = p.rows;
  d.max_new = p.max_new && p.max_new < p.rows ? p.max_new : p.rows;
  d.window = p.window, d.sinks = p.sinks, d.rotary = p.qkv ? p.rotary_dim : 0, d.neighbours = p.neighbours, d.positions = p.positions, d.eps = p.eps;
  d.scale_log2 = (float)((p.scale != 0.f ? (double)p.scale : 1.0 / std::sqrt((double)dim)) * 1.4426950408889634);
  if (!std::isfinite(d.scale_log2)) return refuse(err, SK_ERR_INVALID_ARG, "scale times log2(e) is not finite");
  return SK_OK;
}

}  // namespace

sk_status plan_attn(const sk_attn_problem *problems, int32_t n, int32_t compute_units, int32_t workgroups, AttnPlanHost &out, std::string &err) {
  if (n < 0 || (n > 0 && !problems)) return refuse(err, SK_ERR_INVALID_ARG, "problems is null or n is negative");
  std::vector<std::pair<uintptr_t, uintptr_t>> written;
  int64_t append_grid = 0;
  out.append_first.assign(1, 0u);
  for (int32_t i = 0; i < n; ++i) {
    AttnDev d;
    sk_status st = check_problem(problems[i], d, err);
    if (st != SK_OK) {
      err = "problem " + std::to_string(i) + ": " + err;
      return st;
    }
    out.all_qkv = out.all_qkv && d.qkv;
    out.all_out = out.all_out && d.out;
    if (d.qkv) written.emplace_back((uintptr_t)d.q, (uintptr_t)d.q + 2 * (uintptr_t)extent(d.rows, d.q_row, d.q_heads, d.q_head, d.dim));
    if (d.out) written.emplace_back((uintptr_t)d.out, (uintptr_t)d.out + 2 * (uintptr_t)extent(d.rows, d.out_row, d.q_heads, d.out_head, d.dim));
    // append: 8 elements a lane; a wave takes a whole row's heads where there are rows enough to fill the card, a part of them otherwise
    const int64_t heads = d.q_heads + 2 * (int64_t)d.kv_heads;
    d.lanes_per_head = 1;
    while (d.lanes_per_head * 8 < d.dim) d.lanes_per_head *= 2;
    const int64_t at_once = 64 / d.lanes_per_head, most = (heads + at_once - 1) / at_once;
    d.turns = (int32_t)std::max<int64_t>(1, std::min(most, (int64_t)d.rows * most / APPEND_WAVES));
    d.parts = (int32_t)((most + d.turns - 1) / d.turns);
    append_grid += d.qkv ? ((int64_t)d.rows * d.parts + 3) / 4 : 0;
    if (append_grid > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more rows than a launch's grid can hold");
    out.append_first.push_back((uint32_t)append_grid);
    out.problems.push_back(d);
  }
  int64_t moved = 0;
  for (const AttnDev &d : out.problems) moved += d.qkv ? 4 * (int64_t)d.rows * (d.q_heads + 2 * (int64_t)d.kv_heads) * d.dim : 0;
  out.append_once = moved > PAST_CACHES;
  std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].first < written[i - 1].second) return refuse(err, SK_ERR_OVERLAP, "ranges of q and out overlap");

  for (bool wide : {false, true}) {
    AttnGroup g{};
    g.wide = wide, g.first_seq = (int64_t)out.seqs.size();
    int64_t few = 0, many = 0, few_most = 0, many_most = 0;  // units, and slices of them, at most
    for (int32_t i = 0; i < n; ++i) {
      const AttnDev &d = out.problems[(size_t)i];
      if (!d.out || (d.dim > 128) != wide) continue;
      const int64_t capacity = (int64_t)d.columns << d.page_shift, most_rows = (int64_t)d.max_new * d.group;
      const int64_t blocks = (std::min<int64_t>(most_rows, most_few(d.dim)) + ROWS_FEW - 1) / ROWS_FEW, units = (int64_t)d.sequences * d.kv_heads * blocks;
      few += units;
      if (few > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more units of work than a launch's grid can hold");
      few_most += units * (capacity / (4 * KEYS_FEW) + 2);
      if (most_rows > most_few(d.dim)) {
        // sequences of many rows: their blocks are full but for one each
        const int64_t rows = (int64_t)d.rows * d.group, full = d.kv_heads * (rows / ROWS_MANY + std::min<int64_t>(d.sequences, rows / (most_few(d.dim) + 1) + 1));
        many += full;
        if (many > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more units of work than a launch's grid can hold");
        many_most += full * (capacity / (4 * keys_many(d.dim)) + 2);
      }
      for (int32_t s = 0; s < d.sequences; ++s)
        out.seqs.push_back(AttnSeq{d.lengths + s, d.first_row + s, i, s, d.kv_heads, d.group, d.window, d.sinks, d.rows, d.max_new, most_few(d.dim), 0, capacity});
    }
    g.sequences = (int64_t)out.seqs.size() - g.first_seq;
    if (!g.sequences) continue;
    g.many = many > 0;
    g.workgroups = workgroups ? workgroups : (int64_t)resident(g.wide, g.many) * compute_units;
    g.grid = std::min(few + many + g.workgroups, few_most + many_most);
    g.slots_few = std::min(2 * g.workgroups, few_most);
    g.slots_many = std::min(2 * g.workgroups, many_most);
    if (g.grid > MOST_GRID) return refuse(err, SK_ERR_UNSUPPORTED, "more units of work than a launch's grid can hold");
    const int64_t dim = wide ? 256 : 128;
    out.workspace_floats = std::max(out.workspace_floats, g.slots_few * part_floats(ROWS_FEW, dim) + g.slots_many * part_floats(ROWS_MANY, dim));
    out.counters = std::max(out.counters, g.slots_few + g.slots_many);
    out.groups.push_back(g);
  }
  return SK_OK;
}

// ---- pages -----------------------------------------------------------------------------------------------------------------

PageAccount::PageAccount(int32_t num_pages, int32_t page_tokens, int32_t sequences, int32_t columns)
    : page_tokens_(page_tokens), columns_(columns), free_(num_pages), refs_((size_t)num_pages, 0), tokens_((size_t)sequences, 0),
      table_((size_t)sequences * columns, -1), read_((size_t)num_pages, 0), written_((size_t)num_pages, 0),
      is_dirty_((size_t)sequences, 0), mark_((size_t)sequences, 0) {
  // the device's table starts out unknown
  dirty_.reserve((size_t)sequences);
  for (int32_t s = 0; s < sequences; ++s) touch(s);
}

void PageAccount::touch(int32_t s) {
  if (is_dirty_[s]) return;
  is_dirty_[s] = 1;
  dirty_.push_back(s);
}

int32_t PageAccount::take() {
  while (refs_[lowest_]) ++lowest_;
  refs_[lowest_] = 1;
  --free_;
  return lowest_++;
}

void PageAccount::give(int32_t page) {
  if (--refs_[page]) return;
  ++free_;
  if (page < lowest_) lowest_ = page;
}

// Room for so many more copies: nothing behind it needs memory.
void PageAccount::room_for(size_t moves) {
  const size_t wanted = moves_.size() + moves;
  if (wanted <= std::min(moves_.capacity(), wave_.capacity())) return;
  moves_.reserve(std::max(wanted, 2 * moves_.size()));
  wave_.reserve(std::max(wanted, 2 * moves_.size()));
}

// A copy goes into the first wave behind all that wrote its source or read or wrote its target.
void PageAccount::move(int32_t from, int32_t to) {
  const int32_t w = std::max(written_[from], std::max(read_[to], written_[to])) + 1;
  moves_.push_back(PageMove{from, to});
  wave_.push_back(w);
  read_[from] = std::max(read_[from], w);
  written_[to] = w;
}

std::vector<std::vector<PageMove>> PageAccount::waves() const {
  std::vector<std::vector<PageMove>> waves(wave_.empty() ? 0 : (size_t)*std::max_element(wave_.begin(), wave_.end()));
  for (size_t i = 0; i < moves_.size(); ++i) waves[(size_t)wave_[i] - 1].push_back(moves_[i]);
  return waves;
}

void PageAccount::applied(bool rows) {
  for (const PageMove &m : moves_) read_[m.from] = written_[m.from] = read_[m.to] = written_[m.to] = 0;
  moves_.clear();
  wave_.clear();
  if (!rows) return;
  for (int32_t s : dirty_) is_dirty_[s] = 0;
  dirty_.clear();
}

sk_status PageAccount::check_list(const int32_t *seqs, int32_t n, std::string &err) {
  sk_status st = SK_OK;
  int32_t i = 0;
  for (; i < n; ++i) {
    if (seqs[i] < 0 || seqs[i] >= sequences() || mark_[seqs[i]]) {
      st = refuse(err, SK_ERR_INVALID_ARG, "sequence " + std::to_string(seqs[i]) + " is not one of the account's, or stands twice");
      break;
    }
    mark_[seqs[i]] = 1;
  }
  while (i-- > 0) mark_[seqs[i]] = 0;
  return st;
}

sk_status PageAccount::resize(const int32_t *seqs, const int32_t *tokens, int32_t n, std::string &err) {
  sk_status st = check_list(seqs, n, err);
  if (st != SK_OK) return st;
  int64_t wanted = 0, before = 0;  // pages taken, and those given back by then
  for (int32_t i = 0; i < n; ++i) {
    if (tokens[i] < 0) return refuse(err, SK_ERR_INVALID_ARG, "a negative number of tokens");
    if ((int64_t)tokens[i] > (int64_t)columns_ * page_tokens_) return refuse(err, SK_ERR_INVALID_ARG, "more tokens than a row of the page table can hold");
  }
  room_for((size_t)n);
  // Sequences that shrink go first, so that what they give back serves the others; pages that two of them share are counted as they go.
  for (int32_t i = 0; i < n; ++i) {
    const int32_t s = seqs[i], has = held(tokens_[s]), will = held(tokens[i]);
    if (tokens[i] > tokens_[s]) {
      wanted += will - has;
      const int32_t last = tokens_[s] % page_tokens_ ? row(s)[has - 1] : -1;
      if (last >= 0 && refs_[last] > 1) ++wanted;  // (at most: one of its holders keeps it)
    }
  }
  if (wanted > free_) {
    // exactly, on a copy: rare, and the caller is about to be told that there are too few pages
    std::vector<int32_t> refs = refs_;
    int64_t have = free_;
    for (int32_t i = 0; i < n; ++i)
      for (int32_t c = held(tokens[i]); tokens[i] < tokens_[seqs[i]] && c < held(tokens_[seqs[i]]); ++c)
        if (--refs[row(seqs[i])[c]] == 0) ++have;
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs[i], has = held(tokens_[s]);
      if (tokens[i] <= tokens_[s]) continue;
      before += held(tokens[i]) - has;
      const int32_t last = tokens_[s] % page_tokens_ ? row(s)[has - 1] : -1;
      if (last >= 0 && refs[last] > 1) --refs[last], ++before;
    }
    if (before > have) return refuse(err, SK_ERR_ALLOC, "too few free pages: " + std::to_string(before) + " wanted, " + std::to_string(have) + " free");
  }
  for (int32_t i = 0; i < n; ++i) {
    const int32_t s = seqs[i];
    if (tokens[i] >= tokens_[s]) continue;
    int32_t *r = table_.data() + (size_t)s * columns_;
    const int32_t will = held(tokens[i]), has = held(tokens_[s]);  // (a division each: outside the loop, 784 pages 3 us)
    for (int32_t c = will; c < has; ++c) give(r[c]);
    std::fill(r + will, r + std::max(will, has), -1);
    tokens_[s] = tokens[i];
    touch(s);
  }
  for (int32_t i = 0; i < n; ++i) {
    const int32_t s = seqs[i];
    if (tokens[i] <= tokens_[s]) continue;
    int32_t *r = table_.data() + (size_t)s * columns_;
    const int32_t has = held(tokens_[s]), will = held(tokens[i]);
    if (tokens_[s] % page_tokens_ && refs_[r[has - 1]] > 1) {
      const int32_t own = take();
      move(r[has - 1], own);
      give(r[has - 1]);
      r[has - 1] = own;
      touch(s);
    }
    for (int32_t c = has; c < will; ++c) {
      r[c] = take();
      touch(s);
    }
    tokens_[s] = tokens[i];
  }
  return SK_OK;
}

sk_status PageAccount::fork(int32_t from, const int32_t *to, int32_t n, std::string &err) {
  if (from < 0 || from >= sequences()) return refuse(err, SK_ERR_INVALID_ARG, "sequence " + std::to_string(from) + " is not one of the account's");
  sk_status st = check_list(to, n, err);
  if (st != SK_OK) return st;
  for (int32_t i = 0; i < n; ++i)
    if (to[i] == from || tokens_[to[i]]) return refuse(err, SK_ERR_INVALID_ARG, "sequence " + std::to_string(to[i]) + " is not empty");
  const int32_t has = held(tokens_[from]);
  for (int32_t i = 0; i < n; ++i) {
    std::copy_n(table_.data() + (size_t)from * columns_, columns_, table_.data() + (size_t)to[i] * columns_);
    tokens_[to[i]] = tokens_[from];
    touch(to[i]);
  }
  for (int32_t c = 0; c < has; ++c) refs_[row(from)[c]] += n;
  return SK_OK;
}

sk_status PageAccount::compact() {
  const int32_t used = num_pages() - free_;
  std::vector<int32_t> now((size_t)num_pages(), -1);
  size_t high = 0;
  for (int32_t p = used; p < num_pages(); ++p) high += refs_[p] != 0;
  room_for(high);
  int32_t to = 0;
  for (int32_t p = used; p < num_pages(); ++p) {
    if (!refs_[p]) continue;
    while (refs_[to]) ++to;
    now[p] = to;
    move(p, to);
    std::swap(refs_[p], refs_[to]);
  }
  for (int32_t s = 0; s < sequences(); ++s) {
    int32_t *r = table_.data() + (size_t)s * columns_;
    for (int32_t c = 0, has = held(tokens_[s]); c < has; ++c)
      if (now[r[c]] >= 0) {
        r[c] = now[r[c]];
        touch(s);
      }
  }
  lowest_ = used;
  return SK_OK;
}

}  // namespace sk
