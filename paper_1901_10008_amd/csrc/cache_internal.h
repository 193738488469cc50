// Internal declarations of libsk_cache.so, shared by its host planning and its kernels.  Not part of the public ABI
// (include/sk_cache.h is).
#pragma once

#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "launch_limits.h"
#include "sk_cache.h"
#include "sk_internal.h"

namespace sk {

// Rows of a unit of work (a key-value head of a sequence): few rows go in blocks of ROWS_FEW, whose four waves share the
// keys among them; more than most_few() rows go in blocks of ROWS_MANY, whose waves share the rows.
constexpr int ROWS_FEW = 16, ROWS_MANY = 128;
// Two blocks of few rows read the keys twice (the second time mostly out of the caches), a block of many rows keeps fewer loads in flight: 20 rows on
// caches of 8000 tokens, 16 sequences of 8 heads of 128 elements, 123 us as few and 105 as many, of 4000 tokens with heads of 64, 31 and 37, one head
// of 256 on 8000, 24 rows, 40 and 69.
constexpr int most_few(int dim) { return dim > 64 && dim <= 128 ? 16 : 32; }
constexpr int KEYS_FEW = 32;                                  // keys per step
constexpr int keys_many(int dim) { return dim <= 128 ? 64 : 32; }  // keys of a tile (heads of 256: two tiles of 64 would take 128 KB of LDS and 64 more registers)
constexpr int APPEND_WAVES = 8192;  // append: a problem's rows are cut into parts for at least that many waves where they have the heads for it
constexpr int MOST_SPLITS = 256;              // workgroups that share a unit's keys, at most

// A problem as the kernels see it (strides in elements).
struct AttnDev {
  const void *qkv, *q_weight, *k_weight;
  const float *cos, *sin;
  void *q, *out, *k, *v;
  const int32_t *table, *lengths, *first_row;
  int64_t page_stride, head_stride, token_stride, qkv_row, q_row, q_head, out_row, out_head;
  int32_t dtype, q_heads, kv_heads, group, dim, page_shift, num_pages, columns, sequences, rows, max_new, window, sinks;
  int32_t rotary, neighbours, positions;
  float eps, scale_log2;
  // append: a wave takes `parts`-th of a row's heads, `heads_at_once` (of 8 elements a lane) in each of `turns`
  int32_t lanes_per_head, turns, parts;
  int32_t pad;
  FastDiv by_group;  // divides by `group`
};

// A sequence of a launch: what a workgroup needs to know of it to count its units.
struct AttnSeq {
  const int32_t *length, *first;
  int32_t problem, seq, kv_heads, group, window, sinks, rows, max_new, most_few, pad;
  int64_t capacity;  // tokens that its row of the page table can hold
};

// One kernel launch of sk_attn_launch: the sequences of the problems with heads of up to 128 elements, or those with larger ones.
struct AttnGroup {
  bool wide, many;              // larger heads; units of many rows are possible
  int64_t first_seq, sequences; // in the plan's list
  int64_t workgroups;           // that the device runs at a time
  int64_t grid;                 // of the launch: the most units there can be, and that many for slices
  int64_t slots_many, slots_few;  // places of the workspace: as many as there can be slices of either kind
};
// Workgroups of a kernel that a compute unit holds (its registers and LDS).
constexpr int resident(bool wide, bool many) { return wide ? 1 : many ? 2 : 3; }

struct AttnPlanHost {
  std::vector<AttnDev> problems;
  std::vector<AttnSeq> seqs;
  std::vector<AttnGroup> groups;
  std::vector<uint32_t> append_first;  // first workgroup of each problem, and the number of all
  bool append_once = false;            // append moves more than PAST_CACHES bytes
  bool all_qkv = true, all_out = true;
  int64_t workspace_floats = 0, counters = 0;  // of the largest group: launches of a plan do not overlap
};

// Checks and plans for a device of that many compute units, or for that many workgroups at a time (0: what its compute units hold); no HIP
// call.  Returns SK_OK or an error with `err` set.
sk_status plan_attn(const sk_attn_problem *problems, int32_t n, int32_t compute_units, int32_t workgroups, AttnPlanHost &out, std::string &err);

// Floats of a split unit's partial result: outputs, running maximum and sum of each row.
constexpr int64_t part_floats(int64_t rows, int64_t most_dim) { return rows * (most_dim + 2); }

// One launch of page copies and of changed rows of the page table, by value.  words: n_arrays times base and bytes of a page (64 bits each), n_moves
// times from and to, then (if `rows` is null) n_rows row numbers and the rows; otherwise those stand in host memory.
struct PageMove {
  int32_t from, to;
};
constexpr int COPY_WORDS = 1008;
struct CopyArgs {
  int32_t n_arrays, n_moves, n_rows, columns;
  int64_t chunks;       // of COPY_CHUNK bytes per page, of the array with the largest pages
  int32_t *table;       // device page table
  const int32_t *rows;  // host memory that the device can read, or null
  int32_t words[COPY_WORDS];
};
static_assert(sizeof(CopyArgs) <= 4096, "kernel arguments");
constexpr int COPY_ARRAYS = 64, COPY_MOVES = (COPY_WORDS - 4 * COPY_ARRAYS) / 2;  // of a launch, at most
constexpr int64_t COPY_CHUNK = 32768;
constexpr int64_t COPY_PAGE = (int64_t)1 << 38;  // bytes of a page, at most
constexpr int32_t ROW_GROUPS = 1 << 16;          // workgroups that bring rows of the page table, at most
// Arrays and copies of one launch, at most, for arrays whose largest pages have that many chunks: what its arguments and its grid hold.
struct CopyBatch {
  int32_t arrays, moves;
};
constexpr CopyBatch copy_batch(int64_t chunks) {
  const int64_t groups = MOST_GRID - ROW_GROUPS;
  const int32_t arrays = chunks * COPY_ARRAYS <= groups ? COPY_ARRAYS : (int32_t)(groups / chunks);
  const int64_t moves = groups / (chunks * arrays);
  return CopyBatch{arrays, moves < COPY_MOVES ? (int32_t)moves : COPY_MOVES};
}
static_assert(copy_batch(1).moves == COPY_MOVES && copy_batch((COPY_PAGE + COPY_CHUNK - 1) / COPY_CHUNK).moves >= 1, "every page fits a launch");

// The account of pages.  A call that throws (std::bad_alloc) has changed nothing.
class PageAccount {
 public:
  PageAccount(int32_t num_pages, int32_t page_tokens, int32_t sequences, int32_t columns);
  sk_status resize(const int32_t *seqs, const int32_t *tokens, int32_t n, std::string &err);
  sk_status fork(int32_t from, const int32_t *to, int32_t n, std::string &err);
  sk_status compact();
  // The copies called for so far, in waves: the copies of one wave do not depend on each other, waves go in order.
  std::vector<std::vector<PageMove>> waves() const;
  const std::vector<int32_t> &dirty_rows() const { return dirty_; }
  // The copies have been made and, if `rows`, the changed rows brought to the device's table.
  void applied(bool rows = true);
  int32_t num_pages() const { return (int32_t)refs_.size(); }
  int32_t sequences() const { return (int32_t)tokens_.size(); }
  int32_t columns() const { return columns_; }
  int32_t free_pages() const { return free_; }
  int32_t pending() const { return (int32_t)moves_.size(); }
  int32_t tokens(int32_t s) const { return tokens_[s]; }
  const int32_t *row(int32_t s) const { return table_.data() + (size_t)s * columns_; }

 private:
  int32_t held(int32_t tokens) const { return (int32_t)(((uint32_t)tokens + (uint32_t)page_tokens_ - 1) / (uint32_t)page_tokens_); }
  int32_t take();
  void give(int32_t page);
  void room_for(size_t moves);
  void move(int32_t from, int32_t to);
  void touch(int32_t s);
  sk_status check_list(const int32_t *seqs, int32_t n, std::string &err);

  int32_t page_tokens_, columns_, free_, lowest_ = 0;  // no page below lowest_ is free
  std::vector<int32_t> refs_;                          // per page: sequences that hold it
  std::vector<int32_t> tokens_;                        // per sequence
  std::vector<int32_t> table_;
  std::vector<PageMove> moves_;          // the copies, and the wave of each, from 1 on
  std::vector<int32_t> wave_;
  std::vector<int32_t> read_, written_;  // per page: last wave that reads / writes it
  std::vector<int32_t> dirty_;
  std::vector<uint8_t> is_dirty_, mark_;
};

}  // namespace sk
