// Internal declarations of libsk_layer.so, shared by its host planning and its kernels.  Not part of the public ABI
// (include/sk_layer.h is).
#pragma once

#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "launch_limits.h"
#include "sk_internal.h"
#include "sk_layer.h"

namespace sk {

// Counters of arrivals stand a line of 128 bytes apart: atomics on one line go one after the other, across the whole card.
constexpr int COUNTER_STEP = 32;

// ---- norms -----------------------------------------------------------------------------------------------------------------

// A problem as the kernel sees it (strides in elements).
struct NormDev {
  const int32_t *n_rows;
  const void *block, *gate, *residual, *post_weight, *post_bias, *pre_weight, *pre_bias;
  void *residual_out, *next;
  int64_t block_stride, gate_stride, residual_stride, residual_out_stride, next_stride;  // (gate_stride 0: one gate for all rows)
  int32_t rows, dim;
  float eps, residual_scale, block_scale;
  int8_t dtype, residual_dtype, kind, post, act, pad[3];
};
constexpr int NORM_PROBLEMS = 16;  // of a launch
// Of a launch, in device memory.  (By value in the launch's arguments, which are in host memory, a step of three rows took 4.9 us.)
struct NormTable {
  uint32_t first[NORM_PROBLEMS];  // workgroup of the launch; none: the largest number
  NormDev problems[NORM_PROBLEMS];
};

// What a row gets, and up to how many elements it has: where there are many rows sixteen lanes (256), a wave (1024) or a workgroup of two waves (2048),
// otherwise a workgroup of four (4096), eight (8192) or sixteen (32768).
enum NormForm { NORM_SIXTEEN, NORM_WAVE, NORM_ROWS, NORM_GROUP, NORM_PAIR, NORM_LONG, NORM_FORMS };
constexpr int norm_threads(NormForm f) { return f == NORM_LONG ? 1024 : f == NORM_PAIR ? 512 : f == NORM_ROWS ? 128 : 256; }  // of a workgroup
constexpr int norm_rows_of(NormForm f) { return f == NORM_SIXTEEN ? 16 : f == NORM_WAVE ? 4 : 1; }  // of a workgroup
constexpr int norm_most_dim(NormForm f) {
  return f == NORM_SIXTEEN ? 256 : f == NORM_WAVE ? 1024 : f == NORM_ROWS ? 2048 : f == NORM_GROUP ? 4096 : f == NORM_PAIR ? 8192 : 32768;
}
constexpr int64_t norm_most_grid(NormForm f) { return (((int64_t)1 << 32) - 1) / norm_threads(f); }

struct NormLaunch {
  NormForm form;
  bool once;  // it moves more than PAST_CACHES bytes
  int32_t n;
  int64_t grid;
  NormTable table;
};
struct NormPlanHost {
  std::vector<NormLaunch> launches;
};

// ---- mixture of experts ----------------------------------------------------------------------------------------------------

constexpr int MOE_ROWS = 512;     // rows that are routed together; problems of more are cut
constexpr int MOE_EXPERTS = 512, MOE_TOP = 32;
constexpr int MOE_GROUP = 32;     // rows of an expert that a unit of work takes at most
constexpr int MOE_UP_RESIDENT = 3, MOE_DOWN_RESIDENT = 4;  // workgroups of the products that a compute unit holds (its registers)
constexpr int H_PARTS = 2;     // planes of the first products' results, which are 32 bits: the even and the odd fours of a row
constexpr int ROUTE_ROWS = 4;  // of a unit of the router
constexpr int ADD_COLUMNS = 256;                  // of a row that a wave adds up

// Rows of an expert that go together: its number (or -1: the shared one), the first of their places, how many.
struct MoeGroup {
  int32_t expert, first, rows, pad;
};
// What the router found: groups, rows; all work of the first products, and of the second ones.
struct MoeCount {
  int32_t groups, rows;
  int64_t first_work, second_work;
};

// Up to MOE_ROWS rows of a problem, as the kernels see them (strides in bytes but for logits and y; `h` and `y` have a place for every pair of a row and an expert
// that it chose, then one for every row).
struct MoeDev {
  const int32_t *n_rows;
  const char *x, *router, *gate, *up, *down, *shared_gate, *shared_up, *shared_down;
  const float *bias;
  char *out;
  int32_t *user_ids;
  float *user_weights;
  int64_t x_stride, out_stride, router_stride, up_expert, down_expert, up_row, down_row;
  int32_t row0, rows, dim, experts, top_k, ffn, shared_ffn, act, scoring, normalize, dtype, router_f32;
  float scale;
  int32_t most_groups;                               // with those of the shared expert
  int32_t route_experts;                             // of a unit of the router: 2 or 8
  // workspace
  double *logits;         // [rows][experts]
  int32_t *ids;           // [rows][top_k]: chosen experts
  float *weights;         // [rows][top_k]
  int32_t *row_of;        // [rows * top_k]: of a place
  int32_t *place_at;      // [rows][top_k]
  MoeGroup *groups;       // [most_groups]; those of the shared expert last
  int64_t *first_begin, *second_begin;  // [most_groups]: where a group's work begins, among the first and the second products
  MoeCount *count;
  uint32_t *routed;       // counters, COUNTER_STEP apart: of units of the router per ROUTE_ROWS rows, of such blocks
  uint32_t *blocks_routed;
  char *h;                // [rows * top_k + rows], h_stride bytes apart
  float *y;               // of the second products, y_stride elements apart
  int64_t h_stride, h_part, y_stride;  // h_part: from a row's first plane to its second, in bytes
};

struct MoePlanHost {
  std::vector<MoeDev> parts;          // workspace pointers: offsets until the plan is on the device
  std::vector<uint32_t> route_first, add_first;  // first workgroup of the router, and of the sums, of each part, and the number of all
  MoeCount *counts = nullptr;         // of all parts (an offset)
  int64_t up_workgroups = 0, down_workgroups = 0;  // of the products
  size_t workspace = 0, counters = 0; // bytes; the counters stand first
};

// ---- verification ----------------------------------------------------------------------------------------------------------

// What a workgroup found in a part of a row of logits: sum of 2^((l - top) * c) for c = log2(e) / temperature, the largest and the first place where it
// stands.  A sum that is not finite: there is a NaN or +infinity.
struct VerifyStat {
  double sum;
  float top;
  int32_t at;
};
struct VerifyDev {
  const int32_t *first_row, *drafted;
  const char *logits, *draft_logits;
  const float *temperatures, *accept_random, *sample_random;
  int32_t *tokens, *accepted;
  int64_t logits_stride, draft_stride;  // bytes
  int32_t dtype, sequences, rows, vocab;
  float temperature;
  int32_t pieces, chunks;  // a chunk is 512 * pieces logits
  VerifyStat *stats;       // [rows][2][chunks]
  double *sums;            // [sequences][chunks]
  uint32_t *arrived;       // [sequences], COUNTER_STEP apart
};
constexpr int VERIFY_PIECES = 4;  // of 512 logits that a chunk has at most
constexpr int32_t VERIFY_CHUNKS = 4;  // that a workgroup of the second launch takes
constexpr int VERIFY_PROBLEMS = 16;  // of a launch
struct VerifyTable {
  uint32_t stat_first[VERIFY_PROBLEMS], sum_first[VERIFY_PROBLEMS];  // workgroup of the two launches; none: the largest number
  VerifyDev problems[VERIFY_PROBLEMS];
};
struct VerifyLaunch {
  int32_t n;
  int64_t stat_grid, sum_grid;
  VerifyTable table;  // workspace pointers: offsets until the plan is on the device
};
struct VerifyPlanHost {
  std::vector<VerifyLaunch> launches;
  size_t workspace = 0, counters = 0;
};

// Checks and plans, for a device of that many compute units or for that many workgroups at a time (0: what its compute units hold); no HIP call.  SK_OK or an error with `err` set.
sk_status plan_norm(const sk_norm_problem *problems, int32_t n, NormPlanHost &out, std::string &err);
sk_status plan_moe(const sk_moe_problem *problems, int32_t n, int32_t compute_units, int32_t workgroups, MoePlanHost &out, std::string &err);
sk_status plan_verify(const sk_verify_problem *problems, int32_t n, VerifyPlanHost &out, std::string &err);

}  // namespace sk
