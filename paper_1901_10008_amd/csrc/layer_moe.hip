// A mixture-of-experts layer: the kernels and their entry points.
#include "layer_host.h"
#include "layer_math.hip.h"
#include "layer_units.h"

namespace sk {

struct MoeArgs {
  const MoeDev *parts;
  const uint32_t *first, *add_first;  // of the router, and of the sums: first workgroup of each part
  MoeCount *counts;                   // of each part: what the router found
  int32_t n;
};

__device__ __forceinline__ int32_t rows_of(const SK_CONSTANT MoeDev &P) {
  const int32_t n = P.n_rows ? load_i32(P.n_rows) : 0x7fffffff;
  return __builtin_amdgcn_readfirstlane(min(max(max(n, 0) - P.row0, 0), P.rows));  // (the number is cut first: what is left of -2^31 less row0 would be positive)
}

// What a workgroup needs to find its part.
struct Place {
  const SK_CONSTANT MoeDev *part;
  int32_t unit;
};
__device__ __forceinline__ Place place_of(const MoeArgs &a, const uint32_t *firsts) {
  int32_t part = 0;
  uint32_t first = 0;
  if (a.n > 1) {
    part = __builtin_amdgcn_readfirstlane(last_not_above(firsts, a.n, (int64_t)blockIdx.x, threadIdx.x & 63));
    first = ((const SK_CONSTANT uint32_t *)(uintptr_t)firsts)[part];
  }
  return Place{(const SK_CONSTANT MoeDev *)(uintptr_t)(a.parts + part), (int32_t)(blockIdx.x - first)};
}

// ---------------------------------------------------------------------------
// the router
// ---------------------------------------------------------------------------
// Scores of two experts a wave and ROUTE_ROWS rows; where there are few of them, of two experts a workgroup, a quarter of the reduction's pieces a wave.  Products of numbers of at most 24 and 11 bits are exact in 64 bits, and so, but for 2^-50 or
// so, are their sums: which of two experts is chosen does not depend on the order of a sum.  Vector instructions of 64 bits have the rate of
// those of 32 here, and E * D multiplications a row are little beside the experts' products.
template <int DT, bool F32>
__device__ __forceinline__ void route_scores(const SK_CONSTANT MoeDev &P, int32_t block, int32_t e0, double (*joint)[2 * ROUTE_ROWS], int wave, int lane) {
  double sum[2][ROUTE_ROWS] = {};
  const int32_t last = P.experts - 1;
  const bool split = P.route_experts == 2;
  if (!split) e0 += 2 * wave;
  const char *w[2] = {P.router + (int64_t)min(e0, last) * P.router_stride, P.router + (int64_t)min(e0 + 1, last) * P.router_stride};
  const char *x[ROUTE_ROWS];
#pragma unroll
  for (int r = 0; r < ROUTE_ROWS; ++r) x[r] = P.x + (int64_t)min(block * ROUTE_ROWS + r, P.rows - 1) * P.x_stride;  // (that there is a row is known later)
#pragma unroll 2
  for (int32_t k = (split ? wave * 64 + lane : lane) * 8; k < P.dim; k += split ? 8 * CACHE_THREADS : 512) {
    float a[2][8], b[ROUTE_ROWS][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) load8<F32 ? SK_F32 : DT, false>(w[i] + (int64_t)k * (F32 ? 4 : 2), a[i]);
#pragma unroll
    for (int r = 0; r < ROUTE_ROWS; ++r) load8<DT, false>(x[r] + (int64_t)k * 2, b[r]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double a0 = (double)a[0][j], a1 = (double)a[1][j];
#pragma unroll
      for (int r = 0; r < ROUTE_ROWS; ++r) {
        const double v = (double)b[r][j];
        sum[0][r] = fma(a0, v, sum[0][r]);
        sum[1][r] = fma(a1, v, sum[1][r]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < ROUTE_ROWS; ++r) {
      const double s = wave_sum(sum[i][r]);
      if (lane == 0) joint[wave][i * ROUTE_ROWS + r] = s;
    }
  __syncthreads();
  if ((wave == 0 || !split) && lane < 2 * ROUTE_ROWS) {
    const int32_t e = e0 + lane / ROUTE_ROWS, row = block * ROUTE_ROWS + lane % ROUTE_ROWS;
    double s = joint[wave][lane];
    if (split) {
#pragma unroll
      for (int w = 1; w < CACHE_THREADS / 64; ++w) s += joint[w][lane];
    }
    if (e < P.experts && row < P.rows) put(P.logits + (int64_t)row * P.experts + e, s);
  }
}

// Numbers of 64 bits as whole numbers of the same order; NaN below all others, and 0 for what is out.
__device__ __forceinline__ uint64_t ordered(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);  // (-0 becomes 0)
  return v != v ? 1u : (b >> 63 ? ~b : b | (uint64_t)1 << 63);
}
// The largest of a wave's numbers, the same in all lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t larger(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int32_t)v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = larger<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v = larger<0x112, 0xf>(v);
  v = larger<0x114, 0xf>(v);
  v = larger<0x118, 0xf>(v);
  v = larger<0x142, 0xa>(v);  // row_bcast:15, 31
  v = larger<0x143, 0xc>(v);
  return (uint32_t)lane_of((int32_t)v, 63);
}

// The top_k experts of a row, by one wave: the largest score is taken out top_k times (upper halves first, lower halves among those that are
// equal in them).  N * 64 experts at most.
template <int N>
__device__ __forceinline__ void choose(const SK_CONSTANT MoeDev &P, int32_t row, int lane, int32_t *ids, float *weights) {
  double score[N];
  uint32_t hi[N], lo[N];
  auto set = [&](int i, uint64_t key) { hi[i] = (uint32_t)(key >> 32), lo[i] = (uint32_t)key; };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int32_t e = i * 64 + lane;
    score[i] = e < P.experts ? got(P.logits + (int64_t)row * P.experts + e) : -__builtin_inf();
  }
#pragma unroll
  for (int i = 0; i < N; ++i) set(i, i * 64 + lane < P.experts ? ordered(score[i]) : 0u);
  if (P.scoring == SK_MOE_SOFTMAX) {
    double top = -__builtin_inf(), sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmax(top, score[i]);
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      score[i] = exp(score[i] - top);
      sum += i * 64 + lane < P.experts ? score[i] : 0.0;
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < N; ++i) score[i] /= sum;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) score[i] = 1.0 / (1.0 + exp(-score[i]));
  }
  if (P.bias || P.scoring != SK_MOE_SOFTMAX) {  // (a softmax keeps the order of its logits, which tell apart what it rounds to the same)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t e = i * 64 + lane;
      if (e < P.experts) set(i, ordered(score[i] + (P.bias ? (double)load_f(P.bias + e) : 0.0)));
    }
  }
  int32_t mine = 0;  // lane j: the j-th choice
  double mine_score = 0.0, sum = 0.0;
  for (int32_t j = 0; j < P.top_k; ++j) {
    uint32_t best = 0, second = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) best = max(best, hi[i]);
    best = wave_max(best);
#pragma unroll
    for (int i = 0; i < N; ++i) second = hi[i] == best ? max(second, lo[i]) : second;
    second = wave_max(second);
    bool found = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t hit = __ballot(hi[i] == best && lo[i] == second);
      if (found || !hit) continue;
      found = true;
      const int l = (int)__builtin_ctzll(hit);
      const uint64_t b = __builtin_bit_cast(uint64_t, score[i]);
      const double s = __builtin_bit_cast(double, (uint64_t)(uint32_t)lane_of((int32_t)(b >> 32), l) << 32 | (uint32_t)lane_of((int32_t)b, l));
      sum += s;
      if (lane == j) mine = i * 64 + l, mine_score = s;
      if (lane == l) hi[i] = lo[i] = 0;
    }
  }
  if (lane < P.top_k) {
    const int64_t at = (int64_t)row * P.top_k + lane;
    const float weight = (float)((P.normalize ? mine_score / sum : mine_score) * (double)P.scale);
    if (ids) ids[lane] = mine, weights[lane] = weight;
    else put(P.ids + at, mine), put(P.weights + at, weight);
    if (P.user_ids) P.user_ids[at] = mine;
    if (P.user_weights) P.user_weights[at] = weight;
  }
}

// Which rows go to which expert: every chosen pair gets a place, those of one expert side by side in the order of their rows; and the list of
// groups of up to MOE_GROUP places of an expert.  A bit for every row and expert stands in LDS, so that nothing depends on the order
// of the atomics that set them.
constexpr int SORT_PAIRS = 2048;  // that LDS keeps
struct Sorting {
  uint32_t bits[MOE_EXPERTS][MOE_ROWS / 32];
  int32_t count[MOE_EXPERTS], first[MOE_EXPERTS];
  int32_t ids[SORT_PAIRS];
  float weights[ROUTE_ROWS * MOE_TOP];
};
// Counts of an expert's groups, and sums of them, in one number of 64 bits: rows in the lowest 16 bits, then groups of modes 8, 16 and 32, 16 bits each.  (A
// part has at most 512 experts and 2^14 pairs, so none reaches 2^15.)
__device__ __forceinline__ int64_t groups_of(int32_t n) {
  const int32_t g = (n + MOE_GROUP - 1) / MOE_GROUP, last = moe::mode_of(n - (g - 1) * MOE_GROUP);
  return n ? (int64_t)n + ((int64_t)(g - 1) << 48) + ((int64_t)1 << (last == 8 ? 16 : last == 16 ? 32 : 48)) : 0;
}
__device__ __forceinline__ int32_t rows_in(int64_t counts) { return (int32_t)(counts & 0xffff); }
__device__ __forceinline__ int32_t of_mode(int64_t counts, int mode) { return (int32_t)(counts >> (mode == 8 ? 16 : mode == 16 ? 32 : 48)) & 0xffff; }
__device__ __forceinline__ int32_t groups_in(int64_t counts) { return of_mode(counts, 8) + of_mode(counts, 16) + of_mode(counts, 32); }
// (costs of modes 8, 16 and 32)
struct Costs {
  int64_t of[3];
  __device__ __forceinline__ int64_t sum(int64_t counts) const { return of_mode(counts, 8) * of[0] + of_mode(counts, 16) * of[1] + of_mode(counts, 32) * of[2]; }
};
// (of all tiles of a group)
__device__ __forceinline__ Costs costs_of(int32_t k_len, int32_t matrices, int32_t parts, int32_t rows) {
  return Costs{{moe::cost(k_len, matrices, parts, 8) * moe::tiles_of(rows, matrices, 8), moe::cost(k_len, matrices, parts, 16) * moe::tiles_of(rows, matrices, 16),
                moe::cost(k_len, matrices, parts, 32) * moe::tiles_of(rows, matrices, 32)}};
}

// here: ids and weights are in LDS already.
__device__ __forceinline__ void sort_pairs(const SK_CONSTANT MoeDev &P, int32_t rows, Sorting &s, bool here, int tid) {
  const int32_t pairs = rows * P.top_k, words = (rows + 31) / 32;
  for (int32_t i = tid; i < P.experts * (MOE_ROWS / 32); i += CACHE_THREADS)
    if (i % (MOE_ROWS / 32) < words) s.bits[i / (MOE_ROWS / 32)][i % (MOE_ROWS / 32)] = 0;
  __syncthreads();
  for (int32_t i = tid; i < pairs; i += CACHE_THREADS) {
    const int32_t row = i / P.top_k, e = here ? s.ids[i] : got(P.ids + i);
    if (!here && i < SORT_PAIRS) s.ids[i] = e;
    atomicOr(&s.bits[e][row / 32], 1u << (row % 32));
  }
  __syncthreads();
  for (int32_t e = tid; e < P.experts; e += CACHE_THREADS) {
    int32_t n = 0;
    for (int32_t w = 0; w < words; ++w) n += __popc(s.bits[e][w]);
    s.count[e] = n;
  }
  __syncthreads();
  if (tid < 64) {
    const int32_t matrices = P.gate ? 2 : 1;
    const Costs up = costs_of(P.dim, matrices, 1, P.ffn), down = costs_of(P.ffn, 1, H_PARTS, P.dim);
    int64_t all = 0;
    for (int32_t e0 = 0; e0 < P.experts; e0 += 64) {
      const int32_t e = e0 + tid, n = e < P.experts ? s.count[e] : 0, g = (n + MOE_GROUP - 1) / MOE_GROUP;
      const int64_t mine = groups_of(n), upto = wave_scan(mine), before = all + upto - mine;
      const int32_t place = rows_in(before), at = groups_in(before);
      if (e < P.experts) s.first[e] = place;
      for (int32_t i = 0; i < g; ++i) {  // (all but the last are full)
        P.groups[at + i] = MoeGroup{e, place + i * MOE_GROUP, min(MOE_GROUP, n - i * MOE_GROUP), 0};
        P.first_begin[at + i] = up.sum(before) + i * up.of[2];
        P.second_begin[at + i] = down.sum(before) + i * down.of[2];
      }
      all += lane_of(upto, 63);
    }
    MoeCount c{groups_in(all), rows, up.sum(all), down.sum(all)};
    if (P.shared_ffn) {  // (at most 16 groups)
      const int32_t g = (rows + MOE_GROUP - 1) / MOE_GROUP, n = min(MOE_GROUP, rows - tid * MOE_GROUP);
      const Costs shared_up = costs_of(P.dim, matrices, 1, P.shared_ffn), shared_down = costs_of(P.shared_ffn, 1, H_PARTS, P.dim);
      if (tid < g) {
        P.groups[c.groups + tid] = MoeGroup{-1, tid * MOE_GROUP, n, 0};
        P.first_begin[c.groups + tid] = c.first_work + tid * shared_up.of[2];
        P.second_begin[c.groups + tid] = c.second_work + tid * shared_down.of[2];
      }
      const int64_t counts = groups_of(rows);
      c.groups += g;
      c.first_work += shared_up.sum(counts);
      c.second_work += shared_down.sum(counts);
    }
    if (tid == 0) *P.count = c;
  }
  __syncthreads();
  for (int32_t i = tid; i < pairs; i += CACHE_THREADS) {
    const int32_t row = i / P.top_k, e = i < SORT_PAIRS ? s.ids[i] : got(P.ids + i);
    int32_t at = s.first[e] + __popc(s.bits[e][row / 32] & ((1u << (row % 32)) - 1));
    for (int32_t w = 0; w < row / 32; ++w) at += __popc(s.bits[e][w]);
    P.row_of[at] = row, P.place_at[i] = at;
    if (here) P.weights[i] = s.weights[i];
  }
}

__global__ void __launch_bounds__(CACHE_THREADS) sk_moe_route(MoeArgs a) {
  __shared__ Sorting sorting;
  __shared__ double joint[CACHE_THREADS / 64][2 * ROUTE_ROWS];
  __shared__ uint32_t flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place place = place_of(a, a.first);
  const SK_CONSTANT MoeDev &P = *place.part;
  const int32_t unit = place.unit;
  const int32_t by_experts = (P.experts + P.route_experts - 1) / P.route_experts, blocks = (P.rows + ROUTE_ROWS - 1) / ROUTE_ROWS;
  const int32_t block = unit / by_experts, e0 = unit % by_experts * P.route_experts, rows = rows_of(P);
  if (P.dtype == SK_BF16) P.router_f32 ? route_scores<SK_BF16, true>(P, block, e0, joint, wave, lane) : route_scores<SK_BF16, false>(P, block, e0, joint, wave, lane);
  else P.router_f32 ? route_scores<SK_F16, true>(P, block, e0, joint, wave, lane) : route_scores<SK_F16, false>(P, block, e0, joint, wave, lane);
  if (!last_to_arrive(P.routed + block * COUNTER_STEP, by_experts, &flag)) return;
  const int32_t row = block * ROUTE_ROWS + wave;
  int32_t *ids = blocks == 1 ? sorting.ids + row * P.top_k : nullptr;  // (then there are at most ROUTE_ROWS rows, and no other workgroup has any)
  float *weights = sorting.weights + row * P.top_k;
  if (row < rows) {
    if (P.experts <= 64) choose<1>(P, row, lane, ids, weights);
    else if (P.experts <= 128) choose<2>(P, row, lane, ids, weights);
    else choose<MOE_EXPERTS / 64>(P, row, lane, ids, weights);
  }
  if (blocks > 1 && !last_to_arrive(P.blocks_routed, blocks, &flag)) return;
  sort_pairs(P, rows, sorting, blocks == 1, tid);
}

// ---------------------------------------------------------------------------
// the experts' products
// ---------------------------------------------------------------------------
// A tile is 16 or 32 rows of an expert's weights times the rows of activations of a group; the four waves of a workgroup take the blocks of 64 elements
// (128 bytes a row) of its reduction in turn, and add their sums up in LDS.  Bound by the memory that the weights come from (two rows of eight experts of
// 4096 x 12288 with gates: 1.06 GB in 200 us, 5.3 TB/s; the first products of 61 rows 5.9 TB/s), with more rows an expert by the activations, which come
// out of the dies' caches for every tile (23 rows: 115 MB of weights in 41 and in 59 us).  An instruction loads
// eight whole lines of 128 bytes, lane (r, q) of the 16 x 4 that the matrix instruction sees row r % 8 (+ 8), bytes 16 (q + 4 (r / 8)).
//   Up to 8 rows of activations (MODE 8): the matrix instruction takes the weights as they came, rows 0 .. 7 with the lower half of the block and once
//     more with the upper; its other operand is laid out the same way, by one load.  Of the 16 x 16 sums the 8 x 8 on the diagonal count.
//   Up to 16 or 32: half of the lanes' pieces change places within their row of 16 lanes, and the operands are 16 rows with the lower, and with the upper
//     half of the block.
__device__ __forceinline__ u32x4 low_half(const u32x4 &first, const u32x4 &second) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_update_dpp((int)first[i], (int)second[i], 0x128, 0xF, 0xC, false);
  return r;
}
__device__ __forceinline__ u32x4 high_half(const u32x4 &first, const u32x4 &second) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_update_dpp((int)second[i], (int)first[i], 0x128, 0xF, 0x3, false);
  return r;
}

constexpr int TILE = 16;
constexpr int RUN_PLACES = 512;  // rows of groups that LDS knows
// A workgroup walks through a run of tiles: groups of one mode one after the other, all tiles of each side by side.
struct Run {
  int32_t group, tile, n;  // the first tile; how many
};
// What the waves of a workgroup hand each other: [turn][wave][matrix][row of activations (twice with MODE 8)][row of weights].
template <int W>
__device__ __forceinline__ f32x4 *joint_at(float *joint, int t, int wave, int m, int32_t i, int32_t row) {
  return (f32x4 *)(joint + ((((t & 1) * 4 + wave) * W + m) * MOE_GROUP + i) * TILE + row);
}
constexpr int joint_floats(int w) { return 2 * 4 * w * MOE_GROUP * TILE; }
// Loads by way of a buffer descriptor: a scalar base, and in each lane an offset below 2^31; a lane with OUTSIDE gets zeros and asks for nothing, so
// that no load stands under a branch (which would leave the compiler in doubt how many are on their way).
constexpr uint32_t OUTSIDE = 0x80000000u;
// ONCE: past the caches, where activations and the small launches around these are (two tenants 52.6 + 33.6 -> 48 + 30.9 us, the router with them 11.4 ->
// 9.3).  Not the weights of groups of more than 16 rows, which the next group of their expert is likely to read again (a chunk of 250 rows 42 + 56 -> 46 + 59).
template <bool ONCE>
__device__ __forceinline__ u32x4 load_from(const char *base, uint32_t lane_offset, int32_t offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)OUTSIDE, 0x00027000);
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)lane_offset, offset, ONCE ? 2 : 0));
}

// (an address that is the same in all lanes, where the compiler cannot see it)
__device__ __forceinline__ const char *uniform(const char *p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  return (const char *)(uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(a >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)a));
}

// Eight elements of 32 bits a lane, multiplied by weights of 16 and summed in 32 bits; nothing is rounded on the way.  `even` and `odd`: the first and the
// last four of them.
template <int DT>
struct Wide;
// bf16: 24 bits are three times eight, so they are the sum of three numbers: the upper half of what they are, of what that leaves, and what is left then.
// (With eight instructions of 32 bits instead, as below: two tenants 97 us instead of 94, a chunk of 250 rows 124 instead of 119.)
template <>
struct Wide<SK_BF16> {
  u32x4 part[3];
  __device__ __forceinline__ Wide(const u32x4 &even, const u32x4 &odd) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      uint32_t lo = j < 4 ? even[j % 4] : odd[j % 4], hi = j < 4 ? even[j % 4 + 1] : odd[j % 4 + 1];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        part[p][j / 2] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
        lo = left_of(lo, p), hi = left_of(hi, p);
      }
    }
  }
  static __device__ __forceinline__ uint32_t left_of(uint32_t bits, int p) {
    const float x = __builtin_bit_cast(float, bits) - __builtin_bit_cast(float, bits & 0xffff0000u);
    return __builtin_bit_cast(uint32_t, p > 0 || x == x ? x : 0.f);  // (an infinity leaves nothing)
  }
  __device__ __forceinline__ void times(const u32x4 &w, f32x4 &sums) const {
#pragma unroll
    for (int p = 2; p >= 0; --p) mma16<SK_BF16>(w, part[p], sums);
  }
};
// f16 has not their range: the weights become 32 bits wide.  What a lane has at place j of its eights goes into the j-th of eight matrix instructions, whose
// four places of the reduction are the lanes' q.
template <>
struct Wide<SK_F16> {
  float x[8];
  __device__ __forceinline__ Wide(const u32x4 &even, const u32x4 &odd) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = j < 4 ? even[j % 4] : odd[j % 4];
      x[j] = __builtin_bit_cast(float, bits);
    }
  }
  __device__ __forceinline__ void times(const u32x4 &w, f32x4 &sums) const {
    float wide[8];
    unpack8<SK_F16>(w, wide);
#pragma unroll
    for (int j = 0; j < 8; ++j) sums = __builtin_amdgcn_mfma_f32_16x16x4f32(wide[j], x[j], sums, 0, 0, 0);
  }
};

// W matrices of weights with the same rows and the same activations (gate and up), of each S times 16 rows; activations of
// DT (L = 1), or of 32 bits in L = 2 planes, x_part bytes apart, of the even and of the odd fours of their elements.  The stream of loads runs R blocks ahead of the matrix instructions, from
// tile to tile, so it is only empty at the beginning and the end of a run.  group(i) is the i-th group, base(g, m) its matrix m, x_base(g) and x_offset(g, i)
// where its i-th row of activations stands; done(t, group, tile) takes up the sums of turn t.
template <int DT, int MODE, int W, int S, int L, int R, class G, class B, class XB, class XO, class D>
__device__ __forceinline__ void stream(const Run &run, int32_t tiles, int64_t row_stride, int32_t rows_end, int32_t k_len, int32_t x_part, G group, B base, XB x_base, XO x_offset, D done, float *joint,
                                       int wave, int lane) {
  constexpr int NB = MODE == 32 ? 2 : 1, H = MODE == 8 ? 1 : 2, A = MODE == 8 ? 2 : NB;  // loads of activations for 16 rows, sums
  const int r16 = lane & 15, q = lane >> 4;
  const int32_t steps = (k_len + 255) / 256;  // of the four waves' blocks each
  const uint32_t w_piece = 16 * (q + 4 * (r16 >> 3)), x_piece = MODE == 8 ? w_piece : 16 * q;
  constexpr int WS = W * S;  // (matrix m, rows s at m * S + s)
  u32x4 w[R][WS][2], b[R][L][NB][H];
  f32x4 acc[WS][A] = {};

  // loads
  int32_t p_left = run.n, p_group = run.group, p_tile = run.tile, p_step = 0;
  MoeGroup pg = group(p_group);
  const char *w_base[WS], *x_at;
  uint32_t w_row[S][2], x_row[NB];
  auto new_rows = [&]() {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int32_t row = min((p_tile * S + s) * TILE, rows_end - 1);  // (rows behind the last repeat it and are not used)
#pragma unroll
      for (int m = 0; m < W; ++m) w_base[m * S + s] = uniform(base(pg, m) + (int64_t)row * row_stride);
#pragma unroll
      for (int j = 0; j < 2; ++j) w_row[s][j] = (uint32_t)min(8 * j + (r16 & 7), rows_end - 1 - row) * (uint32_t)row_stride + w_piece;
    }
  };
  auto new_group = [&]() {
    x_at = uniform(x_base(pg));
#pragma unroll
    for (int n = 0; n < NB; ++n) x_row[n] = x_offset(pg, min(MODE == 8 ? r16 & 7 : n * 16 + r16, pg.rows - 1)) + x_piece;  // (columns behind the last repeat it and are not used)
  };
  new_group();
  new_rows();
  auto load = [&](u32x4(&w)[WS][2], u32x4(&b)[L][NB][H]) {
    // zeros behind the end of the reduction and behind the last tile
    const int32_t k = (wave + 4 * p_step) * 128, left = p_left > 0 ? 2 * k_len - k : 0;
    const bool in = (int32_t)w_piece < left;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const uint32_t at = in ? w_row[s][j] : OUTSIDE;
#pragma unroll
        for (int m = 0; m < W; ++m) w[m * S + s][j] = load_from<MODE < 32>(w_base[m * S + s], at, k);
      }
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const bool in_x = (int32_t)x_piece + 64 * h < left;
#pragma unroll
      for (int l = 0; l < L; ++l)
#pragma unroll
        for (int n = 0; n < NB; ++n) b[l][n][h] = load_from<false>(x_at, in_x ? x_row[n] + 64 * h : OUTSIDE, k + l * x_part);
    }
    if (++p_step == steps) {
      p_step = 0;
      if (--p_left > 0) {
        if (++p_tile >= tiles) {
          p_tile = 0;
          pg = group(++p_group);
          new_group();
        }
        new_rows();
      }
    }
  };
#pragma unroll
  for (int u = 0; u < R; ++u) load(w[u], b[u]);

  int32_t c_step = 0, c_group = run.group, c_tile = run.tile, t = 0;
  while (t < run.n) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      u32x4 lo[WS], hi[WS];
#pragma unroll
      for (int m = 0; m < WS; ++m) {
        lo[m] = MODE == 8 ? w[u][m][0] : low_half(w[u][m][0], w[u][m][1]);
        hi[m] = MODE == 8 ? w[u][m][1] : high_half(w[u][m][0], w[u][m][1]);
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int h = 0; h < H; ++h) {
          auto products = [&](auto product) {
#pragma unroll
            for (int m = 0; m < WS; ++m) {
              if constexpr (MODE == 8) product(lo[m], acc[m][0]), product(hi[m], acc[m][1]);
              else product(h ? hi[m] : lo[m], acc[m][n]);
            }
          };
          if constexpr (L == 1) {
            products([&](const u32x4 &w, f32x4 &sums) { mma16<DT>(w, b[u][0][n][h], sums); });
          } else {
            const Wide<DT> x(b[u][0][n][h], b[u][1][n][h]);
            products([&](const u32x4 &w, f32x4 &sums) { x.times(w, sums); });
          }
        }
      load(w[u], b[u]);
      if (++c_step == steps) {
        c_step = 0;
        if (t < run.n) {  // (the steps behind the last tile multiply zeros)
          // lane (r, q) has, for row r of activations, rows 4q .. 4q + 3 of weights
#pragma unroll
          for (int m = 0; m < WS; ++m)
#pragma unroll
            for (int n = 0; n < A; ++n) {
              if constexpr (MODE == 8) {
                if ((q >> 1) == (r16 >> 3)) *joint_at<WS>(joint, t, wave, m, r16, 8 * n + 4 * (q & 1)) = acc[m][n];
              } else {
                *joint_at<WS>(joint, t, wave, m, n * 16 + r16, 4 * q) = acc[m][n];
              }
              acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
          // (only LDS has to be there: the loads ahead stay on their way; the other turn's sums have been read by all that come here)
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          done(t, c_group, c_tile);
          ++t;
          if (++c_tile >= tiles) {
            c_tile = 0;
            ++c_group;
          }
        }
      }
    }
  }
  __syncthreads();
}
// Four rows of weights times row i of activations.
template <int MODE, int W>
__device__ __forceinline__ f32x4 joined(float *joint, int t, int m, int32_t i, int quad) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int wave = 0; wave < 4; ++wave) {
    v += *joint_at<W>(joint, t, wave, m, i, 4 * quad);
    if constexpr (MODE == 8) v += *joint_at<W>(joint, t, wave, m, i + 8, 4 * quad);
  }
  return v;
}

// (What the router wrote is read through the scalar cache: it was another launch.)
__device__ __forceinline__ MoeGroup group_of(const SK_CONSTANT MoeDev &P, int32_t i) {
  const SK_CONSTANT MoeGroup &g = ((const SK_CONSTANT MoeGroup *)(uintptr_t)P.groups)[i];
  return MoeGroup{g.expert, g.first, g.rows, 0};
}
__device__ __forceinline__ const SK_CONSTANT MoeCount &count_of(const MoeArgs &a, int32_t part) { return ((const SK_CONSTANT MoeCount *)(uintptr_t)a.counts)[part]; }
__device__ __forceinline__ const SK_CONSTANT MoeDev &part_of(const MoeArgs &a, int32_t part) { return *(const SK_CONSTANT MoeDev *)(uintptr_t)(a.parts + part); }
// The last group of n that begins at or before a place.
__device__ __forceinline__ int32_t group_at(const int64_t *begin, int32_t n, int64_t at, int lane) { return __builtin_amdgcn_readfirstlane(last_not_above(begin, n, at, lane)); }
__device__ __forceinline__ int64_t begin_of(const int64_t *begin, int32_t i) { return ((const SK_CONSTANT int64_t *)(uintptr_t)begin)[i]; }

// Work is cut into equal shares, one for each workgroup of a launch that fills the card once.

// The run that begins with a group: those behind it of the same kind (shared or not) and mode, up to group `end`; of the first products as many as LDS has
// places for, which their rows go to.
template <bool ROWS>
__device__ __forceinline__ int32_t run_end(const SK_CONSTANT MoeDev &P, int32_t begin, int32_t end, int32_t *row_of, int tid) {
  const MoeGroup g = group_of(P, begin);
  int32_t at = begin + 1, places = g.rows;
  while (at < end) {
    const MoeGroup next = group_of(P, at);
    if ((next.expert < 0) != (g.expert < 0) || moe::mode_of(next.rows) != moe::mode_of(g.rows) || (ROWS && places + next.rows > RUN_PLACES)) break;
    places += next.rows;
    ++at;
  }
  if constexpr (ROWS) {
    for (int32_t i = tid; i < places; i += CACHE_THREADS) row_of[i] = g.expert < 0 ? g.first + i : load_i32(P.row_of + g.first + i);
    __syncthreads();
  }
  return at;
}

template <int DT, int MODE, bool GATED>
__device__ __forceinline__ void up_run(const SK_CONSTANT MoeDev &P, const Run &run, bool shared, float *joint, const int32_t *row_of, int tid) {
  constexpr int W = GATED ? 2 : 1, S = moe::rows_of_tile(W, MODE) / TILE;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t width = shared ? P.shared_ffn : P.ffn, place0 = group_of(P, run.group).first;
  auto base = [&](const MoeGroup &g, int m) {
    if (shared) return m ? P.shared_gate : P.shared_up;
    return (m ? P.gate : P.up) + g.expert * P.up_expert;
  };
  auto done = [&](int32_t t, int32_t group, int32_t tile) {
    const MoeGroup g = group_of(P, group);
    const int32_t i = (tid >> 2) % MOE_GROUP, s = tid / (4 * MOE_GROUP), f = (tile * S + s) * TILE + 4 * (tid & 3);
    if (i >= g.rows || s >= S || f >= width) return;  // (width is a multiple of 8)
    f32x4 h = joined<MODE, W * S>(joint, t, s, i, tid & 3);
    if constexpr (GATED) {
      const f32x4 z = joined<MODE, W * S>(joint, t, S + s, i, tid & 3);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] *= activated(P.act, z[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = activated(P.act, h[k]);
    }
    const int64_t place = (shared ? (int64_t)P.rows * P.top_k : 0) + g.first + i;
    // As it is, in 32 bits: rounded to bf16 it would be most of the output's error (0.0023 of it instead of 0.0017), and f16 has not its range.  Two planes, of the
    // even and of the odd fours of a row, so that a lane's eight elements are loaded from where they would be in 16 bits.
    store16(P.h + place * P.h_stride + (f >> 2 & 1) * P.h_part + 2 * (f & ~7), __builtin_bit_cast(u32x4, h));
  };
  stream<DT, MODE, W, S, 1, MODE == 8 ? 3 : 2>(
      run, moe::tiles_of(width, W, MODE), shared ? 2 * (int64_t)P.dim : P.up_row, width, P.dim, 0, [&](int32_t i) { return group_of(P, i); }, base, [&](const MoeGroup &) { return P.x; },
      [&](const MoeGroup &g, int32_t i) { return (uint32_t)row_of[g.first - place0 + i] * (uint32_t)P.x_stride; }, done, joint, wave, lane);
}

// The sums of a place of the second products stand in the workspace, unweighted and in 32 bits: sk_moe_add takes them from there.  (To walk over all groups
// of 16 columns, add their rows up in LDS and join the slices of the workgroups that share the columns saves those stores, 12 of 230 us where 61 rows have
// 4 of 60 experts each, but 250 rows of 1000 columns took 75 us instead of 45 and the second products of one row 9.7 instead of 5.2 + 2.7.)
template <int DT, int MODE>
__device__ __forceinline__ void down_run(const SK_CONSTANT MoeDev &P, const Run &run, bool shared, float *joint, int tid) {
  constexpr int S = moe::rows_of_tile(1, MODE) / TILE;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t place0 = shared ? (int64_t)P.rows * P.top_k : 0;
  const int32_t width = shared ? P.shared_ffn : P.ffn;
  auto done = [&](int32_t t, int32_t group, int32_t tile) {
    const MoeGroup g = group_of(P, group);
    const int32_t i = (tid >> 2) % MOE_GROUP, s = tid / (4 * MOE_GROUP), d = (tile * S + s) * TILE + 4 * (tid & 3);
    if (i >= g.rows || s >= S || d >= P.dim) return;  // (dim is a multiple of 8)
    *(f32x4 SK_GLOBAL *)(uintptr_t)(P.y + (place0 + g.first + i) * P.y_stride + d) = joined<MODE, S>(joint, t, s, i, tid & 3);
  };
  stream<DT, MODE, 1, S, H_PARTS, MODE == 8 ? 4 : MODE == 16 ? 2 : 1>(
      run, moe::tiles_of(P.dim, 1, MODE), shared ? 2 * (int64_t)width : P.down_row, P.dim, width, (int32_t)P.h_part, [&](int32_t i) { return group_of(P, i); },
      [&](const MoeGroup &g, int) { return shared ? P.shared_down : P.down + g.expert * P.down_expert; }, [&](const MoeGroup &g) { return P.h + (place0 + g.first) * P.h_stride; },
      [&](const MoeGroup &, int32_t i) { return (uint32_t)i * (uint32_t)P.h_stride; }, done, joint, wave, lane);
}

// A workgroup's share of the tiles of the first (UP) or second products.
template <bool UP>
struct Products {
  static __device__ __forceinline__ int64_t work(const SK_CONSTANT MoeCount &c) { return UP ? c.first_work : c.second_work; }
  static __device__ __forceinline__ int32_t tiles(const SK_CONSTANT MoeDev &P, const MoeGroup &g) {
    return moe::tiles_of(!UP ? P.dim : g.expert < 0 ? P.shared_ffn : P.ffn, UP && P.gate ? 2 : 1, moe::mode_of(g.rows));
  }
  static __device__ __forceinline__ int64_t cost(const SK_CONSTANT MoeDev &P, const MoeGroup &g) {
    return UP ? moe::cost(P.dim, P.gate ? 2 : 1, 1, moe::mode_of(g.rows)) : moe::cost(g.expert < 0 ? P.shared_ffn : P.ffn, 1, H_PARTS, moe::mode_of(g.rows));
  }

  // From tile `tile` of group `group` on, up to (not with) tile `last_tile` of group `last`.
  template <int DT, bool GATED>
  static __device__ __forceinline__ void between(const SK_CONSTANT MoeDev &P, int32_t group, int32_t tile, int32_t last, int32_t last_tile, float *joint, int32_t *row_of, int tid) {
    while (group < last || (group == last && tile < last_tile)) {
      const int32_t end = run_end<UP>(P, group, last_tile > 0 ? last + 1 : last, row_of, tid);
      const MoeGroup g = group_of(P, group);
      const bool shared = g.expert < 0;
      const int32_t each = tiles(P, g), mode = moe::mode_of(g.rows);
      const Run run{group, tile, (end - group) * each - tile - (end > last ? each - last_tile : 0)};
      if constexpr (UP) {
        if (mode == 8) up_run<DT, 8, GATED>(P, run, shared, joint, row_of, tid);
        else if (mode == 16) up_run<DT, 16, GATED>(P, run, shared, joint, row_of, tid);
        else up_run<DT, 32, GATED>(P, run, shared, joint, row_of, tid);
      } else {
        if (mode == 8) down_run<DT, 8>(P, run, shared, joint, tid);
        else if (mode == 16) down_run<DT, 16>(P, run, shared, joint, tid);
        else down_run<DT, 32>(P, run, shared, joint, tid);
      }
      group = end, tile = 0;
    }
  }

  static __device__ __forceinline__ void share(const MoeArgs &a, float *joint, int32_t *row_of, int tid) {
    const int lane = tid & 63;
    int64_t total = 0;
    for (int32_t i = 0; i < a.n; ++i) total += work(count_of(a, i));
    const moe::Share share = moe::share_of(total, gridDim.x, blockIdx.x);
    int64_t offset = 0;
    for (int32_t i = 0; i < a.n && offset < share.end; ++i) {
      const SK_CONSTANT MoeDev &P = part_of(a, i);
      const int64_t here = work(count_of(a, i));
      if (share.begin < offset + here && here > 0) {
        const int64_t *begins = UP ? P.first_begin : P.second_begin;
        const int32_t groups = count_of(a, i).groups;
        int32_t group[2], tile[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // beginning and end
          const int64_t at = e ? share.end - offset : max(share.begin - offset, (int64_t)0);
          group[e] = group_at(begins, groups, at, lane);
          const MoeGroup g = group_of(P, group[e]);
          tile[e] = __builtin_amdgcn_readfirstlane(moe::tile_from(at, begin_of(begins, group[e]), cost(P, g), tiles(P, g)));
          if (tile[e] == tiles(P, g)) ++group[e], tile[e] = 0;
        }
        auto run = [&](auto type) {
          constexpr int DT = decltype(type)::value;
          if (UP && P.gate) between<DT, UP>(P, group[0], tile[0], group[1], tile[1], joint, row_of, tid);
          else between<DT, false>(P, group[0], tile[0], group[1], tile[1], joint, row_of, tid);
        };
        if (P.dtype == SK_BF16) run(std::integral_constant<int, SK_BF16>{});
        else run(std::integral_constant<int, SK_F16>{});
      }
      offset += here;
    }
  }
};

__global__ void __launch_bounds__(CACHE_THREADS, MOE_UP_RESIDENT) sk_moe_up(MoeArgs a) {
  __shared__ __attribute__((aligned(16))) float joint[joint_floats(2)];
  __shared__ int32_t row_of[RUN_PLACES];
  Products<true>::share(a, joint, row_of, threadIdx.x);
}

__global__ void __launch_bounds__(CACHE_THREADS, MOE_DOWN_RESIDENT) sk_moe_down(MoeArgs a) {
  __shared__ __attribute__((aligned(16))) float joint[joint_floats(2)];
  Products<false>::share(a, joint, nullptr, threadIdx.x);
}

// out = the weighted sums of a row's places, in the order in which its experts were chosen, the shared expert last; 256 columns a wave.
template <int DT>
__device__ __forceinline__ void add_places(const SK_CONSTANT MoeDev &P, int32_t row, int32_t d) {
  constexpr int AHEAD = 8;
  const int64_t pair0 = (int64_t)row * P.top_k;
  const SK_CONSTANT int32_t *place = (const SK_CONSTANT int32_t *)(uintptr_t)(P.place_at + pair0);
  const SK_CONSTANT float *weight = (const SK_CONSTANT float *)(uintptr_t)(P.weights + pair0);
  auto y = [&](int64_t at) { return *(const f32x4 SK_GLOBAL *)(uintptr_t)(P.y + at * P.y_stride + d); };
  f32x4 sum = {0.f, 0.f, 0.f, 0.f}, shared = {0.f, 0.f, 0.f, 0.f};
  if (P.shared_ffn) shared = y((int64_t)P.rows * P.top_k + row);
  for (int32_t j0 = 0; j0 < P.top_k; j0 += AHEAD) {
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (j0 + u < P.top_k) v[u] = y(place[j0 + u]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (j0 + u < P.top_k) sum += weight[j0 + u] * v[u];
  }
  if (P.shared_ffn) sum += shared;
  store8(P.out + row * P.out_stride + 2 * d, u32x2{pack2<DT>(sum[0], sum[1]), pack2<DT>(sum[2], sum[3])});
}

__global__ void __launch_bounds__(CACHE_THREADS) sk_moe_add(MoeArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Place place = place_of(a, a.add_first);
  const SK_CONSTANT MoeDev &P = *place.part;
  const int32_t columns = (P.dim + ADD_COLUMNS - 1) / ADD_COLUMNS, unit = place.unit * 4 + wave, row = unit / columns, d = unit % columns * ADD_COLUMNS + 4 * lane;
  if (row >= ((const SK_CONSTANT MoeCount *)(uintptr_t)P.count)->rows || d >= P.dim) return;  // (dim is a multiple of 8)
  if (P.dtype == SK_BF16) add_places<SK_BF16>(P, row, d);
  else add_places<SK_F16>(P, row, d);
}

}  // namespace sk

struct sk_moe_plan : sk::PlanOnDevice {
  sk::MoePlanHost host;
  sk::MoeArgs args{};
};

namespace {

sk_status upload(sk_moe_plan &plan) {
  sk::MoePlanHost &h = plan.host;
  // counters, parts, first workgroups of the router
  const size_t o_parts = sk::align_up(h.counters, 256), o_first = o_parts + sk::align_up(h.parts.size() * sizeof(sk::MoeDev), 256),
               o_add = o_first + h.route_first.size() * 4;
  std::vector<char> image(o_add + h.add_first.size() * 4, 0);
  char *ws = nullptr;
  const sk_status st = sk::upload_image(plan, image, h.workspace, &ws);
  if (st != SK_OK) return st;
  auto moved = [](auto *&p, char *base) { p = (std::decay_t<decltype(p)>)(base + (uintptr_t)p); };
  std::vector<sk::MoeDev> parts = h.parts;
  for (sk::MoeDev &d : parts) {
    moved(d.routed, plan.blob), moved(d.blocks_routed, plan.blob);
    moved(d.logits, ws), moved(d.ids, ws), moved(d.weights, ws), moved(d.row_of, ws), moved(d.place_at, ws), moved(d.groups, ws), moved(d.first_begin, ws), moved(d.second_begin, ws), moved(d.count, ws), moved(d.h, ws), moved(d.y, ws);
  }
  if (!parts.empty()) std::memcpy(image.data() + o_parts, parts.data(), parts.size() * sizeof(sk::MoeDev));
  std::memcpy(image.data() + o_first, h.route_first.data(), h.route_first.size() * 4);
  sk::MoeCount *counts = h.counts;
  std::memcpy(image.data() + o_add, h.add_first.data(), h.add_first.size() * 4);
  moved(counts, ws);
  plan.args = sk::MoeArgs{(const sk::MoeDev *)(plan.blob + o_parts), (const uint32_t *)(plan.blob + o_first), (const uint32_t *)(plan.blob + o_add), counts, (int32_t)parts.size()};
  return sk::copy_image(plan, image);
}

}  // namespace

extern "C" {

sk_status sk_moe_plan_create(const sk_moe_problem *problems, int32_t n, const sk_layer_params *params, sk_moe_plan **out) {
  return sk::create_plan<sk_moe_plan>(params, out, [&](sk_moe_plan &plan, int32_t cus, int32_t workgroups, std::string &err) { return sk::plan_moe(problems, n, cus, workgroups, plan.host, err); }, upload);
}

sk_status sk_moe_plan_destroy(sk_moe_plan *plan) {
  if (!plan) return SK_OK;
  return sk::guarded([&]() -> sk_status { return sk::destroy_plan(plan, false); });
}

sk_status sk_moe_launch(sk_moe_plan *plan, void *hip_stream) {
  return sk::guarded([&]() -> sk_status {
    const hipStream_t stream = (hipStream_t)hip_stream;
    bool in_capture = false;
    sk_status st = sk::admit(plan, stream, &in_capture);
    if (st != SK_OK || plan->host.parts.empty()) return st;
    const hipEvent_t behind = in_capture ? nullptr : plan->last_use;
    const sk::MoePlanHost &h = plan->host;
    st = sk::launch(sk::sk_moe_route, (int64_t)h.route_first.back(), stream, nullptr, plan->args);
    if (st == SK_OK) st = sk::launch(sk::sk_moe_up, h.up_workgroups, stream, nullptr, plan->args);
    if (st == SK_OK) st = sk::launch(sk::sk_moe_down, h.down_workgroups, stream, nullptr, plan->args);
    if (st == SK_OK) st = sk::launch(sk::sk_moe_add, (int64_t)h.add_first.back(), stream, behind, plan->args);
    plan->ledger.after_launch((uintptr_t)stream, in_capture, behind && st == SK_OK);  // also after a failure: some launches may be out
    return st;
  });
}

sk_status sk_moe_plan_info(const sk_moe_plan *plan, int32_t *launches, int64_t *workspace_bytes) {
  return sk::guarded([&]() -> sk_status {
    if (!plan) return sk::set_last_error(SK_ERR_INVALID_ARG, "plan is null");
    if (launches) *launches = plan->host.parts.empty() ? 0 : 4;
    if (workspace_bytes) *workspace_bytes = (int64_t)(plan->host.workspace + plan->host.counters);
    return SK_OK;
  });
}

}  // extern "C"
