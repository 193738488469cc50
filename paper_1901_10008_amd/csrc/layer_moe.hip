// A mixture-of-experts layer: the kernels and their entry points.
#include "layer_host.h"
#include "layer_math.hip.h"

namespace sk {

struct MoeArgs {
  const MoeDev *parts;
  const uint32_t *first;  // first workgroup of each part
  int32_t n;
};

__device__ __forceinline__ int32_t rows_of(const SK_CONSTANT MoeDev &P) {
  const int32_t n = P.n_rows ? load_i32(P.n_rows) : 0x7fffffff;
  return __builtin_amdgcn_readfirstlane(min(max(n - P.row0, 0), P.rows));
}

// ---------------------------------------------------------------------------
// the router
// ---------------------------------------------------------------------------
// Scores of two experts a wave and ROUTE_ROWS rows.  Products of numbers of at most 24 and 11 bits are exact in 64 bits, and so, but for 2^-50 or
// so, are their sums: which of two experts is chosen does not depend on the order of a sum.  Vector instructions of 64 bits have the rate of
// those of 32 here, and E * D multiplications a row are little beside the experts' products.
template <int DT, bool F32>
__device__ __forceinline__ void route_scores(const SK_CONSTANT MoeDev &P, int32_t rows, int32_t block, int32_t e0, int lane) {
  double sum[2][ROUTE_ROWS] = {};
  const int32_t last = P.experts - 1;
  const char *w[2] = {P.router + (int64_t)min(e0, last) * P.router_stride, P.router + (int64_t)min(e0 + 1, last) * P.router_stride};
  const char *x[ROUTE_ROWS];
#pragma unroll
  for (int r = 0; r < ROUTE_ROWS; ++r) x[r] = P.x + (int64_t)min(block * ROUTE_ROWS + r, rows - 1) * P.x_stride;
  for (int32_t k = lane * 8; k < P.dim; k += 512) {
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
      const int32_t row = block * ROUTE_ROWS + r;
      if (lane == 0 && e0 + i < P.experts && row < rows) put(P.logits + (int64_t)row * P.experts + e0 + i, s);
    }
}

// Numbers of 64 bits as whole numbers of the same order; NaN below all others, and 0 for what is out.
__device__ __forceinline__ uint64_t ordered(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);  // (-0 becomes 0)
  return v != v ? 1u : (b >> 63 ? ~b : b | (uint64_t)1 << 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  auto larger = [](uint64_t a, uint64_t b) { return a > b ? a : b; };
  auto as_d = [](uint64_t x) { return __builtin_bit_cast(double, x); };
  auto as_u = [](double x) { return __builtin_bit_cast(uint64_t, x); };
  v = larger(v, as_u(other_lane<0xb1>(as_d(v))));
  v = larger(v, as_u(other_lane<0x4e>(as_d(v))));
  v = larger(v, as_u(other_lane<0x141>(as_d(v))));
  v = larger(v, as_u(other_lane<0x140>(as_d(v))));
  double a, b;
  across<16>(as_d(v), a, b);
  v = larger(as_u(a), as_u(b));
  across<32>(as_d(v), a, b);
  return larger(as_u(a), as_u(b));
}

// The top_k experts of a row, by one wave: the largest score is taken out top_k times.
__device__ __forceinline__ void choose(const SK_CONSTANT MoeDev &P, int32_t row, int lane) {
  constexpr int N = MOE_EXPERTS / 64;
  const int32_t most = (P.experts + 63) / 64;
  double score[N];
  uint64_t key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int32_t e = i * 64 + lane;
    score[i] = i < most && e < P.experts ? got(P.logits + (int64_t)row * P.experts + e) : -__builtin_inf();
  }
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = i * 64 + lane < P.experts ? ordered(score[i]) : 0u;
  if (P.scoring == SK_MOE_SOFTMAX) {
    double top = -__builtin_inf(), sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmax(top, score[i]);
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < most) {
        score[i] = exp(score[i] - top);
        sum += i * 64 + lane < P.experts ? score[i] : 0.0;
      }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < N; ++i) score[i] /= sum;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < most) score[i] = 1.0 / (1.0 + exp(-score[i]));
  }
  if (P.bias || P.scoring != SK_MOE_SOFTMAX) {  // (a softmax keeps the order of its logits, which tell apart what it rounds to the same)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t e = i * 64 + lane;
      if (e < P.experts) key[i] = ordered(score[i] + (P.bias ? (double)load_f(P.bias + e) : 0.0));
    }
  }
  int32_t mine = 0;  // lane j: the j-th choice
  double mine_score = 0.0, sum = 0.0;
  for (int32_t j = 0; j < P.top_k; ++j) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) best = key[i] > best ? key[i] : best;
    best = wave_max(best);
    bool found = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t hit = __ballot(key[i] == best);
      if (found || !hit) continue;
      found = true;
      const int l = (int)__builtin_ctzll(hit);
      const uint64_t b = __builtin_bit_cast(uint64_t, score[i]);
      const double s = __builtin_bit_cast(double, (uint64_t)(uint32_t)lane_of((int32_t)(b >> 32), l) << 32 | (uint32_t)lane_of((int32_t)b, l));
      sum += s;
      if (lane == j) mine = i * 64 + l, mine_score = s;
      if (lane == l) key[i] = 0;
    }
  }
  if (lane < P.top_k) {
    const int64_t at = (int64_t)row * P.top_k + lane;
    const float weight = (float)((P.normalize ? mine_score / sum : mine_score) * (double)P.scale);
    put(P.ids + at, mine);
    put(P.weights + at, weight);
    if (P.user_ids) P.user_ids[at] = mine;
    if (P.user_weights) P.user_weights[at] = weight;
  }
}

// Which rows go to which expert: every chosen pair gets a place, those of one expert side by side in the order of their rows; and the list of
// groups of up to MOE_GROUP places of an expert.  A bit for every row and expert stands in LDS, so that nothing depends on the order
// of the atomics that set them.
struct Sorting {
  uint32_t bits[MOE_EXPERTS][MOE_ROWS / 32];
  int32_t count[MOE_EXPERTS], first[MOE_EXPERTS];
};
__device__ __forceinline__ void sort_pairs(const SK_CONSTANT MoeDev &P, int32_t rows, Sorting &s, int tid) {
  const int32_t pairs = rows * P.top_k, words = (rows + 31) / 32;
  for (int32_t i = tid; i < P.experts * (MOE_ROWS / 32); i += CACHE_THREADS) (&s.bits[0][0])[i] = 0;
  __syncthreads();
  for (int32_t i = tid; i < pairs; i += CACHE_THREADS) {
    const int32_t row = i / P.top_k, e = got(P.ids + i);
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
    int32_t places = 0, groups = 0;
    for (int32_t e0 = 0; e0 < P.experts; e0 += 64) {
      const int32_t e = e0 + tid, n = e < P.experts ? s.count[e] : 0, g = (n + MOE_GROUP - 1) / MOE_GROUP;
      const int32_t to_n = wave_scan(n), to_g = wave_scan(g);
      if (e < P.experts) s.first[e] = places + to_n - n;
      for (int32_t i = 0; i < g; ++i) {
        MoeGroup *at = P.groups + groups + to_g - g + i;
        put(&at->expert, e);
        put(&at->first, places + to_n - n + i * MOE_GROUP);
        put(&at->rows, min(MOE_GROUP, n - i * MOE_GROUP));
      }
      places += lane_of(to_n, 63);
      groups += lane_of(to_g, 63);
    }
    if (tid == 0) put(P.n_groups, groups);
  }
  __syncthreads();
  for (int32_t i = tid; i < pairs; i += CACHE_THREADS) {
    const int32_t row = i / P.top_k, e = got(P.ids + i);
    int32_t at = s.first[e] + __popc(s.bits[e][row / 32] & ((1u << (row % 32)) - 1));
    for (int32_t w = 0; w < row / 32; ++w) at += __popc(s.bits[e][w]);
    put(P.places + i, at);
    put(P.row_of + at, row);
  }
}

__global__ void __launch_bounds__(CACHE_THREADS) sk_moe_route(MoeArgs a) {
  __shared__ Sorting sorting;
  __shared__ uint32_t flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t part = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, lane));
  const SK_CONSTANT MoeDev &P = *(const SK_CONSTANT MoeDev *)(uintptr_t)(a.parts + part);
  const int32_t unit = (int32_t)(blockIdx.x - ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[part]);
  const int32_t by_experts = (P.experts + ROUTE_EXPERTS - 1) / ROUTE_EXPERTS, blocks = (P.rows + ROUTE_ROWS - 1) / ROUTE_ROWS;
  const int32_t block = unit / by_experts, e0 = unit % by_experts * ROUTE_EXPERTS + 2 * wave, rows = rows_of(P);
  if (block * ROUTE_ROWS < rows && e0 < P.experts) {
    if (P.dtype == SK_BF16) P.router_f32 ? route_scores<SK_BF16, true>(P, rows, block, e0, lane) : route_scores<SK_BF16, false>(P, rows, block, e0, lane);
    else P.router_f32 ? route_scores<SK_F16, true>(P, rows, block, e0, lane) : route_scores<SK_F16, false>(P, rows, block, e0, lane);
  }
  if (!last_to_arrive(P.routed + block, by_experts, &flag)) return;
  const int32_t row = block * ROUTE_ROWS + wave;
  if (row < rows) choose(P, row, lane);
  if (!last_to_arrive(P.blocks_routed, blocks, &flag)) return;
  sort_pairs(P, rows, sorting, tid);
}

// ---------------------------------------------------------------------------
// the experts' products
// ---------------------------------------------------------------------------
// Rows of weights times up to 16 * NB rows of activations, both with their reduction in blocks of 64 elements (128 bytes a row): the four waves of a
// workgroup take the blocks in turn, and their sums are added up in LDS.
//
// An instruction loads eight whole lines of 128 bytes: lane (r, q) of the 16 x 4 that the matrix instruction sees has row r % 8 (+ 8), bytes
// 16 (q + 4 (r / 8)).  Half of the lanes' pieces change places within their row of 16 lanes, and the matrix instruction's operands are there.
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

// W matrices of weights with the same rows and the same activations (gate and up).
template <int DT, int NB, int W>
__device__ __forceinline__ void product(const char *const (&weights)[W], int64_t row_stride, int32_t row0, int32_t rows_end, const char *const (&x)[NB], int32_t k_len, int wave, int lane,
                                        f32x4 (&acc)[W][NB]) {
  constexpr int R = NB == 4 ? 2 : NB == 2 ? 3 : 4;  // blocks in flight
  const int r16 = lane & 15, q = lane >> 4;
  const int32_t blocks = (k_len + 63) / 64, mine = blocks > wave ? (blocks - wave + 3) / 4 : 0;
  const char *at[W][2];
#pragma unroll
  for (int m = 0; m < W; ++m)
#pragma unroll
    for (int j = 0; j < 2; ++j) at[m][j] = weights[m] + (int64_t)min(row0 + 8 * j + (r16 & 7), rows_end - 1) * row_stride;
  u32x4 w[R][W][2], b[R][NB][2];
  auto load = [&](int32_t i, u32x4(&w)[W][2], u32x4(&b)[NB][2]) {
    const int32_t block = wave + 4 * i, k = block * 64 + 8 * (q + 4 * (r16 >> 3));
    const bool in = i < mine && k < k_len;
#pragma unroll
    for (int m = 0; m < W; ++m)
#pragma unroll
      for (int j = 0; j < 2; ++j) w[m][j] = load16(in ? at[m][j] + 2 * (int64_t)k : (const char *)g_zeros);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t kx = block * 64 + 32 * h + 8 * q;
      const bool in_x = i < mine && kx < k_len;
#pragma unroll
      for (int n = 0; n < NB; ++n) b[n][h] = load16(in_x ? x[n] + 2 * (int64_t)kx : (const char *)g_zeros);
    }
  };
#pragma unroll
  for (int u = 0; u < R; ++u) load(u, w[u], b[u]);
  for (int32_t i = 0; i < mine; i += R) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
#pragma unroll
      for (int m = 0; m < W; ++m) {
        const u32x4 lo = low_half(w[u][m][0], w[u][m][1]), hi = high_half(w[u][m][0], w[u][m][1]);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          mma16<DT>(lo, b[u][n][0], acc[m][n]);
          mma16<DT>(hi, b[u][n][1], acc[m][n]);
        }
      }
      load(i + u + R, w[u], b[u]);
    }
  }
}

// The waves' sums, in LDS: [wave][matrix][block of 16 rows][lane].  Returns the sum of what the waves have for (matrix, block) in lane `lane`.
template <int NB, int W>
struct Joined {
  f32x4 (*red)[W][NB][64];
  __device__ __forceinline__ void put(int wave, int lane, const f32x4 (&acc)[W][NB]) {
#pragma unroll
    for (int m = 0; m < W; ++m)
#pragma unroll
      for (int n = 0; n < NB; ++n) red[wave][m][n][lane] = acc[m][n];
    __syncthreads();
  }
  __device__ __forceinline__ f32x4 get(int m, int n, int lane) const { return (red[0][m][n][lane] + red[1][m][n][lane]) + (red[2][m][n][lane] + red[3][m][n][lane]); }
};

// h of 16 columns of an expert for the rows of a group.
template <int DT, int NB, bool GATED>
__device__ __forceinline__ void up_tile(const SK_CONSTANT MoeDev &P, const char *gate, const char *up, int64_t row_stride, int32_t width, int32_t f0, const MoeGroup &g, unsigned char *lds,
                                        int tid) {
  constexpr int W = GATED ? 2 : 1;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q = lane >> 4;
  const char *x[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int32_t i = min(n * 16 + r16, g.rows - 1);  // (columns behind the last repeat it and are not stored)
    x[n] = P.x + (int64_t)(g.expert < 0 ? g.first + i : got(P.row_of + g.first + i)) * P.x_stride;
  }
  f32x4 acc[W][NB] = {};
  const char *weights[W];
  weights[0] = up;
  if constexpr (GATED) weights[1] = gate;
  product<DT, NB, W>(weights, row_stride, f0, width, x, P.dim, wave, lane, acc);
  Joined<NB, W> joined{(f32x4(*)[W][NB][64])lds};
  joined.put(wave, lane, acc);
  for (int n = wave; n < NB; n += 4) {
    f32x4 h = joined.get(0, n, lane);
    if constexpr (GATED) {
      const f32x4 z = joined.get(1, n, lane);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] *= activated(P.act, z[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = activated(P.act, h[k]);
    }
    const int32_t i = n * 16 + r16, f = f0 + 4 * q;
    if (i < g.rows && f < width) {  // (width is a multiple of 8)
      const int64_t place = g.expert < 0 ? (int64_t)P.rows * P.top_k + g.first + i : g.first + i;
      put((uint64_t *)(P.h + place * P.h_stride + 2 * f), (uint64_t)pack2<DT>(h[2], h[3]) << 32 | pack2<DT>(h[0], h[1]));
    }
  }
}

constexpr int MOE_LDS = 4 * 2 * 4 * 64 * 16;

template <int DT>
__device__ __forceinline__ void up_unit(const SK_CONSTANT MoeDev &P, const MoeGroup &g, int32_t tile, unsigned char *lds, int tid) {
  const bool shared = g.expert < 0;
  const char *gate = shared ? P.shared_gate : P.gate + g.expert * P.up_expert, *up = shared ? P.shared_up : P.up + g.expert * P.up_expert;
  const int64_t stride = shared ? 2 * (int64_t)P.dim : P.up_row;
  const int32_t width = shared ? P.shared_ffn : P.ffn, f0 = tile * P.up_rows;
  if (P.gate) {
    if (g.rows <= 16) up_tile<DT, 1, true>(P, gate, up, stride, width, f0, g, lds, tid);
    else if (g.rows <= 32) up_tile<DT, 2, true>(P, gate, up, stride, width, f0, g, lds, tid);
    else up_tile<DT, 4, true>(P, gate, up, stride, width, f0, g, lds, tid);
  } else {
    if (g.rows <= 16) up_tile<DT, 1, false>(P, gate, up, stride, width, f0, g, lds, tid);
    else if (g.rows <= 32) up_tile<DT, 2, false>(P, gate, up, stride, width, f0, g, lds, tid);
    else up_tile<DT, 4, false>(P, gate, up, stride, width, f0, g, lds, tid);
  }
}

template <int DT, int NB>
__device__ __forceinline__ void down_tile(const SK_CONSTANT MoeDev &P, const char *weights, int64_t row_stride, int32_t width, int32_t d0, const MoeGroup &g, unsigned char *lds, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q = lane >> 4;
  const int64_t place0 = g.expert < 0 ? (int64_t)P.rows * P.top_k + g.first : g.first;
  const char *x[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) x[n] = P.h + (place0 + min(n * 16 + r16, g.rows - 1)) * P.h_stride;
  f32x4 acc[1][NB] = {};
  const char *const w[1] = {weights};
  product<DT, NB, 1>(w, row_stride, d0, P.dim, x, width, wave, lane, acc);
  Joined<NB, 1> joined{(f32x4(*)[1][NB][64])lds};
  joined.put(wave, lane, acc);
  for (int n = wave; n < NB; n += 4) {
    const f32x4 v = joined.get(0, n, lane);
    const int32_t i = n * 16 + r16, d = d0 + 4 * q;
    if (i < g.rows && d < P.dim) {
      float *at = P.part + (place0 + i) * P.part_stride + d;
      store_shared(at, f32x2{v[0], v[1]});
      store_shared(at + 2, f32x2{v[2], v[3]});
    }
  }
}

template <int DT>
__device__ __forceinline__ void down_unit(const SK_CONSTANT MoeDev &P, const MoeGroup &g, int32_t tile, unsigned char *lds, int tid) {
  const bool shared = g.expert < 0;
  const char *w = shared ? P.shared_down : P.down + g.expert * P.down_expert;
  const int32_t width = shared ? P.shared_ffn : P.ffn, d0 = tile * P.down_rows;
  const int64_t stride = shared ? 2 * (int64_t)width : P.down_row;
  if (g.rows <= 16) down_tile<DT, 1>(P, w, stride, width, d0, g, lds, tid);
  else if (g.rows <= 32) down_tile<DT, 2>(P, w, stride, width, d0, g, lds, tid);
  else down_tile<DT, 4>(P, w, stride, width, d0, g, lds, tid);
}

// The weighted sum of a tile's columns for all rows, in the order of the choices.
template <int DT>
__device__ __forceinline__ void add_up(const SK_CONSTANT MoeDev &P, int32_t rows, int32_t tile, int tid) {
  const int32_t quads = min(P.down_rows, P.dim - tile * P.down_rows) / 4;
  for (int32_t i = tid; i < rows * quads; i += CACHE_THREADS) {
    const int32_t row = i / quads, d = tile * P.down_rows + 4 * (i % quads);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (P.shared_ffn) {
      const float *at = P.part + ((int64_t)P.rows * P.top_k + row) * P.part_stride + d;
      const f32x2 a = load_shared(at), b = load_shared(at + 2);
      sum = f32x4{a[0], a[1], b[0], b[1]};
    }
    for (int32_t j = 0; j < P.top_k; ++j) {
      const float w = got(P.weights + row * P.top_k + j);
      const float *at = P.part + (int64_t)got(P.places + row * P.top_k + j) * P.part_stride + d;
      const f32x2 a = load_shared(at), b = load_shared(at + 2);
      sum[0] += w * a[0], sum[1] += w * a[1], sum[2] += w * b[0], sum[3] += w * b[1];
    }
    store8(P.out + row * P.out_stride + 2 * d, u32x2{pack2<DT>(sum[0], sum[1]), pack2<DT>(sum[2], sum[3])});
  }
}

// The group of a unit, those of the shared expert first, and its tile; no rows: there is no such unit.
__device__ __forceinline__ MoeGroup find_unit(const SK_CONSTANT MoeDev &P, int32_t rows, int32_t unit, int32_t shared_tiles, int32_t tiles, int32_t &tile) {
  const int32_t shared = P.shared_ffn ? (rows + MOE_GROUP - 1) / MOE_GROUP * shared_tiles : 0;
  const bool is_shared = unit < shared;
  const int32_t of = is_shared ? shared_tiles : tiles, at = is_shared ? unit : unit - shared, i = at / of;
  tile = at - i * of;
  const int32_t first = i * MOE_GROUP;
  if (is_shared) return MoeGroup{-1, first, min(MOE_GROUP, rows - first), 0};
  if (i >= __builtin_amdgcn_readfirstlane(got(P.n_groups))) return MoeGroup{0, 0, 0, 0};
  return MoeGroup{__builtin_amdgcn_readfirstlane(got(&P.groups[i].expert)), __builtin_amdgcn_readfirstlane(got(&P.groups[i].first)),
                  __builtin_amdgcn_readfirstlane(got(&P.groups[i].rows)), 0};
}

__global__ void __launch_bounds__(CACHE_THREADS, 3) sk_moe_up(MoeArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[MOE_LDS];
  const int32_t part = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, threadIdx.x & 63));
  const SK_CONSTANT MoeDev &P = *(const SK_CONSTANT MoeDev *)(uintptr_t)(a.parts + part);
  const int32_t unit = (int32_t)(blockIdx.x - ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[part]);
  int32_t tile;
  const MoeGroup g = find_unit(P, rows_of(P), unit, P.shared_tiles, P.up_tiles, tile);
  if (!g.rows) return;
  if (P.dtype == SK_BF16) up_unit<SK_BF16>(P, g, tile, lds, threadIdx.x);
  else up_unit<SK_F16>(P, g, tile, lds, threadIdx.x);
}

__global__ void __launch_bounds__(CACHE_THREADS, 3) sk_moe_down(MoeArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[MOE_LDS];
  __shared__ uint32_t flag;
  const int32_t part = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, threadIdx.x & 63));
  const SK_CONSTANT MoeDev &P = *(const SK_CONSTANT MoeDev *)(uintptr_t)(a.parts + part);
  const int32_t unit = (int32_t)(blockIdx.x - ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[part]);
  const int32_t rows = rows_of(P);
  int32_t tile;
  const MoeGroup g = find_unit(P, rows, unit, P.down_tiles, P.down_tiles, tile);
  if (!g.rows) return;
  if (P.dtype == SK_BF16) down_unit<SK_BF16>(P, g, tile, lds, threadIdx.x);
  else down_unit<SK_F16>(P, g, tile, lds, threadIdx.x);
  const int32_t groups = got(P.n_groups) + (P.shared_ffn ? (rows + MOE_GROUP - 1) / MOE_GROUP : 0);
  if (!last_to_arrive(P.summed + tile, groups, &flag)) return;
  if (P.dtype == SK_BF16) add_up<SK_BF16>(P, rows, tile, threadIdx.x);
  else add_up<SK_F16>(P, rows, tile, threadIdx.x);
}

}  // namespace sk

struct sk_moe_plan : sk::PlanOnDevice {
  sk::MoePlanHost host;
  const sk::MoeDev *parts = nullptr;
  const uint32_t *first[3] = {};  // of the router, of up, of down
};

namespace {

sk_status upload(sk_moe_plan &plan) {
  sk::MoePlanHost &h = plan.host;
  const std::vector<uint32_t> *firsts[3] = {&h.route_first, &h.up_first, &h.down_first};
  // counters, parts, first workgroups
  const size_t o_parts = sk::align_up(h.counters, 256);
  size_t o_first[4] = {o_parts + sk::align_up(h.parts.size() * sizeof(sk::MoeDev), 256)};
  for (int i = 0; i < 3; ++i) o_first[i + 1] = o_first[i] + sk::align_up(firsts[i]->size() * 4, 256);
  std::vector<char> image(o_first[3], 0);
  char *ws = nullptr;
  const sk_status st = sk::upload_image(plan, image, h.workspace, &ws);
  if (st != SK_OK) return st;
  auto moved = [](auto *&p, char *base) { p = (std::decay_t<decltype(p)>)(base + (uintptr_t)p); };
  std::vector<sk::MoeDev> parts = h.parts;
  for (sk::MoeDev &d : parts) {
    moved(d.routed, plan.blob), moved(d.blocks_routed, plan.blob), moved(d.summed, plan.blob);
    moved(d.logits, ws), moved(d.ids, ws), moved(d.places, ws), moved(d.weights, ws), moved(d.row_of, ws), moved(d.groups, ws), moved(d.n_groups, ws), moved(d.h, ws), moved(d.part, ws);
  }
  if (!parts.empty()) std::memcpy(image.data() + o_parts, parts.data(), parts.size() * sizeof(sk::MoeDev));
  for (int i = 0; i < 3; ++i) {
    std::memcpy(image.data() + o_first[i], firsts[i]->data(), firsts[i]->size() * 4);
    plan.first[i] = (const uint32_t *)(plan.blob + o_first[i]);
  }
  plan.parts = (const sk::MoeDev *)(plan.blob + o_parts);
  return sk::copy_image(plan, image);
}

}  // namespace

extern "C" {

sk_status sk_moe_plan_create(const sk_moe_problem *problems, int32_t n, const sk_layer_params *params, sk_moe_plan **out) {
  return sk::create_plan<sk_moe_plan>(params, out, [&](sk_moe_plan &plan, int32_t workgroups, std::string &err) { return sk::plan_moe(problems, n, workgroups, plan.host, err); }, upload);
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
    auto args = [&](int i) { return sk::MoeArgs{plan->parts, plan->first[i], (int32_t)plan->host.parts.size()}; };
    st = sk::launch(sk::sk_moe_route, (int64_t)plan->host.route_first.back(), stream, nullptr, args(0));
    if (st == SK_OK) st = sk::launch(sk::sk_moe_up, (int64_t)plan->host.up_first.back(), stream, nullptr, args(1));
    if (st == SK_OK) st = sk::launch(sk::sk_moe_down, (int64_t)plan->host.down_first.back(), stream, behind, args(2));
    plan->ledger.after_launch((uintptr_t)stream, in_capture, behind && st == SK_OK);  // also after a failure: some launches may be out
    return st;
  });
}

sk_status sk_moe_plan_info(const sk_moe_plan *plan, int32_t *launches, int64_t *workspace_bytes) {
  return sk::guarded([&]() -> sk_status {
    if (!plan) return sk::set_last_error(SK_ERR_INVALID_ARG, "plan is null");
    if (launches) *launches = plan->host.parts.empty() ? 0 : 3;
    if (workspace_bytes) *workspace_bytes = (int64_t)(plan->host.workspace + plan->host.counters);
    return SK_OK;
  });
}

}  // extern "C"
