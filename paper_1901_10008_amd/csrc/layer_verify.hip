// Verification of drafted tokens and sampling: the kernels and their entry points.
#include "layer_host.h"
#include "layer_math.hip.h"

namespace sk {

struct VerifyArgs {
  const VerifyDev *problems;
  const uint32_t *first;  // first workgroup of each problem
  int32_t n;
};

// 2^t for t <= 0, 0 below 2^-1000, to 8e-13 of itself: 2^f of the rest f in [-1/2, 1/2] by the polynomial of degree 8 with the least largest relative
// error, which moves a border between two tokens by less than one in 10^12 of the sum.  Fused multiplications and additions of 64 bits have the
// rate of those of 32 here; there is no exponential of 64 bits in the hardware.  (t is a NaN where a logit is: the caller looks for those.)
__device__ __forceinline__ double exp2_64(double t) {
  const double shift = 6755399441055744.0;  // 1.5 * 2^52: t + shift has the nearest whole number of t in its lowest bits
  const double moved = t + shift, f = t - (moved - shift);
  double r = 1.3175858118613272e-06;
  r = fma(r, f, 1.530973742145504e-05);
  r = fma(r, f, 1.5403851748706403e-04);
  r = fma(r, f, 1.3333452062251156e-03);
  r = fma(r, f, 9.618128542862427e-03);
  r = fma(r, f, 5.550410939341707e-02);
  r = fma(r, f, 2.4022650698880368e-01);
  r = fma(r, f, 6.931471805465141e-01);
  r = fma(r, f, 9.999999999997623e-01);
  const uint64_t b = __builtin_bit_cast(uint64_t, r);
  const uint32_t hi = (uint32_t)(b >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, moved) << 20);
  return t > -1000.0 ? __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)b) : 0.0;
}

// log2(e) / temperature of a sequence; 0: the first of the largest.
__device__ __forceinline__ double scale_of(const SK_CONSTANT VerifyDev &P, int32_t seq) {
  const float t = P.temperatures ? load_f(P.temperatures + seq) : P.temperature;
  return t > 0.f ? fmax(1.4426950408889634074 / (double)t, 1e-300) : 0.0;  // (not 0 where t is infinite)
}
__device__ __forceinline__ bool greedy(double c) { return c == 0.0; }

// Eight logits from place `at` on, -infinity behind the last.
template <int DT>
__device__ __forceinline__ void logits8(const char *row, int64_t at, int32_t vocab, float (&x)[8]) {
  constexpr int S = DT == SK_F32 ? 4 : 2;
  if (at + 8 <= vocab) {
    load8<DT, false>(row + at * S, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = load1<DT>(row + min(at + k, (int64_t)vocab - 1) * S);
      x[k] = at + k < vocab ? v : -__builtin_inff();
    }
  }
}

struct VerifyShared {
  double d[4];
  float f[4];
  int32_t i[4], any[4];
};

// A chunk of a row: its largest logit, and the sum of 2^((l - largest) * c).
template <int DT>
__device__ __forceinline__ void chunk_stat(const SK_CONSTANT VerifyDev &P, const char *row, int32_t chunk, double c, VerifyStat *out, VerifyShared &s, int tid) {
  constexpr int P_MOST = 4;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float x[P_MOST][8];
  const int64_t at0 = (int64_t)chunk * 2048 * P.pieces + tid * 8;
#pragma unroll
  for (int i = 0; i < P_MOST; ++i)
    if (i < P.pieces) logits8<DT>(row, at0 + i * 2048, P.vocab, x[i]);
  float top = -__builtin_inff();
  bool bad = false;
#pragma unroll
  for (int i = 0; i < P_MOST; ++i)
    if (i < P.pieces) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        top = fmaxf(top, x[i][k]);
        bad |= !(x[i][k] < __builtin_inff());
      }
    }
  top = wave_max(top);
  const bool any_bad = __ballot(bad) != 0;
  if (lane == 0) s.f[wave] = top, s.any[wave] = any_bad;
  __syncthreads();
  top = fmaxf(fmaxf(s.f[0], s.f[1]), fmaxf(s.f[2], s.f[3]));
  double sum = 0.0;
  int32_t at = 0x7fffffff;
  if (greedy(c)) {
#pragma unroll
    for (int i = 0; i < P_MOST; ++i)
      if (i < P.pieces) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (x[i][k] == top) at = min(at, (int32_t)(at0 + i * 2048) + k);
      }
    at = wave_min(at);
    sum = 1.0;
  } else if (top > -__builtin_inff()) {
    const double m = (double)top;
#pragma unroll
    for (int i = 0; i < P_MOST; ++i)
      if (i < P.pieces) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += exp2_64(((double)x[i][k] - m) * c);
      }
    sum = wave_sum(sum);
  }
  if (lane == 0) s.d[wave] = sum, s.i[wave] = at;
  __syncthreads();
  if (tid == 0) {
    const bool not_one = s.any[0] | s.any[1] | s.any[2] | s.any[3];
    *out = VerifyStat{not_one ? __builtin_nan("") : greedy(c) ? 1.0 : (s.d[0] + s.d[1]) + (s.d[2] + s.d[3]), top, min(min(s.i[0], s.i[1]), min(s.i[2], s.i[3]))};
  }
}

__device__ __forceinline__ int32_t first_of(const SK_CONSTANT VerifyDev &P, int32_t s) { return min(max(load_i32(P.first_row + s), 0), P.rows); }

__global__ void __launch_bounds__(CACHE_THREADS) sk_verify_stats(VerifyArgs a) {
  __shared__ VerifyShared shared;
  const int tid = threadIdx.x, lane = tid & 63;
  const int32_t problem = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, lane));
  const SK_CONSTANT VerifyDev &P = *(const SK_CONSTANT VerifyDev *)(uintptr_t)(a.problems + problem);
  const uint32_t unit = blockIdx.x - ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[problem];
  const uint32_t sides = P.draft_logits ? 2 : 1, line = unit / (uint32_t)P.chunks;
  const int32_t chunk = (int32_t)(unit - line * (uint32_t)P.chunks), row = (int32_t)(line / sides);
  const bool draft = sides == 2 && (line & 1);
  const int32_t seq = __builtin_amdgcn_readfirstlane(last_not_above(P.first_row, P.sequences, row, lane));
  const int32_t r0 = first_of(P, seq), r1 = first_of(P, seq + 1);
  if (row < r0 || row >= r1 || (draft && row == r1 - 1)) return;
  const double c = scale_of(P, seq);
  if (draft && greedy(c)) return;
  const char *at = draft ? P.draft_logits + row * P.draft_stride : P.logits + row * P.logits_stride;
  VerifyStat *out = P.stats + ((int64_t)row * 2 + draft) * P.chunks + chunk;
  if (P.dtype == SK_F32) chunk_stat<SK_F32>(P, at, chunk, c, out, shared, tid);
  else if (P.dtype == SK_BF16) chunk_stat<SK_BF16>(P, at, chunk, c, out, shared, tid);
  else chunk_stat<SK_F16>(P, at, chunk, c, out, shared, tid);
}

// A row's distribution from its chunks, by a wave: p(k) = 2^((l_k - top) * c) / sum.  sum 0: it has none.
struct Row {
  double top, sum;
  int32_t at;  // (temperature 0) the only token
};
__device__ __forceinline__ Row row_stat(const VerifyStat *stats, int32_t chunks, double c, int lane) {
  float top = -__builtin_inff();
  bool bad = false;
  for (int32_t i = lane; i < chunks; i += 64) {
    top = fmaxf(top, stats[i].top);
    bad |= stats[i].sum != stats[i].sum;
  }
  top = wave_max(top);
  Row r{(double)top, 0.0, -1};
  if (__ballot(bad) || !(top > -__builtin_inff())) return r;
  int32_t at = 0x7fffffff;
  for (int32_t i = lane; i < chunks; i += 64) {
    const double scale = exp2_64(((double)stats[i].top - r.top) * c);
    r.sum += stats[i].top > -__builtin_inff() ? stats[i].sum * scale : 0.0;
    if (stats[i].top == top) at = min(at, stats[i].at);
  }
  r.sum = wave_sum(r.sum);
  r.at = wave_min(at);
  return r;
}

template <int DT>
__device__ __forceinline__ double logit(const char *row, int32_t at) {
  return (double)load1<DT>(row + (int64_t)at * (DT == SK_F32 ? 4 : 2));
}

// What the sampled token of a sequence is drawn from.
enum { FROM_NOTHING, FROM_ONE, FROM_TARGET, FROM_OTHERS, FROM_DIFFERENCE };
struct Draw {
  int32_t stop, mode, token;  // row within the sequence; FROM_OTHERS: all but this token
  Row p, q;
};

// Weights of eight tokens.
template <int DT>
__device__ __forceinline__ void weights8(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, int64_t at, double c, double (&w)[8]) {
  float x[8], y[8];
  logits8<DT>(p_row, at, P.vocab, x);
  if (d.mode == FROM_DIFFERENCE) logits8<DT>(q_row, at, P.vocab, y);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    w[k] = exp2_64(((double)x[k] - d.p.top) * c);
    if (d.mode == FROM_DIFFERENCE) w[k] = fmax(w[k] / d.p.sum - exp2_64(((double)y[k] - d.q.top) * c) / d.q.sum, 0.0);
    if (d.mode == FROM_OTHERS && at + k == d.token) w[k] = 0.0;
  }
}

// The sum of a chunk's weights, in all threads.
template <int DT>
__device__ __forceinline__ double chunk_sum(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, int32_t chunk, double c, VerifyShared &s, int tid) {
  double sum = 0.0;
  for (int32_t i = 0; i < P.pieces; ++i) {
    const int64_t at = ((int64_t)chunk * P.pieces + i) * 2048 + tid * 8;
    if (at >= P.vocab) break;
    double w[8];
    weights8<DT>(P, d, p_row, q_row, at, c, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += w[k];
  }
  sum = wave_sum(sum);
  __syncthreads();
  if ((tid & 63) == 0) s.d[tid >> 6] = sum;
  __syncthreads();
  return (s.d[0] + s.d[1]) + (s.d[2] + s.d[3]);
}

// The first token whose weight and those before it add up to more than `random` times all.  sum_of(i) is the sum of chunk i (asked for by the first
// wave).  -1: all weights are 0.
template <int DT, class F>
__device__ __forceinline__ int32_t pick(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, double c, double random, F sum_of, VerifyShared &s, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __syncthreads();
  if (wave == 0) {
    double total = 0.0;
    int32_t last = -1;
    for (int32_t i0 = 0; i0 < P.chunks; i0 += 64) {
      const double v = i0 + lane < P.chunks ? sum_of(i0 + lane) : 0.0;
      const uint64_t some = __ballot(v > 0.0);
      if (some) last = i0 + 63 - (int)__builtin_clzll(some);
      const double upto = total + wave_scan(v);
      total = __shfl(upto, 63);
    }
    const double bound = random * total;
    double before = 0.0, begin = 0.0, all = 0.0;
    int32_t chunk = -1;
    for (int32_t i0 = 0; i0 < P.chunks && chunk < 0; i0 += 64) {
      const double v = i0 + lane < P.chunks ? sum_of(i0 + lane) : 0.0;
      const double upto = all + wave_scan(v);
      const uint64_t past = __ballot(upto > bound && v > 0.0);
      const int l = past ? (int)__builtin_ctzll(past) : 0;
      const double below = __shfl_up(upto, 1);
      before = lane == 0 ? all : below;
      if (past) chunk = i0 + l, begin = __shfl(before, l);
      all = __shfl(upto, 63);
    }
    if (chunk < 0) chunk = last, begin = -1.0;  // (rounding: the last token with a weight)
    if (lane == 0) s.d[0] = begin, s.d[1] = bound, s.i[0] = chunk;
  }
  __syncthreads();
  const double bound = s.d[1];
  double begin = s.d[0];
  const int32_t chunk = s.i[0];
  if (chunk < 0) return -1;
  const bool none = begin < 0.0;
  int32_t last = -1;
  for (int32_t i = 0; i < P.pieces; ++i) {
    const int64_t at = ((int64_t)chunk * P.pieces + i) * 2048 + tid * 8;
    double w[8] = {}, mine = 0.0;
    if (at < P.vocab) weights8<DT>(P, d, p_row, q_row, at, c, w);
    int32_t my_last = -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      mine += w[k];
      if (w[k] > 0.0) my_last = (int32_t)at + k;
    }
    const double upto = wave_scan(mine);
    __syncthreads();
    if (lane == 63) s.d[wave] = upto;
    __syncthreads();
    double sum = begin + (wave > 0 ? s.d[0] : 0.0) + (wave > 1 ? s.d[1] : 0.0) + (wave > 2 ? s.d[2] : 0.0);
    begin += (s.d[0] + s.d[1]) + (s.d[2] + s.d[3]);
    const double below = __shfl_up(upto, 1);
    sum += lane ? below : 0.0;
    int32_t found = 0x7fffffff;
#pragma unroll
    for (int k = 7; k >= 0; --k) {
      double upto_k = sum;
#pragma unroll
      for (int j = 0; j <= k; ++j) upto_k += w[j];
      if (!none && upto_k > bound && w[k] > 0.0) found = (int32_t)at + k;
    }
    found = wave_min(found);
    my_last = -wave_min(-my_last);
    if (lane == 0) s.i[wave] = found, s.any[wave] = my_last;
    __syncthreads();
    found = min(min(s.i[0], s.i[1]), min(s.i[2], s.i[3]));
    last = max(last, max(max(s.any[0], s.any[1]), max(s.any[2], s.any[3])));
    __syncthreads();
    if (found != 0x7fffffff) return found;
  }
  return last;
}

__device__ __forceinline__ double random_of(const float *p) {
  const float u = load_f(p);
  return u > 0.f ? (double)fminf(u, 0.99999994f) : 0.0;
}

// What becomes of a sequence's drafts: by all waves, a row each at a time.
template <int DT>
__device__ __forceinline__ void decide(const SK_CONSTANT VerifyDev &P, int32_t r0, int32_t n, double c, Draw *draws, int32_t *stop, int tid, Draw &out) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid == 0) *stop = 0x7fffffff;
  __syncthreads();
  for (int32_t i0 = 0;; i0 += 4) {
    const int32_t i = i0 + wave;
    if (i < n) {
      const int64_t row = r0 + i;
      Draw d{};
      d.stop = i, d.token = -1;
      d.p = row_stat(P.stats + row * 2 * P.chunks, P.chunks, c, lane);
      bool accept = false;
      if (!(d.p.sum > 0.0)) {
        d.mode = FROM_NOTHING;
      } else {
        d.mode = greedy(c) ? FROM_ONE : FROM_TARGET;
        const int32_t token = i < n - 1 && P.drafted ? load_i32(P.drafted + row) : -1;
        if (token >= 0 && token < P.vocab) {
          double q = 1.0;
          bool certain = greedy(c) || !P.draft_logits;
          if (!certain) {
            d.q = row_stat(P.stats + (row * 2 + 1) * P.chunks, P.chunks, c, lane);
            certain = !(d.q.sum > 0.0);
            if (!certain) q = exp2_64((logit<DT>(P.draft_logits + row * P.draft_stride, token) - d.q.top) * c) / d.q.sum;
          }
          const double p = greedy(c) ? (token == d.p.at ? 1.0 : 0.0) : exp2_64((logit<DT>(P.logits + row * P.logits_stride, token) - d.p.top) * c) / d.p.sum;
          accept = random_of(P.accept_random + row) * q < p;
          if (!greedy(c)) d.mode = certain ? FROM_OTHERS : FROM_DIFFERENCE;
          d.token = token;
        }
        if (greedy(c)) d.token = d.p.at;
      }
      if (lane == 0) {
        draws[wave] = d;
        if (!accept) atomicMin(stop, i);
      }
    }
    __syncthreads();
    const int32_t at = *stop;
    if (at != 0x7fffffff) {  // (the last row accepts nothing, so there is one)
      out = draws[at - i0];
      return;
    }
    __syncthreads();
  }
}

template <int DT>
__device__ __forceinline__ void sample(const SK_CONSTANT VerifyDev &P, int32_t seq, int32_t chunk, VerifyShared &s, Draw *draws, int32_t *stop, uint32_t *flag, int tid) {
  const int32_t r0 = first_of(P, seq), n = first_of(P, seq + 1) - r0;
  if (n <= 0) {
    if (chunk == 0 && tid == 0) P.accepted[seq] = 0;
    return;
  }
  const double c = scale_of(P, seq);
  Draw d;
  decide<DT>(P, r0, n, c, draws, stop, tid, d);
  const char *p_row = P.logits + (int64_t)(r0 + d.stop) * P.logits_stride, *q_row = d.mode == FROM_DIFFERENCE ? P.draft_logits + (int64_t)(r0 + d.stop) * P.draft_stride : nullptr;
  const double random = random_of(P.sample_random + seq);
  const VerifyStat *stats = P.stats + (int64_t)(r0 + d.stop) * 2 * P.chunks;
  auto from_stats = [&](int32_t i) { return stats[i].top > -__builtin_inff() ? stats[i].sum * exp2_64(((double)stats[i].top - d.p.top) * c) : 0.0; };
  int32_t token = -1;
  if (d.mode == FROM_DIFFERENCE) {
    double *sums = P.sums + (int64_t)seq * P.chunks;
    const double sum = chunk_sum<DT>(P, d, p_row, q_row, chunk, c, s, tid);
    if (tid == 0) put(sums + chunk, sum);
    if (!last_to_arrive(P.arrived + seq, P.chunks, flag)) return;
    token = pick<DT>(P, d, p_row, q_row, c, random, [&](int32_t i) { return got(sums + i); }, s, tid);
  } else if (chunk != 0) {
    return;
  } else if (d.mode == FROM_OTHERS) {
    const int32_t without = d.token / (2048 * P.pieces);
    const double rest = chunk_sum<DT>(P, d, p_row, q_row, without, c, s, tid);
    token = pick<DT>(P, d, p_row, q_row, c, random, [&](int32_t i) { return i == without ? rest : from_stats(i); }, s, tid);
  }
  if (d.mode == FROM_ONE) token = d.token;
  if (d.mode == FROM_TARGET || (d.mode >= FROM_OTHERS && token < 0)) {  // (where p - q is 0 everywhere: from p)
    d.mode = FROM_TARGET;
    token = pick<DT>(P, d, p_row, q_row, c, random, from_stats, s, tid);
  }
  for (int32_t i = tid; i < n; i += CACHE_THREADS) P.tokens[r0 + i] = i < d.stop ? load_i32(P.drafted + r0 + i) : i == d.stop ? token : -1;
  if (tid == 0) P.accepted[seq] = d.stop;
}

__global__ void __launch_bounds__(CACHE_THREADS) sk_verify_sample(VerifyArgs a) {
  __shared__ VerifyShared shared;
  __shared__ Draw draws[4];
  __shared__ int32_t stop;
  __shared__ uint32_t flag;
  const int tid = threadIdx.x;
  const int32_t problem = __builtin_amdgcn_readfirstlane(last_not_above(a.first, a.n, (int64_t)blockIdx.x, tid & 63));
  const SK_CONSTANT VerifyDev &P = *(const SK_CONSTANT VerifyDev *)(uintptr_t)(a.problems + problem);
  const uint32_t unit = blockIdx.x - ((const SK_CONSTANT uint32_t *)(uintptr_t)a.first)[problem];
  const int32_t seq = (int32_t)(unit / (uint32_t)P.chunks), chunk = (int32_t)(unit % (uint32_t)P.chunks);
  if (P.dtype == SK_F32) sample<SK_F32>(P, seq, chunk, shared, draws, &stop, &flag, tid);
  else if (P.dtype == SK_BF16) sample<SK_BF16>(P, seq, chunk, shared, draws, &stop, &flag, tid);
  else sample<SK_F16>(P, seq, chunk, shared, draws, &stop, &flag, tid);
}

}  // namespace sk

struct sk_verify_plan : sk::PlanOnDevice {
  sk::VerifyPlanHost host;
  const sk::VerifyDev *problems = nullptr;
  const uint32_t *first[2] = {};
};

namespace {

sk_status upload(sk_verify_plan &plan) {
  sk::VerifyPlanHost &h = plan.host;
  const std::vector<uint32_t> *firsts[2] = {&h.stat_first, &h.sum_first};
  // counters, problems, first workgroups
  const size_t o_problems = sk::align_up(h.counters, 256);
  size_t o_first[3] = {o_problems + sk::align_up(h.problems.size() * sizeof(sk::VerifyDev), 256)};
  for (int i = 0; i < 2; ++i) o_first[i + 1] = o_first[i] + sk::align_up(firsts[i]->size() * 4, 256);
  std::vector<char> image(o_first[2], 0);
  char *ws = nullptr;
  const sk_status st = sk::upload_image(plan, image, h.workspace, &ws);
  if (st != SK_OK) return st;
  auto moved = [](auto *&p, char *base) { p = (std::decay_t<decltype(p)>)(base + (uintptr_t)p); };
  std::vector<sk::VerifyDev> problems = h.problems;
  for (sk::VerifyDev &d : problems) moved(d.arrived, plan.blob), moved(d.stats, ws), moved(d.sums, ws);
  if (!problems.empty()) std::memcpy(image.data() + o_problems, problems.data(), problems.size() * sizeof(sk::VerifyDev));
  for (int i = 0; i < 2; ++i) {
    std::memcpy(image.data() + o_first[i], firsts[i]->data(), firsts[i]->size() * 4);
    plan.first[i] = (const uint32_t *)(plan.blob + o_first[i]);
  }
  plan.problems = (const sk::VerifyDev *)(plan.blob + o_problems);
  return sk::copy_image(plan, image);
}

}  // namespace

extern "C" {

sk_status sk_verify_plan_create(const sk_verify_problem *problems, int32_t n, const sk_layer_params *params, sk_verify_plan **out) {
  return sk::create_plan<sk_verify_plan>(params, out, [&](sk_verify_plan &plan, int32_t, int32_t, std::string &err) { return sk::plan_verify(problems, n, plan.host, err); }, upload);
}

sk_status sk_verify_plan_destroy(sk_verify_plan *plan) {
  if (!plan) return SK_OK;
  return sk::guarded([&]() -> sk_status { return sk::destroy_plan(plan, false); });
}

sk_status sk_verify_launch(sk_verify_plan *plan, void *hip_stream) {
  return sk::guarded([&]() -> sk_status {
    const hipStream_t stream = (hipStream_t)hip_stream;
    bool in_capture = false;
    sk_status st = sk::admit(plan, stream, &in_capture);
    if (st != SK_OK || plan->host.problems.empty()) return st;
    const hipEvent_t behind = in_capture ? nullptr : plan->last_use;
    auto args = [&](int i) { return sk::VerifyArgs{plan->problems, plan->first[i], (int32_t)plan->host.problems.size()}; };
    st = sk::launch(sk::sk_verify_stats, (int64_t)plan->host.stat_first.back(), stream, nullptr, args(0));
    if (st == SK_OK) st = sk::launch(sk::sk_verify_sample, (int64_t)plan->host.sum_first.back(), stream, behind, args(1));
    plan->ledger.after_launch((uintptr_t)stream, in_capture, behind && st == SK_OK);  // also after a failure: some launches may be out
    return st;
  });
}

sk_status sk_verify_plan_info(const sk_verify_plan *plan, int32_t *launches, int64_t *workspace_bytes) {
  return sk::guarded([&]() -> sk_status {
    if (!plan) return sk::set_last_error(SK_ERR_INVALID_ARG, "plan is null");
    if (launches) *launches = plan->host.problems.empty() ? 0 : 2;
    if (workspace_bytes) *workspace_bytes = (int64_t)(plan->host.workspace + plan->host.counters);
    return SK_OK;
  });
}

}  // extern "C"
