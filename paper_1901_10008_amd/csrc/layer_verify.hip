// Verification of drafted tokens and sampling: the kernels and their entry points.
#include "layer_host.h"
#include "layer_math.hip.h"

namespace sk {

struct VerifyArgs {
  const VerifyTable *table;
  int32_t n;
};

// 2^(d c) to 8e-13 of itself, for -1000 < d c <= 0: 2^f of what the nearest whole number leaves, |f| <= 1/2, by the polynomial of degree 8 with the least
// largest relative error, which moves a border between two tokens by less than one in 10^12 of the sum.  Fused multiplications and additions of
// 64 bits have the rate of those of 32 here; there is no exponential of 64 bits in the hardware.
__device__ __forceinline__ double exp2_of(double d, double c) {
  const double shift = 6755399441055744.0;  // 1.5 * 2^52: behind it, the nearest whole number stands in the lowest bits
  const double moved = fma(d, c, shift), f = fma(d, c, shift - moved);
  double r = 1.3175858118613272e-06;
  r = fma(r, f, 1.530973742145504e-05);
  r = fma(r, f, 1.5403851748706403e-04);
  r = fma(r, f, 1.3333452062251156e-03);
  r = fma(r, f, 9.618128542862427e-03);
  r = fma(r, f, 5.550410939341707e-02);
  r = fma(r, f, 2.4022650698880368e-01);
  r = fma(r, f, 6.931471805465141e-01);
  r = fma(r, f, 9.999999999997623e-01);
  u32x2 bits = __builtin_bit_cast(u32x2, r);
  const u32x2 whole = __builtin_bit_cast(u32x2, moved);
  bits[1] += (uint32_t)whole[0] << 20;
  return __builtin_bit_cast(double, bits);
}
// The same, 0 below 2^-1000 (and for a NaN).
__device__ __forceinline__ double weight_of(double d, double c) { return d * c > -1000.0 ? exp2_of(d, c) : 0.0; }

// log2(e) / temperature of a sequence; 0: the first of the largest.
__device__ __forceinline__ double scale_of(const SK_CONSTANT VerifyDev &P, int32_t seq) {
  const float t = P.temperatures ? load_f(P.temperatures + seq) : P.temperature;
  return t > 0.f ? fmax(1.4426950408889634074 / (double)t, 1e-300) : 0.0;  // (not 0 where t is infinite)
}
__device__ __forceinline__ bool greedy(double c) { return c == 0.0; }

// Eight logits of a row, as they come.  A lane wants those from place `at` on (the wave as a whole 512, from `wave_at` on); where they would end behind the
// row it reads the row's last eight and has -infinity in place of those that belong to the lanes before it.  `first` is the place of the first.
template <int DT>
struct Eight {
  static constexpr int S = DT == SK_F32 ? 4 : 2;
  u32x4 raw[S / 2];
  int32_t first;
  // SHORT: rows may have fewer than eight (without it they must not: the planner gives those chunks of one piece)
  template <bool SHORT>
  __device__ __forceinline__ void load(const char *row, int32_t wave_at, int lane, int32_t vocab) {
    constexpr uint32_t lowest = DT == SK_F32 ? 0xff800000u : DT == SK_BF16 ? 0xff80u : 0xfc00u;
    const int32_t at = wave_at + 8 * lane;
    uint32_t e[8];
    if (SHORT && vocab < 8) {
      first = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const char *p = row + min(k, vocab - 1) * S;
        e[k] = DT == SK_F32 ? *(const uint32_t SK_GLOBAL *)(uintptr_t)p : load_u16(p);
        e[k] = at == 0 && k < vocab ? e[k] : lowest;
      }
      pack(e);
      return;
    }
    first = min(at, vocab - 8);
#pragma unroll
    for (int i = 0; i < S / 2; ++i) raw[i] = *(const u32x4_any SK_GLOBAL *)(uintptr_t)(row + (int64_t)first * S + 16 * i);
  }
  // Behind all loads: -infinity for what belongs to other lanes.
  __device__ __forceinline__ void cut(int32_t wave_at, int lane, int32_t vocab) {
    if (wave_at + 512 <= vocab || vocab < 8) return;  // (the same in all lanes)
    constexpr uint32_t lowest = DT == SK_F32 ? 0xff800000u : DT == SK_BF16 ? 0xff80u : 0xfc00u;
    const int32_t others = wave_at + 8 * lane - first;
    uint32_t e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      e[k] = DT == SK_F32 ? raw[S == 4 ? k / 4 : 0][k % 4] : (k & 1 ? raw[0][k / 2] >> 16 : raw[0][k / 2] & 0xffffu);
      e[k] = k < others ? lowest : e[k];
    }
    pack(e);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    if constexpr (DT == SK_F32) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __builtin_bit_cast(float, (uint32_t)raw[k / 4][k % 4]);
    } else {
      unpack8<DT>(raw[0], x);
    }
  }

 private:
  __device__ __forceinline__ void pack(const uint32_t (&e)[8]) {
    if constexpr (DT == SK_F32) raw[0] = u32x4{e[0], e[1], e[2], e[3]}, raw[1] = u32x4{e[4], e[5], e[6], e[7]};
    else raw[0] = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
  }
};

struct VerifyShared {
  double begin, bound, piece[VERIFY_PIECES];
  int32_t chunk, found;
};

__device__ __forceinline__ int32_t first_of(const SK_CONSTANT VerifyDev &P, int32_t s) { return min(max(load_i32(P.first_row + s), 0), P.rows); }

// The sequence that a row belongs to; none: rows of no sequence, and of sequences whose numbers of rows make no sense.
struct Owner {
  int32_t seq, begin, end;
};
__device__ __forceinline__ Owner owner_of(const SK_CONSTANT VerifyDev &P, int32_t row, int lane) {
  Owner o;
  if (P.sequences <= 64) {  // a sequence a lane
    const int32_t s = min(lane, P.sequences - 1), begin = first_of(P, s), end = first_of(P, s + 1);
    o.seq = max(1, (int32_t)__popcll(__ballot(lane < P.sequences && begin <= row))) - 1;
    o.begin = lane_of(begin, o.seq), o.end = lane_of(end, o.seq);
  } else {
    o.seq = __builtin_amdgcn_readfirstlane(last_not_above(P.first_row, P.sequences, row, lane));
    o.begin = first_of(P, o.seq), o.end = first_of(P, o.seq + 1);
  }
  return o;
}

// A chunk of a row, 512 * PIECES logits, by a wave: a lane has eight of each piece, takes them relative to its own largest, and the lanes are joined at
// the end.  Bound by the vector unit (19 to 20 instructions a logit, half of its time) about as much as by memory: rows of 128000 and
// 50257, 29 million 16-bit logits in all, in 23 us (2.5 TB/s), 102 MB of 32-bit logits in 23 us (4.5 TB/s).
template <int DT, int PIECES>
__device__ __forceinline__ void chunk_stat(const SK_CONSTANT VerifyDev &P, const char *from, int32_t chunk, double c, VerifyStat *out, int lane) {
  Eight<DT> raw[PIECES];
  const int32_t at0 = chunk * 512 * PIECES;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) raw[i].template load<PIECES == 1>(from, at0 + i * 512, lane, P.vocab);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) raw[i].cut(at0 + i * 512, lane, P.vocab);
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    float x[8];
    raw[i].get(x);
#pragma unroll
    for (int k = 0; k < 8; ++k) top = __builtin_elementwise_maximum(top, x[k]);  // (a NaN, once there, stays)
  }
  VerifyStat r{0.0, wave_max(top), 0x7fffffff};
  if (__ballot(!(top < __builtin_inff()))) {
    r.sum = __builtin_nan("");
  } else if (greedy(c)) {
    r.sum = 1.0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float x[8];
      raw[i].get(x);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (x[k] == r.top) r.at = min(r.at, raw[i].first + k);
    }
    r.at = wave_min(r.at);
  } else if (r.top > -__builtin_inff()) {
    const double m = (double)fmaxf(top, -3.402823466e+38f);  // (a lane may have nothing but -infinity: the lowest number is not above any other top)
    const double lowest = -990.0 / c;  // what is further below counts as this, for 10^-298
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float x[8];
      raw[i].get(x);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);  // (four at a time: more would take the registers of waves)
        sum += exp2_of(fmax((double)x[k] - m, lowest), c);
      }
    }
    r.sum = wave_sum(top > -__builtin_inff() ? sum * weight_of(m - (double)r.top, c) : 0.0);
  }
  if (lane == 0) *out = r;
}

template <int DT>
__device__ __forceinline__ void row_chunk(const SK_CONSTANT VerifyDev &P, uint32_t unit, int lane) {
  const uint32_t sides = P.draft_logits ? 2 : 1, line = unit / (uint32_t)P.chunks;
  const int32_t chunk = (int32_t)(unit - line * (uint32_t)P.chunks), row = (int32_t)(line / sides);
  const bool draft = sides == 2 && (line & 1);
  if (row >= P.rows) return;
  const Owner o = owner_of(P, row, lane);
  if (row < o.begin || row >= o.end) return;
  const double c = scale_of(P, o.seq);
  if (draft && (row == o.end - 1 || greedy(c))) return;
  const char *from = draft ? P.draft_logits + row * P.draft_stride : P.logits + row * P.logits_stride;
  VerifyStat *out = P.stats + ((int64_t)row * 2 + draft) * P.chunks + chunk;
  if (P.pieces == 1) chunk_stat<DT, 1>(P, from, chunk, c, out, lane);
  else if (P.pieces == 2) chunk_stat<DT, 2>(P, from, chunk, c, out, lane);
  else chunk_stat<DT, VERIFY_PIECES>(P, from, chunk, c, out, lane);
}

__global__ void __launch_bounds__(CACHE_THREADS, 8) sk_verify_stats(VerifyArgs a) {
  const SK_CONSTANT VerifyTable &table = *(const SK_CONSTANT VerifyTable *)(uintptr_t)a.table;
  int i = 0;
  uint32_t first = 0;
  if (a.n > 1) {
#pragma unroll
    for (int k = 1; k < VERIFY_PROBLEMS; ++k) i += table.stat_first[k] <= blockIdx.x ? 1 : 0;
    first = table.stat_first[i];
  }
  const SK_CONSTANT VerifyDev &P = table.problems[i];
  const uint32_t unit = (blockIdx.x - first) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (P.dtype == SK_F32) row_chunk<SK_F32>(P, unit, lane);
  else if (P.dtype == SK_BF16) row_chunk<SK_BF16>(P, unit, lane);
  else row_chunk<SK_F16>(P, unit, lane);
}

// A row's distribution from its chunks, by a wave: p(k) = 2^((l_k - top) * c) / sum.  sum 0: it has none.
struct Row {
  double top, sum;
  int32_t at;  // (temperature 0) the only token
};
__device__ __forceinline__ VerifyStat stat_of(const VerifyStat *stats, int32_t chunks, int32_t i) {
  return i < chunks ? stats[i] : VerifyStat{0.0, -__builtin_inff(), 0x7fffffff};
}
// own: this lane's chunk of the first 64.
__device__ __forceinline__ Row row_stat(const VerifyStat &own, const VerifyStat *stats, int32_t chunks, double c, int lane) {
  float top = own.top;
  bool bad = own.sum != own.sum;
  for (int32_t i = 64 + lane; i < chunks; i += 64) {
    top = fmaxf(top, stats[i].top);
    bad |= stats[i].sum != stats[i].sum;
  }
  top = wave_max(top);
  Row r{(double)top, 0.0, -1};
  if (__ballot(bad) || !(top > -__builtin_inff())) return r;
  int32_t at = 0x7fffffff;
  auto add = [&](const VerifyStat &s) {
    r.sum += s.top > -__builtin_inff() ? s.sum * weight_of((double)s.top - r.top, c) : 0.0;
    if (s.top == top) at = min(at, s.at);
  };
  add(own);
  for (int32_t i = 64 + lane; i < chunks; i += 64) add(stats[i]);
  r.sum = wave_sum(r.sum);
  r.at = greedy(c) ? wave_min(at) : -1;
  return r;
}

// What the sampled token of a sequence is drawn from.
enum { FROM_NOTHING, FROM_ONE, FROM_TARGET, FROM_OTHERS, FROM_DIFFERENCE };
struct Draw {
  int32_t stop, mode, token;  // row within the sequence; FROM_OTHERS: all but this token
  Row p, q;
};

// max(p / p_sum - q / q_sum, 0), times both sums.  Two rounded products: where p and q are the same, so are they, and nothing is left.
__device__ __forceinline__ double difference(double p, double q_sum, double q, double p_sum) {
#pragma clang fp contract(off)
  const double a = p * q_sum, b = q * p_sum;
  return fmax(a - b, 0.0);
}

// Weights of eight tokens.
template <int DT>
__device__ __forceinline__ void weights8(const Draw &d, const Eight<DT> &p, const Eight<DT> &q, double c, double (&w)[8]) {
  float x[8], y[8];
  p.get(x);
  q.get(y);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    w[k] = weight_of((double)x[k] - d.p.top, c);
    if (d.mode == FROM_DIFFERENCE) w[k] = difference(w[k], d.q.sum, weight_of((double)y[k] - d.q.top, c), d.p.sum);
    if (d.mode == FROM_OTHERS && p.first + k == d.token) w[k] = 0.0;
  }
}

// The weights of a chunk, by a workgroup: a wave has a piece, whose sum goes to LDS.  Returns the chunk's sum.
template <int DT>
__device__ __forceinline__ double chunk_weights(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, int32_t chunk, double c, double (&w)[8], int32_t &place,
                                                VerifyShared &s, int tid) {
  static_assert(VERIFY_PIECES == CACHE_THREADS / 64, "a piece a wave");
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t at = wave < P.pieces ? (chunk * P.pieces + wave) * 512 : P.vocab;
  double sum = 0.0;
  place = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = 0.0;
  if (at < P.vocab) {  // (the same in all lanes)
    Eight<DT> p, q;
    p.template load<true>(p_row, at, lane, P.vocab);
    q.template load<true>(q_row, at, lane, P.vocab);
    p.cut(at, lane, P.vocab);
    q.cut(at, lane, P.vocab);
    weights8<DT>(d, p, q, c, w);
    place = p.first;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += w[k];
    sum = wave_sum(sum);
  }
  if (lane == 0) s.piece[wave] = sum;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < VERIFY_PIECES; ++i) all += s.piece[i];
  return all;
}

// The sum of a chunk's weights, by a wave, in all lanes.
template <int DT>
__device__ __forceinline__ double chunk_sum(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, int32_t chunk, double c, int lane) {
  Eight<DT> p, q, p_next, q_next;
  int32_t at = chunk * 512 * P.pieces;
  p.template load<true>(p_row, at, lane, P.vocab);
  q.template load<true>(q_row, at, lane, P.vocab);
  double sum = 0.0;
  for (int32_t i = 0; i < P.pieces && at < P.vocab; ++i, at += 512) {
    p_next.template load<true>(p_row, at + 512, lane, P.vocab);  // (behind the chunk: not used)
    q_next.template load<true>(q_row, at + 512, lane, P.vocab);
    p.cut(at, lane, P.vocab);
    q.cut(at, lane, P.vocab);
    double w[8];
    weights8<DT>(d, p, q, c, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += w[k];
    p = p_next, q = q_next;
  }
  return wave_sum(sum);
}

// The first token whose weight and those before it add up to more than `random` times all, by a workgroup.  sum_of(i) is the sum of chunk i (asked for
// by the first wave).  -1: all weights are 0.
template <int DT, class F>
__device__ __forceinline__ int32_t pick(const SK_CONSTANT VerifyDev &P, const Draw &d, const char *p_row, const char *q_row, double c, double random, F sum_of, VerifyShared &s, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __syncthreads();
  if (wave == 0) {
    const double own = lane < P.chunks ? sum_of(lane) : 0.0;  // of the first 64 chunks
    auto value = [&](int32_t i0) { return i0 == 0 ? own : i0 + lane < P.chunks ? sum_of(i0 + lane) : 0.0; };
    double total = 0.0;
    int32_t last = -1;
    for (int32_t i0 = 0; i0 < P.chunks; i0 += 64) {
      const double v = value(i0);
      const uint64_t some = __ballot(v > 0.0);
      if (some) last = i0 + 63 - (int)__builtin_clzll(some);
      total = lane_of(total + wave_scan(v), 63);
    }
    const double bound = random * total;
    double begin = 0.0, all = 0.0;
    int32_t chunk = -1;
    for (int32_t i0 = 0; i0 < P.chunks && chunk < 0; i0 += 64) {
      const double v = value(i0), upto = all + wave_scan(v);
      const uint64_t past = __ballot(upto > bound && v > 0.0);
      if (past) {
        const int l = (int)__builtin_ctzll(past);
        chunk = i0 + l;
        begin = l ? lane_of(upto, l - 1) : all;
      }
      all = lane_of(upto, 63);
    }
    if (lane == 0) s.begin = begin, s.bound = chunk < 0 ? __builtin_inf() : bound, s.chunk = chunk < 0 ? last : chunk;  // (rounding: the last token with a weight)
  }
  __syncthreads();
  const double bound = s.bound;
  const int32_t chunk = s.chunk;
  if (chunk < 0) return -1;
  double mine[8];
  int32_t place;
  if (tid == 0) s.found = -1;
  chunk_weights<DT>(P, d, p_row, q_row, chunk, c, mine, place, s, tid);
  // the piece that passes the bound, or the last with a weight
  double begin = s.begin, at_begin = 0.0;
  int32_t piece = -1;
#pragma unroll
  for (int i = 0; i < VERIFY_PIECES; ++i) {
    const double sum = s.piece[i];
    if (sum > 0.0 && (piece < 0 || !(at_begin + s.piece[piece] > bound))) piece = i, at_begin = begin;
    begin += sum;
  }
  if (piece < 0) return -1;  // (not where the chunk has a weight)
  if (piece == wave) {
    double upto = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) upto += mine[k];
    const double scanned = wave_scan(upto);
    const uint32_t lo = (uint32_t)__builtin_bit_cast(uint64_t, scanned), hi = (uint32_t)(__builtin_bit_cast(uint64_t, scanned) >> 32);
    const uint64_t below = (uint64_t)(uint32_t)__shfl_up((int)hi, 1) << 32 | (uint32_t)__shfl_up((int)lo, 1);
    double sum = at_begin + (lane ? __builtin_bit_cast(double, below) : 0.0);
    int32_t found = 0x7fffffff, last = -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      sum += mine[k];
      if (mine[k] > 0.0) {
        if (sum > bound) found = min(found, place + k);
        last = place + k;
      }
    }
    found = wave_min(found);
    last = -wave_min(-last);
    if (lane == 0) s.found = found != 0x7fffffff ? found : last;
  }
  __syncthreads();
  return s.found;
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
      const bool judged = i < n - 1 && P.drafted, two = judged && P.draft_logits && !greedy(c);
      const int32_t token = judged ? load_i32(P.drafted + row) : -1;
      const double random = judged ? random_of(P.accept_random + row) : 0.0;
      const VerifyStat *p_stats = P.stats + row * 2 * P.chunks, *q_stats = p_stats + P.chunks;
      const VerifyStat p_own = stat_of(p_stats, P.chunks, lane), q_own = stat_of(q_stats, two ? P.chunks : 0, lane);
      const bool known = token >= 0 && token < P.vocab;
      constexpr int S = DT == SK_F32 ? 4 : 2;
      const double p_logit = known ? (double)load1<DT>(P.logits + row * P.logits_stride + (int64_t)token * S) : 0.0;
      const double q_logit = known && two ? (double)load1<DT>(P.draft_logits + row * P.draft_stride + (int64_t)token * S) : 0.0;
      Draw d{};
      d.stop = i, d.token = -1;
      d.p = row_stat(p_own, p_stats, P.chunks, c, lane);
      bool accept = false;
      if (!(d.p.sum > 0.0)) {
        d.mode = FROM_NOTHING;
      } else {
        d.mode = greedy(c) ? FROM_ONE : FROM_TARGET;
        if (known) {
          double q = 1.0;
          bool certain = !two;
          if (two) {
            d.q = row_stat(q_own, q_stats, P.chunks, c, lane);
            certain = !(d.q.sum > 0.0);
            if (!certain) q = weight_of(q_logit - d.q.top, c) / d.q.sum;
          }
          const double p = greedy(c) ? (token == d.p.at ? 1.0 : 0.0) : weight_of(p_logit - d.p.top, c) / d.p.sum;
          accept = random * q < p;
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
__device__ __forceinline__ void sample(const SK_CONSTANT VerifyDev &P, int32_t seq, int32_t part, VerifyShared &s, Draw *draws, int32_t *stop, uint32_t *flag, int tid) {
  const int32_t r0 = first_of(P, seq), n = first_of(P, seq + 1) - r0;
  if (n <= 0) {
    if (part == 0 && tid == 0) P.accepted[seq] = 0;
    return;
  }
  const double c = scale_of(P, seq);
  Draw d;
  decide<DT>(P, r0, n, c, draws, stop, tid, d);
  const char *p_row = P.logits + (int64_t)(r0 + d.stop) * P.logits_stride, *q_row = d.mode == FROM_DIFFERENCE ? P.draft_logits + (int64_t)(r0 + d.stop) * P.draft_stride : p_row;
  const double random = random_of(P.sample_random + seq);
  const VerifyStat *stats = P.stats + (int64_t)(r0 + d.stop) * 2 * P.chunks;
  auto from_stats = [&](int32_t i) { return stats[i].top > -__builtin_inff() ? stats[i].sum * weight_of((double)stats[i].top - d.p.top, c) : 0.0; };
  int32_t token = -1;
  double w[8];
  int32_t place;
  if (d.mode == FROM_DIFFERENCE) {  // a chunk a wave
    double *sums = P.sums + (int64_t)seq * P.chunks;
    const int32_t chunk = part * VERIFY_CHUNKS + __builtin_amdgcn_readfirstlane(tid >> 6);
    if (chunk < P.chunks) {
      const double sum = chunk_sum<DT>(P, d, p_row, q_row, chunk, c, tid & 63);
      if ((tid & 63) == 0) put(sums + chunk, sum);
    }
    if (!last_to_arrive(P.arrived + (int64_t)seq * COUNTER_STEP, (P.chunks + VERIFY_CHUNKS - 1) / VERIFY_CHUNKS, flag)) return;
    token = pick<DT>(P, d, p_row, q_row, c, random, [&](int32_t i) { return got(sums + i); }, s, tid);
  } else if (part != 0) {
    return;
  } else if (d.mode == FROM_OTHERS) {
    const int32_t without = d.token / (512 * P.pieces);
    const double rest = chunk_weights<DT>(P, d, p_row, q_row, without, c, w, place, s, tid);
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

__global__ void __launch_bounds__(CACHE_THREADS, 4) sk_verify_sample(VerifyArgs a) {
  __shared__ VerifyShared shared;
  __shared__ Draw draws[4];
  __shared__ int32_t stop;
  __shared__ uint32_t flag;
  const int tid = threadIdx.x;
  const SK_CONSTANT VerifyTable &table = *(const SK_CONSTANT VerifyTable *)(uintptr_t)a.table;
  int i = 0;
  uint32_t first = 0;
  if (a.n > 1) {
#pragma unroll
    for (int k = 1; k < VERIFY_PROBLEMS; ++k) i += table.sum_first[k] <= blockIdx.x ? 1 : 0;
    first = table.sum_first[i];
  }
  const SK_CONSTANT VerifyDev &P = table.problems[i];
  const uint32_t unit = blockIdx.x - first;
  const uint32_t parts = ((uint32_t)P.chunks + VERIFY_CHUNKS - 1) / VERIFY_CHUNKS;
  const int32_t seq = (int32_t)(unit / parts), part = (int32_t)(unit % parts);
  if (P.dtype == SK_F32) sample<SK_F32>(P, seq, part, shared, draws, &stop, &flag, tid);
  else if (P.dtype == SK_BF16) sample<SK_BF16>(P, seq, part, shared, draws, &stop, &flag, tid);
  else sample<SK_F16>(P, seq, part, shared, draws, &stop, &flag, tid);
}

}  // namespace sk

struct sk_verify_plan : sk::PlanOnDevice {
  sk::VerifyPlanHost host;
};

namespace {

sk_status upload(sk_verify_plan &plan) {
  sk::VerifyPlanHost &h = plan.host;
  if (h.launches.empty()) return SK_OK;
  // tables, counters
  const size_t o_counters = sk::align_up(h.launches.size() * sizeof(sk::VerifyTable), 256);
  std::vector<char> image(o_counters + h.counters, 0);
  char *ws = nullptr;
  const sk_status st = sk::upload_image(plan, image, h.workspace, &ws);
  if (st != SK_OK) return st;
  auto moved = [](auto *&p, char *base) { p = (std::decay_t<decltype(p)>)(base + (uintptr_t)p); };
  for (size_t k = 0; k < h.launches.size(); ++k) {
    sk::VerifyTable table = h.launches[k].table;
    for (int32_t i = 0; i < h.launches[k].n; ++i) {
      sk::VerifyDev &d = table.problems[i];
      moved(d.arrived, plan.blob + o_counters), moved(d.stats, ws), moved(d.sums, ws);
    }
    std::memcpy(image.data() + k * sizeof(table), &table, sizeof(table));
  }
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
    if (st != SK_OK || plan->host.launches.empty()) return st;
    const hipEvent_t behind = in_capture ? nullptr : plan->last_use;
    sk::VerifyArgs args{(const sk::VerifyTable *)plan->blob, 0};
    for (const sk::VerifyLaunch &l : plan->host.launches) {
      args.n = l.n;
      if (st == SK_OK) st = sk::launch(sk::sk_verify_stats, l.stat_grid, stream, nullptr, args);
      if (st == SK_OK) st = sk::launch(sk::sk_verify_sample, l.sum_grid, stream, &l == &plan->host.launches.back() ? behind : nullptr, args);
      ++args.table;
    }
    plan->ledger.after_launch((uintptr_t)stream, in_capture, behind && st == SK_OK);  // also after a failure: some launches may be out
    return st;
  });
}

sk_status sk_verify_plan_info(const sk_verify_plan *plan, int32_t *launches, int64_t *workspace_bytes) {
  return sk::guarded([&]() -> sk_status {
    if (!plan) return sk::set_last_error(SK_ERR_INVALID_ARG, "plan is null");
    if (launches) *launches = 2 * (int32_t)plan->host.launches.size();
    if (workspace_bytes) *workspace_bytes = (int64_t)(plan->host.workspace + plan->host.counters);
    return SK_OK;
  });
}

}  // extern "C"
