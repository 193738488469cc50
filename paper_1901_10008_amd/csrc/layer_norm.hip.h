// Device code of norms before and after a block, with its gate and scales.
#pragma once

#include "layer_math.hip.h"

namespace sk {

// A row lives in the registers of T threads, P pieces of 8 elements each, from its loads to its stores.
//
//   u = N(block) w + b,  r = rs * residual + bs * u * act(gate),  next = N(r) w' + b'
//
// Each norm is one sum over the row, or two (the mean, then the squares of what lies beside it: nothing cancels).  All of a row's loads, those of the
// weights among them, are on their way before the number of rows is known and before the first sum.  Bound by memory where there is much (16000 rows of 4096
// elements, bf16 beside a stream of 32 bits: 786 MB in 134 us, 5.9 TB/s), by that chain where there is little (64 rows of each of four widths 7.2 us, three
// rows 3.3); rows of a few hundred to two thousand elements by the latency of their sums and by the vector unit (5003 of 1283 with both norms, biases and a
// gate: 25.7 us, 2 TB/s).
struct NormArgs {
  const NormTable *table;
  int32_t n;
};
// The sum over the T threads of a row.
template <int T>
struct RowSum {
  float (*red)[16];
  int wave, turn = 0;
  __device__ __forceinline__ float operator()(float v) {
    if constexpr (T < 64) return sum_over(v, T);
    v = wave_sum(v);
    if constexpr (T > 64) {  // neighbouring sums have places of their own, so that one barrier each is enough
      red[turn & 3][wave] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < T / 64; ++w) v += red[turn & 3][w];
      ++turn;
    }
    return v;
  }
};

template <int T, int P, bool ONCE, int DT, int RT>
__device__ __forceinline__ void norm_rows(const SK_CONSTANT NormDev &p, int64_t row, int t, float (*red)[16]) {
  constexpr int ES = DT == SK_F32 ? 4 : 2, RS = RT == SK_F32 ? 4 : 2;
  constexpr bool LATE = T > 512 || DT == SK_F32;  // gates and weights are loaded when they are wanted: there are not the registers to keep them
  const int dim = p.dim;
  const float by = 1.f / (float)dim;
  const int wave_at = T >= 64 ? __builtin_amdgcn_readfirstlane(t & ~63) : 0;
  RowSum<T> sum{red, wave_at >> 6};
  using Own = std::integral_constant<int, DT>;
  using Res = std::integral_constant<int, RT>;

  // pieces of 8 elements as they come; the last one of a row may be shorter: only its elements are read and written
  auto load = [&](auto type, bool once, const void *base, int i, u32x4 *raw) {
    constexpr int D = decltype(type)::value, S = D == SK_F32 ? 4 : 2;
    const int at = (i * T + t) * 8;
    const char *q = (const char *)base + (int64_t)at * S;
    if (at + 8 <= dim) {
#pragma unroll
      for (int j = 0; j < S / 2; ++j) {
        const u32x4_any SK_GLOBAL *g = (const u32x4_any SK_GLOBAL *)(uintptr_t)(q + 16 * j);
        raw[j] = ONCE && once ? (u32x4)__builtin_nontemporal_load(g) : (u32x4)*g;
      }
    } else if (at < dim) {
      uint32_t e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const char *g = (const char *)base + (int64_t)min(at + k, dim - 1) * S;
        e[k] = S == 4 ? *(const uint32_t SK_GLOBAL *)(uintptr_t)g : load_u16(g);
        e[k] = at + k < dim ? e[k] : 0u;
      }
      if constexpr (S == 4) raw[0] = u32x4{e[0], e[1], e[2], e[3]}, raw[1] = u32x4{e[4], e[5], e[6], e[7]};
      else raw[0] = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
    } else {
#pragma unroll
      for (int j = 0; j < S / 2; ++j) raw[j] = u32x4{0, 0, 0, 0};
    }
  };
  auto values = [&](auto type, const u32x4 *raw, float(&x)[8]) {
    constexpr int D = decltype(type)::value;
    if constexpr (D == SK_F32) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __builtin_bit_cast(float, (uint32_t)raw[k / 4][k % 4]);
    } else {
      unpack8<D>(raw[0], x);
    }
  };
  auto store = [&](auto type, char *base, int i, const float(&x)[8]) {
    constexpr int D = decltype(type)::value, S = D == SK_F32 ? 4 : 2;
    const int at = (i * T + t) * 8;
    if (at >= dim) return;
    char *q = base + (int64_t)at * S;
    if (at + 8 <= dim) {
      store8_elements<D, ONCE>(q, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (at + k < dim) store1<D>(q + k * S, x[k]);
    }
  };
  auto each_piece = [&](auto f) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if ((i * T + wave_at) * 8 < dim) f(i);  // (the same in all lanes: what a wave has nothing of costs it nothing)
  };

  auto behind_is_zero = [&](int i, float(&x)[8]) {  // (a branch: most waves have nothing there)
    const int at = (i * T + t) * 8;
    if (at + 8 > dim) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = at + k < dim ? x[k] : 0.f;
    }
  };

  const bool has_block = p.block != nullptr, has_gate = p.gate != nullptr, has_residual = p.residual != nullptr;
  const bool post = has_block && p.post, post_weight = post && p.post_weight, pre_weight = p.next && p.pre_weight;
  struct Raw {
    u32x4 block[P][ES / 2], gate[P][ES / 2], residual[P][RS / 2];
  };
  auto gate_of = [&](int64_t row) { return (const char *)p.gate + row * p.gate_stride * ES; };
  auto load_row = [&](int64_t row, Raw &to) {
    each_piece([&](int i) {
      if (has_block) load(Own{}, true, (const char *)p.block + row * p.block_stride * ES, i, to.block[i]);
      if (has_residual) load(Res{}, true, (const char *)p.residual + row * p.residual_stride * RS, i, to.residual[i]);
      if (!LATE && has_gate) load(Own{}, p.gate_stride != 0, gate_of(row), i, to.gate[i]);
    });
  };
  Raw now;
  u32x4 post_raw[P][ES / 2], pre_raw[P][ES / 2];
  load_row(row, now);
  if (!LATE) {
    each_piece([&](int i) {
      if (post_weight) load(Own{}, false, p.post_weight, i, post_raw[i]);
      if (pre_weight) load(Own{}, false, p.pre_weight, i, pre_raw[i]);
    });
  }
  const int64_t rows = p.n_rows ? min(load_i32(p.n_rows), p.rows) : p.rows;

  // x becomes x - mean, and what it is to be multiplied by is returned
  auto standard = [&](float(&x)[P][8]) {
    float s = 0.f;
    if (p.kind == SK_NORM_LAYER) {
      each_piece([&](int i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[i][k];
      });
      const float mean = sum(s) * by;
      each_piece([&](int i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[i][k] -= mean;
        behind_is_zero(i, x[i]);
      });
    }
    s = 0.f;
    each_piece([&](int i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s += x[i][k] * x[i][k];
    });
    return 1.f / sqrtf(sum(s) * by + p.eps);
  };
  // y = x * scale * weight + bias
  auto weighted = [&](int i, const float(&x)[8], float scale, const void *weight, u32x4 *raw, const void *bias, float(&y)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = x[k] * scale;
    if (weight) {
      float w[8];
      if (LATE) load(Own{}, false, weight, i, raw);
      values(Own{}, raw, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] *= w[k];
    }
    if (bias) {
      float b[8];
      u32x4 bias_raw[ES / 2];
      load(Own{}, false, bias, i, bias_raw);
      values(Own{}, bias_raw, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] += b[k];
    }
  };

  if (row >= rows) return;
  float u[P][8], r[P][8];
  if (has_block) {
    each_piece([&](int i) { values(Own{}, now.block[i], u[i]); });
    const float scale = post ? standard(u) : 1.f;
    each_piece([&](int i) {
      if (post) weighted(i, u[i], scale, p.post_weight, post_raw[i], p.post_bias, u[i]);
    });
    auto gated = [&](auto act) {
      each_piece([&](int i) {
        float g[8];
        if (LATE) load(Own{}, p.gate_stride != 0, gate_of(row), i, now.gate[i]);
        values(Own{}, now.gate[i], g);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[i][k] *= activated(decltype(act)::value, g[k]);
      });
    };
    if (has_gate) {
      switch (p.act) {
        case SK_ACT_SIGMOID: gated(std::integral_constant<int, SK_ACT_SIGMOID>{}); break;
        case SK_ACT_SILU: gated(std::integral_constant<int, SK_ACT_SILU>{}); break;
        case SK_ACT_TANH: gated(std::integral_constant<int, SK_ACT_TANH>{}); break;
        case SK_ACT_GELU: gated(std::integral_constant<int, SK_ACT_GELU>{}); break;
        case SK_ACT_RELU: gated(std::integral_constant<int, SK_ACT_RELU>{}); break;
        default: gated(std::integral_constant<int, SK_ACT_NONE>{});
      }
    }
  }
  each_piece([&](int i) {
    // (a missing part adds nothing, not its scale times 0)
    if (has_residual) values(Res{}, now.residual[i], r[i]);
    if (!has_block) {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] *= p.residual_scale;
    } else if (!has_residual) {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] = p.block_scale * u[i][k];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] = p.residual_scale * r[i][k] + p.block_scale * u[i][k];
    }
    if (p.post_bias) behind_is_zero(i, r[i]);  // (a bias stands there as well)
    if (p.residual_out) store(Res{}, (char *)p.residual_out + row * p.residual_out_stride * RS, i, r[i]);
  });
  if (p.next) {
    const float scale = standard(r);
    each_piece([&](int i) {
      float y[8];
      weighted(i, r[i], scale, p.pre_weight, pre_raw[i], p.pre_bias, y);
      store(Own{}, (char *)p.next + row * p.next_stride * ES, i, y);
    });
  }
}

template <int T, int P, bool ONCE>
__global__ void __launch_bounds__(T < 128 ? CACHE_THREADS : T) sk_norm(NormArgs a) {
  __shared__ float red[4][16];
  const SK_CONSTANT NormTable &table = *(const SK_CONSTANT NormTable *)(uintptr_t)a.table;
  int i = 0;
  uint32_t first = 0;
  if (a.n > 1) {
#pragma unroll
    for (int k = 1; k < NORM_PROBLEMS; ++k) i += table.first[k] <= blockIdx.x ? 1 : 0;
    first = table.first[i];
  }
  const SK_CONSTANT NormDev &p = table.problems[i];
  constexpr int ROWS = T < 128 ? CACHE_THREADS / T : 1;  // of a workgroup
  const int t = (int)threadIdx.x % T, part = T >= 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : (int)threadIdx.x / T;
  const int64_t row = (int64_t)(blockIdx.x - first) * ROWS + part;
  if (row >= p.rows) return;
  if (p.dtype == SK_F32) norm_rows<T, P, ONCE, SK_F32, SK_F32>(p, row, t, red);
  else if (p.dtype == SK_BF16 && p.residual_dtype == SK_BF16) norm_rows<T, P, ONCE, SK_BF16, SK_BF16>(p, row, t, red);
  else if (p.dtype == SK_BF16) norm_rows<T, P, ONCE, SK_BF16, SK_F32>(p, row, t, red);
  else if (p.residual_dtype == SK_F16) norm_rows<T, P, ONCE, SK_F16, SK_F16>(p, row, t, red);
  else norm_rows<T, P, ONCE, SK_F16, SK_F32>(p, row, t, red);
}

}  // namespace sk
