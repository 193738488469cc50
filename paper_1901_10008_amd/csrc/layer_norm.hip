// Norms before and after a block, with its gate and scales: the kernel and its entry points.
#include "layer_host.h"
#include "layer_math.hip.h"

namespace sk {

// A row lives in the registers of T threads, P pieces of 8 elements each, from its loads to its stores.
//
//   u = N(block) w + b,  r = rs * residual + bs * u * act(gate),  next = N(r) w' + b'
//
// Each norm is one sum over the row, or two (the mean, then the squares of what lies beside it: nothing cancels).  All of a row's loads are on their
// way before the first sum.
template <int T>
struct RowSum {
  float (*red)[16];
  int wave, turn = 0;
  __device__ __forceinline__ float operator()(float v) {
    v = wave_sum(v);
    if constexpr (T > 64) {  // each sum of a row has a place of its own, so that one barrier is enough
      red[turn][wave] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < T / 64; ++w) v += red[turn][w];
      ++turn;
    }
    return v;
  }
};

template <int T, int P, bool ONCE, int DT, int RT>
__device__ __forceinline__ void norm_row(const NormDev &p, int64_t row, int t, float (*red)[16]) {
  constexpr int ES = DT == SK_F32 ? 4 : 2, RS = RT == SK_F32 ? 4 : 2;
  const int dim = p.dim;
  const float by = 1.f / (float)dim;
  RowSum<T> sum{red, t >> 6};
  float u[P][8], r[P][8], g[P][8];

  // pieces of 8 elements; the last one of a row may be shorter: only its elements are read and written
  auto load = [&](auto type, auto once, const void *base, int64_t at, float(&x)[8], float missing) {
    constexpr int D = decltype(type)::value;
    constexpr int S = D == SK_F32 ? 4 : 2;
    if (!base || at >= dim) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = base ? 0.f : missing;
      return;
    }
    const char *q = (const char *)base + at * S;
    if (at + 8 <= dim) {
      load8<D, decltype(once)::value>(q, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float v = load1<D>((const char *)base + min(at + k, (int64_t)dim - 1) * S);
        x[k] = at + k < dim ? v : 0.f;
      }
    }
  };
  auto store = [&](auto type, char *base, int64_t at, const float(&x)[8]) {
    constexpr int D = decltype(type)::value;
    constexpr int S = D == SK_F32 ? 4 : 2;
    if (at >= dim) return;
    char *q = base + at * S;
    if (at + 8 <= dim) {
      store8_elements<D, ONCE>(q, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (at + k < dim) store1<D>(q + k * S, x[k]);
    }
  };
  using Own = std::integral_constant<int, DT>;
  using Res = std::integral_constant<int, RT>;
  using Once = std::integral_constant<bool, ONCE>;
  using Again = std::integral_constant<bool, false>;

  const char *block = p.block ? (const char *)p.block + row * p.block_stride * ES : nullptr;
  const char *gate = p.gate ? (const char *)p.gate + row * p.gate_stride * ES : nullptr;
  constexpr bool LATE = T > 256;  // its threads have 128 registers each: gates are loaded when they are wanted
  auto load_gate = [&](int i, int64_t at) {
    if (p.gate_stride) load(Own{}, Once{}, gate, at, g[i], 1.f);
    else load(Own{}, Again{}, gate, at, g[i], 1.f);
  };
  const char *residual = p.residual ? (const char *)p.residual + row * p.residual_stride * RS : nullptr;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int64_t at = ((int64_t)i * T + t) * 8;
    if (i * T * 8 < dim) {
      load(Own{}, Once{}, block, at, u[i], 0.f);
      if (gate && !LATE) load_gate(i, at);
      load(Res{}, Once{}, residual, at, r[i], 0.f);
    }
  }

  // x becomes (x - mean) * scale, or x * scale
  auto standard = [&](float(&x)[P][8]) {
    float s = 0.f;
    if (p.kind == SK_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i * T * 8 < dim) {
#pragma unroll
          for (int k = 0; k < 8; ++k) s += x[i][k];
        }
      const float mean = sum(s) * by;
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i * T * 8 < dim) {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[i][k] = (i * T + t) * 8 + k < dim ? x[i][k] - mean : 0.f;
        }
    }
    s = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (i * T * 8 < dim) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[i][k] * x[i][k];
      }
    return 1.f / sqrtf(sum(s) * by + p.eps);
  };

  if (block) {
    if (p.post) {
      const float scale = standard(u);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i * T * 8 < dim) {
          const int64_t at = ((int64_t)i * T + t) * 8;
          float w[8], b[8];
          load(Own{}, Again{}, p.post_weight, at, w, 1.f);
          load(Own{}, Again{}, p.post_bias, at, b, 0.f);
#pragma unroll
          for (int k = 0; k < 8; ++k) u[i][k] = u[i][k] * scale * w[k] + b[k];
        }
    }
    if (gate) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i * T * 8 < dim) {
          if (LATE) load_gate(i, ((int64_t)i * T + t) * 8);
#pragma unroll
          for (int k = 0; k < 8; ++k) u[i][k] *= activated(p.act, g[i][k]);
        }
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (i * T * 8 < dim) {
      // (a missing part adds nothing, not its scale times 0)
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] = !block ? p.residual_scale * r[i][k] : !residual ? p.block_scale * u[i][k] : p.residual_scale * r[i][k] + p.block_scale * u[i][k];
      if (p.residual_out) store(Res{}, (char *)p.residual_out + row * p.residual_out_stride * RS, ((int64_t)i * T + t) * 8, r[i]);
    }
  if (!p.next) return;
  const float scale = standard(r);
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (i * T * 8 < dim) {
      const int64_t at = ((int64_t)i * T + t) * 8;
      float w[8], b[8];
      load(Own{}, Again{}, p.pre_weight, at, w, 1.f);
      load(Own{}, Again{}, p.pre_bias, at, b, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = r[i][k] * scale * w[k] + b[k];
      store(Own{}, (char *)p.next + row * p.next_stride * ES, at, w);
    }
}

template <int T, int P, bool ONCE>
__global__ void __launch_bounds__(T > CACHE_THREADS ? T : CACHE_THREADS) sk_norm(NormArgs a) {
  __shared__ float red[4][16];
  int i = 0;
#pragma unroll
  for (int k = 1; k < NORM_PROBLEMS; ++k) i += a.first[k] <= blockIdx.x ? 1 : 0;
  const NormDev &p = a.problems[i];
  const int64_t n = p.n_rows ? min(load_i32(p.n_rows), p.rows) : p.rows;
  const int t = (int)threadIdx.x % T;
  int64_t row = (int64_t)(blockIdx.x - a.first[i]);
  if constexpr (T == 64) row = row * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  if (row >= n) return;
  if (p.dtype == SK_F32) norm_row<T, P, ONCE, SK_F32, SK_F32>(p, row, t, red);
  else if (p.dtype == SK_BF16 && p.residual_dtype == SK_BF16) norm_row<T, P, ONCE, SK_BF16, SK_BF16>(p, row, t, red);
  else if (p.dtype == SK_BF16) norm_row<T, P, ONCE, SK_BF16, SK_F32>(p, row, t, red);
  else if (p.residual_dtype == SK_F16) norm_row<T, P, ONCE, SK_F16, SK_F16>(p, row, t, red);
  else norm_row<T, P, ONCE, SK_F16, SK_F32>(p, row, t, red);
}

}  // namespace sk

struct sk_norm_plan : sk::PlanOnDevice {
  sk::NormPlanHost host;
  bool launched = false;
};

namespace {

void (*norm_kernel(sk::NormForm form, bool once))(sk::NormArgs) {
  switch (form) {
    case sk::NORM_WAVE: return once ? sk::sk_norm<64, 4, true> : sk::sk_norm<64, 4, false>;
    case sk::NORM_GROUP: return once ? sk::sk_norm<256, 4, true> : sk::sk_norm<256, 4, false>;
    default: return once ? sk::sk_norm<1024, 4, true> : sk::sk_norm<1024, 4, false>;
  }
}

}  // namespace

extern "C" {

void sk_layer_params_default(sk_layer_params *params) {
  if (params) *params = sk_layer_params{};
}

sk_status sk_norm_plan_create(const sk_norm_problem *problems, int32_t n, const sk_layer_params *params, sk_norm_plan **out) {
  return sk::create_plan<sk_norm_plan>(params, out, [&](sk_norm_plan &plan, int32_t, int32_t, std::string &err) { return sk::plan_norm(problems, n, plan.host, err); },
                                       [](sk_norm_plan &) { return SK_OK; });
}

sk_status sk_norm_plan_destroy(sk_norm_plan *plan) {
  if (!plan) return SK_OK;
  return sk::guarded([&]() -> sk_status { return sk::destroy_plan(plan, plan->launched); });
}

sk_status sk_norm_launch(sk_norm_plan *plan, void *hip_stream) {
  return sk::guarded([&]() -> sk_status {
    sk_status st = sk::check_resident(plan);
    if (st != SK_OK) return st;
    for (const sk::NormLaunch &l : plan->host.launches) {
      if (st != SK_OK) break;
      st = sk::launch(norm_kernel(l.form, l.once), l.grid, (hipStream_t)hip_stream, nullptr, l.args, l.form == sk::NORM_LONG ? sk::NORM_LONG_THREADS : sk::CACHE_THREADS);
      plan->launched = true;
    }
    return st;
  });
}

}  // extern "C"
