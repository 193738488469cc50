// Device code that the operators of libsk_layer.so share: elements of any alignment, activations, sums over a wave.
#pragma once

#include "device.hip.h"

#include <type_traits>

#include "layer_internal.h"

namespace sk {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Eight elements at an address that is a multiple of the element's size (a global load of 16 bytes takes any), as fp32.
template <int DT, bool ONCE>
__device__ __forceinline__ void load8(const char *p, float (&x)[8]) {
  if constexpr (DT == SK_F32) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4_any SK_GLOBAL *q = (const f32x4_any SK_GLOBAL *)(uintptr_t)(p + 4 * i);
      const f32x4 v = ONCE ? (f32x4)__builtin_nontemporal_load(q) : (f32x4)*q;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i + j] = v[j];
    }
  } else {
    const u32x4_any SK_GLOBAL *q = (const u32x4_any SK_GLOBAL *)(uintptr_t)p;
    unpack8<DT>(ONCE ? (u32x4)__builtin_nontemporal_load(q) : (u32x4)*q, x);
  }
}
template <int DT>
__device__ __forceinline__ float load1(const char *p) {
  if constexpr (DT == SK_F32) return load_f((const float *)p);
  return elem<DT>(load_u16(p));
}
template <int DT, bool ONCE>
__device__ __forceinline__ void store8_elements(char *p, const float (&x)[8]) {
  if constexpr (DT == SK_F32) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      f32x4_any SK_GLOBAL *q = (f32x4_any SK_GLOBAL *)(uintptr_t)(p + 4 * i);
      const f32x4_any v = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
      if (ONCE) __builtin_nontemporal_store(v, q);
      else *q = v;
    }
  } else {
    u32x4_any SK_GLOBAL *q = (u32x4_any SK_GLOBAL *)(uintptr_t)p;
    const u32x4_any v = u32x4{pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7])};
    if (ONCE) __builtin_nontemporal_store(v, q);
    else *q = v;
  }
}
template <int DT>
__device__ __forceinline__ void store1(char *p, float x) {
  if constexpr (DT == SK_F32) *(float SK_GLOBAL *)(uintptr_t)p = x;
  else *(uint16_t SK_GLOBAL *)(uintptr_t)p = (uint16_t)(pack2<DT>(x, x) & 0xffffu);
}

// Values that another workgroup of the launch reads, maybe behind another L2: written through to memory, and read from there.
template <class T>
__device__ __forceinline__ void put(T *p, T v) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "");
  if constexpr (sizeof(T) == 4) __hip_atomic_store((uint32_t *)p, __builtin_bit_cast(uint32_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else __hip_atomic_store((unsigned long long *)p, __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T got(const T *p) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "");
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __hip_atomic_load((const uint32_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  else return __builtin_bit_cast(T, __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// ---- sums and maxima over a wave ----
template <int CTRL>
__device__ __forceinline__ double other_lane(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int32_t)(uint32_t)b, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int32_t)(b >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// (the sum of a lane's value and that of the lane 16 or 32 places away)
template <int D>
__device__ __forceinline__ void across(double v, double &a, double &b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, v);
  const uint32_t l = (uint32_t)x, h = (uint32_t)(x >> 32);
  const auto lo = D == 16 ? __builtin_amdgcn_permlane16_swap(l, l, false, false) : __builtin_amdgcn_permlane32_swap(l, l, false, false);
  const auto hi = D == 16 ? __builtin_amdgcn_permlane16_swap(h, h, false, false) : __builtin_amdgcn_permlane32_swap(h, h, false, false);
  const uint32_t l0 = lo[0], l1 = lo[1], h0 = hi[0], h1 = hi[1];
  a = __builtin_bit_cast(double, (uint64_t)h0 << 32 | l0);
  b = __builtin_bit_cast(double, (uint64_t)h1 << 32 | l1);
}
template <class F>
__device__ __forceinline__ double over_wave(double v, F f) {
  v = f(v, other_lane<0xb1>(v));
  v = f(v, other_lane<0x4e>(v));
  v = f(v, other_lane<0x141>(v));
  v = f(v, other_lane<0x140>(v));
  double a, b;
  across<16>(v, a, b);
  v = f(a, b);
  across<32>(v, a, b);
  return f(a, b);
}
__device__ __forceinline__ double wave_sum(double v) { return over_wave(v, [](double a, double b) { return a + b; }); }
__device__ __forceinline__ double wave_max(double v) { return over_wave(v, [](double a, double b) { return fmax(a, b); }); }

__device__ __forceinline__ float wave_sum(float v) { return sum32(sum_over(v, 32)); }
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, other_lane<0xb1>(v));
  v = fmaxf(v, other_lane<0x4e>(v));
  v = fmaxf(v, other_lane<0x141>(v));
  v = fmaxf(v, other_lane<0x140>(v));
  return max32(max16(v));
}
// (the same in all lanes)
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t lesser(int32_t v) {
  return min(v, __builtin_amdgcn_update_dpp(v, v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int32_t wave_min(int32_t v) {
  v = lesser<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v = lesser<0x112, 0xf>(v);
  v = lesser<0x114, 0xf>(v);
  v = lesser<0x118, 0xf>(v);
  v = lesser<0x142, 0xa>(v);  // row_bcast:15, 31
  v = lesser<0x143, 0xc>(v);
  return lane_of(v, 63);
}

// e^x to about 2 units of the last place: what x * log2(e) loses by rounding is put back.  Not to an infinity (from x = 88.8 on, where it would be a
// NaN if the rest is 0 or negative), and not a rest that is none itself.
__device__ __forceinline__ float exp_of(float x) {
  const float p = x * 1.44269504f, e = exp2_fast(p);
  const float rest = fmaf(x, 1.44269504f, -p) + x * 1.92596299e-8f, r = fmaf(e, 0.693147181f * rest, e);
  return __builtin_isfinite(r) ? r : e;
}
// One exponential whatever the activation: z/2 (1 + tanh(w)) = z / (1 + e^-2w), and tanh(z) = 2 / (1 + e^-2z) - 1, near 0 by its series.
// (e^-t overflows to infinity where it should; a NaN stays one.)
__device__ __forceinline__ float activated(int act, float z) {
  if (act == SK_ACT_NONE) return z;
  if (act == SK_ACT_RELU) return z < 0.f ? 0.f : z;
  const float t = act == SK_ACT_TANH ? 2.f * z : act == SK_ACT_GELU ? 1.5957691216f * (z + 0.044715f * z * z * z) : z;
  const float s = __builtin_amdgcn_rcpf(1.f + exp_of(-t));  // (to a unit of the last place; 0 of infinity)
  if (act == SK_ACT_SIGMOID) return s;
  if (act == SK_ACT_TANH) {
    const float q = z * z;  // |z| < 1/4: the next term is below 2^-25 of z
    const float series = z + z * q * (-0.333333333f + q * (0.133333333f + q * (-0.0539682540f + q * 0.0218694885f)));
    return fabsf(z) < 0.25f ? series : 2.f * s - 1.f;
  }
  return z * s;
}

}  // namespace sk
