// Device code that the libraries of decoder steps share (gfx950 / CDNA4 only): types, loads and stores, rounding, matrix instructions,
// sums over lanes, partial results handed from workgroup to workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sk_internal.h"

#if defined(__HIP_DEVICE_COMPILE__) && !defined(__gfx950__)
#error "written for gfx950"
#endif

namespace sk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// (pointers out of descriptors: said to be global, so that loads are not flat ones)
#define SK_GLOBAL __attribute__((address_space(1)))
__device__ __forceinline__ u32x4 load16(const void *p) { return *(const u32x4 SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ int32_t load_i32(const int32_t *p) { return *(const int32_t SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ void store16(void *p, u32x4 v) { *(u32x4 SK_GLOBAL *)(uintptr_t)p = v; }
__device__ __forceinline__ void store8(void *p, u32x2 v) { *(u32x2 SK_GLOBAL *)(uintptr_t)p = v; }

// What a lane reads that must count as zeros: its address is replaced, so that no load stands under a branch.
__device__ __attribute__((aligned(16))) const uint32_t g_zeros[4] = {0u, 0u, 0u, 0u};

template <int DT>
__device__ __forceinline__ float elem(uint32_t bits) {
  if constexpr (DT == SK_BF16) return __builtin_bit_cast(float, bits << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <int DT>
__device__ __forceinline__ void unpack8(const u32x4 &v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = elem<DT>(v[i] & 0xffffu);
    x[2 * i + 1] = elem<DT>(v[i] >> 16);
  }
}
// Two values rounded to nearest even, the first in the low half.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  if constexpr (DT == SK_BF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  }
}
template <int DT>
__device__ __forceinline__ void mma16(const u32x4 &a, const u32x4 &b, f32x4 &c) {
  if constexpr (DT == SK_BF16)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ void mma32(const u32x4 &a, const u32x4 &b, f32x16 &c) {
  if constexpr (DT == SK_BF16)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// The transposing LDS read: each group of 16 lanes reads four rows of 16 16-bit elements, lane i of the group elements
// 4 (i % 4) .. + 3 of row i / 4, and gets column i: four elements, one per row.
__device__ __forceinline__ u32x2 read_transposed(const unsigned char *p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(unsigned char *)p));
}
// What nothing writes while the kernel runs, read through the scalar cache (its address the same in all lanes).
#define SK_CONSTANT __attribute__((address_space(4)))
// Sum over the lanes up to this one, in the vector unit: within rows of 16, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t shifted(int32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t shifted(int64_t v) {
  const uint32_t lo = (uint32_t)shifted<CTRL, ROWS>((int32_t)v), hi = (uint32_t)shifted<CTRL, ROWS>((int32_t)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double v) {
  return __builtin_bit_cast(double, shifted<CTRL, ROWS>(__builtin_bit_cast(int64_t, v)));
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
  v += shifted<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v += shifted<0x112, 0xf>(v);
  v += shifted<0x114, 0xf>(v);
  v += shifted<0x118, 0xf>(v);
  v += shifted<0x142, 0xa>(v);  // row_bcast:15 into the second and fourth row
  v += shifted<0x143, 0xc>(v);  // row_bcast:31 into the upper half
  return v;
}
__device__ __forceinline__ int32_t lane_of(int32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int64_t lane_of(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)lane_of((int32_t)(v >> 32), lane) << 32 | (uint32_t)lane_of((int32_t)v, lane));
}
__device__ __forceinline__ double lane_of(double v, int lane) { return __builtin_bit_cast(double, lane_of(__builtin_bit_cast(int64_t, v), lane)); }
// The larger (or the sum) of a lane's value and that of the lane 16, or 32, places away, without a trip through LDS.
__device__ __forceinline__ void across16(float v, float &a, float &b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  const uint32_t x = r[0], y = r[1];  // (a bit cast of a single vector element reads element 0)
  a = __builtin_bit_cast(float, x);
  b = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ void across32(float v, float &a, float &b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  const uint32_t x = r[0], y = r[1];  // (a bit cast of a single vector element reads element 0)
  a = __builtin_bit_cast(float, x);
  b = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float max16(float v) { float a, b; across16(v, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float max32(float v) { float a, b; across32(v, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float sum16(float v) { float a, b; across16(v, a, b); return a + b; }
__device__ __forceinline__ float sum32(float v) { float a, b; across32(v, a, b); return a + b; }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Partial results that another workgroup reads, maybe behind another L2: written through to memory and read from there
// (device scope).
__device__ __forceinline__ void store_shared(float *p, f32x2 v) {
  __hip_atomic_store((unsigned long long *)p, __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_shared(const float *p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// The slices of a unit but the last to arrive leave; true for that one.  Every wave's partial results have gone through to memory
// (device-scope stores, waited for) before one thread counts the workgroup in, so a relaxed count is enough on this hardware; the
// last one reads them with device-scope loads.  It also sets the count back for the next launch.
__device__ __forceinline__ bool last_to_arrive(uint32_t *arrivals, int32_t splits, uint32_t *flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t n = __hip_atomic_fetch_add(arrivals, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = n;
    if (n + 1 == (uint32_t)splits) __hip_atomic_store(arrivals, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *flag + 1 == (uint32_t)splits;
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ f32x4 load_f4_any(const float *p) { return *(const f32x4_any SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ float load_f(const float *p) { return *(const float SK_GLOBAL *)(uintptr_t)p; }
__device__ __forceinline__ uint32_t load_u16(const void *p) { return *(const uint16_t SK_GLOBAL *)(uintptr_t)p; }

// The last index i of [0, n) with first[i] <= x, 64 candidates at a time (first[0] <= x, not decreasing; x the same in all lanes).
template <class T>
__device__ __forceinline__ int32_t last_not_above(const T *first, int32_t n, int64_t x, int lane) {
  int32_t lo = 0;
  while (n > 1) {
    const int32_t step = (n + 63) / 64, i = lo + lane * step;
    const bool le = lane * step < n && (int64_t)(*(const T SK_GLOBAL *)(uintptr_t)(first + i)) <= x;
    const int32_t hit = max(1, (int32_t)__popcll(__ballot(le))) - 1;
    lo += hit * step;
    n = min(step, n - hit * step);
  }
  return lo;
}

// Loads and stores of what a launch will not see again, past the caches (ONCE) where it moves more than PAST_CACHES bytes: what is there
// stays there, and the launch is faster by as much (19000 rows of 48 heads of 128 by 7 %, 1 GB of pages by 3 %).  A smaller launch's
// outputs would be found in the caches by the one that reads them.
template <bool ONCE>
__device__ __forceinline__ u32x4 load16_once(const void *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4 SK_GLOBAL *)(uintptr_t)p);
  return load16(p);
}
template <bool ONCE>
__device__ __forceinline__ void store16_once(void *p, u32x4 v) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(v, (u32x4 SK_GLOBAL *)(uintptr_t)p);
  else
    store16(p, v);
}

// The sum over groups of 1, 2, 4, .. 32 neighbouring lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ float other_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int32_t, v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_over(float v, int lanes) {
  if (lanes >= 2) v += other_lane<0xb1>(v);    // quad_perm: the other of two
  if (lanes >= 4) v += other_lane<0x4e>(v);    // quad_perm: the other two of four
  if (lanes >= 8) v += other_lane<0x141>(v);   // row_half_mirror
  if (lanes >= 16) v += other_lane<0x140>(v);  // row_mirror
  if (lanes >= 32) v = sum16(v);
  return v;
}

}  // namespace sk
