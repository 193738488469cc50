// The kernels of norms, in units of compilation (-DSK_UNIT=0 to 5).
#include "layer_norm.hip.h"

namespace sk {
#define SK_NORM_FORM(T, P)                               \
  template __global__ void sk_norm<T, P, false>(NormArgs); \
  template __global__ void sk_norm<T, P, true>(NormArgs);
#if SK_UNIT == 0
SK_NORM_FORM(16, 2)
#elif SK_UNIT == 1
SK_NORM_FORM(64, 2)
#elif SK_UNIT == 2
SK_NORM_FORM(128, 2)
#elif SK_UNIT == 3
SK_NORM_FORM(256, 2)
#elif SK_UNIT == 4
SK_NORM_FORM(512, 2)
#elif SK_UNIT == 5
SK_NORM_FORM(1024, 4)
#else
#error "SK_UNIT is 0 to 5"
#endif
}  // namespace sk
