// The attention kernels, in units of compilation (-DSK_UNIT=0 to 3).
#include "cache_kernels.hip.h"

namespace sk {
#if SK_UNIT == 0
template __global__ void sk_attend<false, false>(AttnArgs);
#elif SK_UNIT == 1
template __global__ void sk_attend<true, false>(AttnArgs);
#elif SK_UNIT == 2
template __global__ void sk_attend<false, true>(AttnArgs);
#elif SK_UNIT == 3
template __global__ void sk_attend<true, true>(AttnArgs);
#else
#error "SK_UNIT is 0 to 3"
#endif
}  // namespace sk
