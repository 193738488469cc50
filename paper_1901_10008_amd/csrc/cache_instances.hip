// The attention kernels, in units of compilation (-DSK_UNIT=0 to 7), one per element type and class of head sizes.
#include "cache_kernels.hip.h"

namespace sk {
#define SK_ATTEND(dt, dp) template __global__ void sk_attend<dt, dp>(AttnArgs);
#if SK_UNIT == 0
SK_ATTEND(SK_BF16, 64)
#elif SK_UNIT == 1
SK_ATTEND(SK_BF16, 96)
#elif SK_UNIT == 2
SK_ATTEND(SK_BF16, 128)
#elif SK_UNIT == 3
SK_ATTEND(SK_BF16, 256)
#elif SK_UNIT == 4
SK_ATTEND(SK_F16, 64)
#elif SK_UNIT == 5
SK_ATTEND(SK_F16, 96)
#elif SK_UNIT == 6
SK_ATTEND(SK_F16, 128)
#elif SK_UNIT == 7
SK_ATTEND(SK_F16, 256)
#else
#error "SK_UNIT is 0 to 7"
#endif
}  // namespace sk
