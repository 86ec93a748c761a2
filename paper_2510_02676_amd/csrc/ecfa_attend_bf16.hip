// The attention kernels for a cache in BF16.
#include "ecfa_attend_launch.h"

namespace ecfa {
int launch_attend_bf16(const AttendArgs &a, uint32_t kc, bool few, bool many, hipStream_t s) { return launch_attend<false>(a, kc, few, many, s); }
} // namespace ecfa
