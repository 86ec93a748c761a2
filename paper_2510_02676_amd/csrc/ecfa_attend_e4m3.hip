// The attention kernels for a cache in E4M3: the same, with the bytes turned into BF16 (which holds each of them) in registers.
#include "ecfa_attend_launch.h"

namespace ecfa {
int launch_attend_e4m3(const AttendArgs &a, uint32_t kc, bool few, bool many, hipStream_t s) { return launch_attend<true>(a, kc, few, many, s); }
} // namespace ecfa
