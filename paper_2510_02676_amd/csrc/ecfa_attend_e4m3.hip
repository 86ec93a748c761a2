// The attention kernels for a cache in E4M3: the same, with the bytes turned into BF16 (which holds each of them) in registers.
#include "ecfa_attend_few.h"
#include "ecfa_attend_many.h"

namespace ecfa {
int launch_few_rows_e4m3(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s) { return launch_few_rows<true>(a, kc, tiles, s); }
int launch_many_rows_e4m3(const AttendArgs &a, uint32_t kc, hipStream_t s) { return launch_many_rows<true>(a, kc, s); }
} // namespace ecfa
