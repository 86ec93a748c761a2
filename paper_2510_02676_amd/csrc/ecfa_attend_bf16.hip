// The attention kernels for a cache in BF16.
#include "ecfa_attend_few.h"
#include "ecfa_attend_many.h"

namespace ecfa {
int launch_few_rows_bf16(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s) { return launch_few_rows<false>(a, kc, tiles, s); }
int launch_many_rows_bf16(const AttendArgs &a, uint32_t kc, hipStream_t s) { return launch_many_rows<false>(a, kc, s); }
} // namespace ecfa
