// Launches of the attention kernels for one type of cache.
#pragma once
#include "ecfa_attend_few.h"
#include "ecfa_attend_many.h"

namespace ecfa {

// Chunks and single tokens of one step in one launch: the tiles of many rows first, which take longest, then the items of few rows, which fill
// compute units as they come free.  13 sequences of 1 to 517 tokens, window 1000, scores capped, E4M3: 50 us with the second
// kernel where two launches, and a workgroup for each row that is joined, took 75.  The items first: 2 us more.
template <int KC, bool F8, bool EXTRA>
__global__ __launch_bounds__(256, KC <= 4 ? 2 : 1) void ecfa_attend_mixed_kernel(const AttendArgs a, uint32_t many_blocks)
{
    constexpr int FEW = FewShape<KC, F8, 1>::BYTES, MANY = ManyShape<KC>::BYTES;
    __shared__ __align__(16) uint8_t lds[FEW > MANY ? FEW : MANY];
    if (blockIdx.x < many_blocks) attend_many<KC, F8, EXTRA>(a, blockIdx.x, lds);
    else attend_few<KC, F8, 1>(a, blockIdx.x - many_blocks, lds);
}

template <int KC, bool F8>
int launch_attend_kc(const AttendArgs &a, bool few, bool many, hipStream_t s)
{
    // Caps and slopes in instances of their own: with them in every one 4680 x 4680 tokens of 40 heads took 593 us, without 484.
    const bool extra = a.cap > 0.f || a.slopes;
    const uint32_t few_blocks = a.few_items * a.kv_heads, many_blocks = a.many_tiles * a.kv_heads * a.many_splits;
    if (few && many && a.few_tile == 16) {
        if (extra) hipLaunchKernelGGL((ecfa_attend_mixed_kernel<KC, F8, true>), dim3(many_blocks + few_blocks), dim3(256), 0, s, a, many_blocks);
        else hipLaunchKernelGGL((ecfa_attend_mixed_kernel<KC, F8, false>), dim3(many_blocks + few_blocks), dim3(256), 0, s, a, many_blocks);
        return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
    }
    if (many) {
        if (extra) hipLaunchKernelGGL((ecfa_attend_many_kernel<KC, F8, true>), dim3(many_blocks), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((ecfa_attend_many_kernel<KC, F8, false>), dim3(many_blocks), dim3(256), 0, s, a);
        if (hipGetLastError() != hipSuccess) return ECF8_E_HIP;
    }
    if (few) {
        if (a.few_tile == 16) hipLaunchKernelGGL((ecfa_attend_few_kernel<KC, F8, 1>), dim3(few_blocks), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((ecfa_attend_few_kernel<KC, F8, 2>), dim3(few_blocks), dim3(256), 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

template <bool F8>
int launch_attend(const AttendArgs &a, uint32_t kc, bool few, bool many, hipStream_t s)
{
    switch (kc) {
    case 2: return launch_attend_kc<2, F8>(a, few, many, s);
    case 3: return launch_attend_kc<3, F8>(a, few, many, s);
    case 4: return launch_attend_kc<4, F8>(a, few, many, s);
    case 6: return launch_attend_kc<6, F8>(a, few, many, s);
    default: return launch_attend_kc<8, F8>(a, few, many, s);
    }
}

} // namespace ecfa
