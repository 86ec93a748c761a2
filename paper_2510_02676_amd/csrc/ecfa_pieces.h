// Eight elements at a time: from memory to fp32, to BF16, to E4M3 with the scale of the largest of a group.
#pragma once
#include "ecfa_device.h"

namespace ecfa {

// Eight elements from memory as fp32.
template <bool F32>
__device__ inline void load8(const uint8_t *p, float *x)
{
    if constexpr (F32) {
        const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 16);
        for (int i = 0; i < 4; i++) x[i] = a[i], x[4 + i] = b[i];
    } else {
        const bf16x8 a = *(const bf16x8 *)p;
        for (int i = 0; i < 8; i++) x[i] = (float)a[i];
    }
}

__device__ inline void store8_bf16(uint8_t *p, const float *x)
{
    bf16x8 y;
    for (int i = 0; i < 8; i++) y[i] = (__bf16)x[i];          // to nearest even
    *(bf16x8 *)p = y;
}

// Eight fp32 as E4M3, to nearest even, limited to the largest number of the format; NaN stays NaN.
__device__ inline u32x2 pack8_e4m3(const float *x)
{
    float y[8];
    for (int i = 0; i < 8; i++) y[i] = x[i] > 448.f ? 448.f : x[i] < -448.f ? -448.f : x[i];
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    return u32x2{(uint32_t)lo, (uint32_t)hi};
}

// The largest |x| of eight, as bits: ordered like the numbers, infinity above all of them and NaN above that.
__device__ inline uint32_t most8(const float *x)
{
    uint32_t m = 0;
    for (int i = 0; i < 8; i++) {
        const uint32_t b = f32_bits(x[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

template <int LANES>
__device__ inline uint32_t most_of_lanes(uint32_t m)          // LANES consecutive lanes of a wave
{
#pragma unroll
    for (int k = 1; k < LANES; k *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)m, k);
        m = o > m ? o : m;
    }
    return m;
}

constexpr uint32_t SMALLEST_BITS = 0x0d800000u;               // 2^-100

__device__ inline float inverse_and_scale(uint32_t m, float *scale)
{
    const float a = __builtin_bit_cast(float, m > SMALLEST_BITS ? m : SMALLEST_BITS);
    *scale = a / 448.f;
    return 448.f / a;
}

__device__ inline void store_e4m3(uint8_t *q, const float *x, float inv)
{
    float y[8];
    for (int i = 0; i < 8; i++) y[i] = x[i] * inv;
    __builtin_nontemporal_store(pack8_e4m3(y), (u32x2 *)q);    // (past the caches: with what reads it next 11.7 -> 10.3 us at 2048 x 4096)
}

} // namespace ecfa
