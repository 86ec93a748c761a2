// Rows between the products of experts: silu(gate) * up to E4M3 with scales (ecfm_gate), and the experts' rows back to their tokens
// (ecfm_combine).  Both are one pass over their data and bound by memory, or, for a few tokens, by the launch.
#include <cmath>

#include "ecfa_host.h"
#include "ecfa_pieces.h"
#include "ecfm_device.h"

namespace ecfm {
namespace {
using namespace ecfa;

// at / per of the launch's pieces, at below 2^31, by the host's multiplier.
struct By {
    uint32_t times, shift;
    __device__ uint32_t of(uint32_t at) const { return __umulhi(at, times) >> shift; }
};

By divide_by(uint32_t n)                                       // n from 2 on: ceil(2^(31 + l) / n) with 2^l >= n is below 2^32, and right for 31 bits
{
    uint32_t l = 1;
    while ((1u << l) < n) l++;
    return By{(uint32_t)(((1ull << (31 + l)) + n - 1) / n), l - 1};
}

struct GateArgs {
    const uint8_t *g, *u;
    uint8_t *q;
    float *scale;
    int64_t g_row, u_row;                    // bytes
    uint32_t rows, cols;                     // of this launch
    By by_row;
};

// silu(g) * u of eight: with t = exp(-|g|), g / (1 + t), or g t / (1 + t) below zero, so that nothing overflows on the way.
// t = 2^e (1 + r ln 2), e the product of -|g| and log2(e) in fp32 and r what that leaves out, is within two of its last places.  From g = -87.3 on
// down t is below fp32's normal numbers, which the instruction puts to 0, though with a large u the product is not: there, and from LOW on, t is taken
// 2^136 times as large and u as much smaller (1 + t is 1).  That reaches to g = -181; below, the product is less than 2^-126, which is 0 beside 2^-100,
// and so it is at -infinity, where g t would be NaN.
// exp, a division and clamps were 373 instructions for the eight and as long as their bytes (86 us at 32768 x 2048; 72 with a reciprocal, 59 so: 5.7 TB/s;
// 58.3 where all products below -87.3 are zeros).
template <bool F32>
__device__ inline void gated8(const uint8_t *g, const uint8_t *u, float *h)
{
    constexpr float LOG2E = 1.44269502f, REST = 1.92596303e-8f, LN2 = 0.693147181f;       // LOG2E + REST = log2(e)
    constexpr float LOW = -87.f;
    float x[8], silu[8];
    uint32_t lowest = 0;                                       // as bits: of two numbers below zero the lower one has more
    load8<F32>(g, x);
    load8<F32>(u, h);
    // 2^to (1 + r ln 2), `to` e or e and a whole number
    const auto exp_of = [](float a, float e, float to) {
        const float r = fmaf(a, REST, fmaf(a, LOG2E, -e)), t = __builtin_amdgcn_exp2f(to);
        return t > 0.f ? fmaf(t, r * LN2, t) : t;              // (at infinity r is not a number)
    };
    for (int i = 0; i < 8; i++) {
        const float a = -fabsf(x[i]), e = a * LOG2E, t = exp_of(a, e, e);
        silu[i] = (x[i] < 0.f ? x[i] * t : x[i]) * __builtin_amdgcn_rcpf(1.f + t);
        lowest = f32_bits(x[i]) > lowest ? f32_bits(x[i]) : lowest;
    }
    if (__builtin_expect(lowest > f32_bits(LOW), 0))           // (in its place, not behind the end, 60 us)
        for (int i = 0; i < 8; i++)
            if (x[i] < LOW) {
#pragma clang fp contract(off)                                 // (e + 136 is exact, but not as one operation with the product that r is the rest of)
                const float e = x[i] * LOG2E, t = exp_of(x[i], e, e + 136.f);
                silu[i] = t == 0.f ? 0.f : x[i] * t;
                h[i] = __builtin_ldexpf(h[i], -136);
            }
    for (int i = 0; i < 8; i++) h[i] = silu[i] * h[i];
}

// Eight to E4M3 where none is further than a rounding beyond 448: they need not be limited.
__device__ inline void store_scaled(uint8_t *q, const float *x, float inv)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, hi, true);
    __builtin_nontemporal_store(ecfa::u32x2{(uint32_t)lo, (uint32_t)hi}, (ecfa::u32x2 *)q);
}

template <bool F32>
__global__ __launch_bounds__(256) void ecfm_gate_groups_kernel(const GateArgs a)
{
    constexpr int SRC = F32 ? 4 : 2;
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = a.by_row.of(at), p = at - row * (a.cols / 8);
    if (row >= a.rows) return;               // the sixteen lanes of a group together: there is a multiple of 16 pieces
    float h[8];
    gated8<F32>(a.g + (int64_t)row * a.g_row + (uint64_t)p * 8 * SRC, a.u + (int64_t)row * a.u_row + (uint64_t)p * 8 * SRC, h);
    const uint32_t m = most_of_lanes<16>(most8(h));
    float scale;
    const float inv = inverse_and_scale(m, &scale);
    if ((threadIdx.x & 15) == 0) a.scale[(uint64_t)row * (a.cols / 128) + p / 16] = scale;
    store_scaled(a.q + (uint64_t)row * a.cols + (uint64_t)p * 8, h, inv);
}

// A scale per row: THREADS threads a row, the row held in registers between its two uses up to HELD pieces of eight a thread, computed again
// beyond that.
template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void ecfm_gate_rows_kernel(const GateArgs a)
{
    constexpr int SRC = F32 ? 4 : 2, HELD = 4, BLOCK = THREADS == 64 ? 256 : THREADS, WAVES = BLOCK / 64;
    const uint32_t row = THREADS == 64 ? blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x, t = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
    const bool there = row < a.rows;
    const uint8_t *g = a.g + (int64_t)(there ? row : 0) * a.g_row, *u = a.u + (int64_t)(there ? row : 0) * a.u_row;
    const uint32_t pieces = a.cols / 8;
    float held[HELD][8];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < HELD; k++)
        if (t + k * THREADS < pieces) {
            const uint64_t at = (uint64_t)(t + k * THREADS) * 8 * SRC;
            gated8<F32>(g + at, u + at, held[k]);
            const uint32_t o = most8(held[k]);
            m = o > m ? o : m;
        }
    for (uint32_t p = t + HELD * THREADS; p < pieces; p += THREADS) {
        float h[8];
        gated8<F32>(g + (uint64_t)p * 8 * SRC, u + (uint64_t)p * 8 * SRC, h);
        const uint32_t o = most8(h);
        m = o > m ? o : m;
    }
    m = most_of_lanes<64>(m);
    if constexpr (THREADS > 64) {
        __shared__ uint32_t of_wave[WAVES];
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x / 64] = m;
        __syncthreads();
        for (int w = 0; w < WAVES; w++) m = of_wave[w] > m ? of_wave[w] : m;
    }
    if (!there) return;
    float scale;
    const float inv = inverse_and_scale(m, &scale);
    if (t == 0) a.scale[row] = scale;
    uint8_t *q = a.q + (uint64_t)row * a.cols;
#pragma unroll
    for (int k = 0; k < HELD; k++)
        if (t + k * THREADS < pieces) store_scaled(q + (uint64_t)(t + k * THREADS) * 8, held[k], inv);
    for (uint32_t p = t + HELD * THREADS; p < pieces; p += THREADS) {
        float h[8];
        gated8<F32>(g + (uint64_t)p * 8 * SRC, u + (uint64_t)p * 8 * SRC, h);
        store_scaled(q + (uint64_t)p * 8, h, inv);
    }
}

template <bool F32>
void launch_gate(const GateArgs &a, uint32_t group, hipStream_t s)
{
    if (group) hipLaunchKernelGGL((ecfm_gate_groups_kernel<F32>), dim3((unsigned)(((uint64_t)a.rows * (a.cols / 8) + 255) / 256)), dim3(256), 0, s, a);
    else if (a.cols <= 1024) hipLaunchKernelGGL((ecfm_gate_rows_kernel<F32, 64>), dim3((a.rows + 3) / 4), dim3(256), 0, s, a);
    else if (a.cols <= 8192) hipLaunchKernelGGL((ecfm_gate_rows_kernel<F32, 256>), dim3(a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((ecfm_gate_rows_kernel<F32, 1024>), dim3(a.rows), dim3(1024), 0, s, a);
}

struct CombineArgs {
    const uint8_t *y, *add;
    uint8_t *out;
    const int32_t *place;
    const float *weights;
    int64_t y_row, add_row, out_row;         // bytes
    uint32_t y_rows, first, tokens, top, cols;
    uint32_t add_f32, out_f32;
    By by_row;
};

// Eight elements as they come from memory, past the caches: nobody reads them again (4096 tokens of 8 x 7168: 116 us through them, 106 so).
template <bool F32>
struct Eight {
    f32x4 a, b;
    __device__ void load(const uint8_t *p) { a = __builtin_nontemporal_load((const f32x4 *)p), b = __builtin_nontemporal_load((const f32x4 *)(p + 16)); }
    __device__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

template <>
struct Eight<false> {
    ecfa::bf16x8 a;
    __device__ void load(const uint8_t *p) { a = __builtin_nontemporal_load((const ecfa::bf16x8 *)p); }
    __device__ float at(int i) const { return (float)a[i]; }
};

template <bool F32>
__global__ __launch_bounds__(256) void ecfm_combine_kernel(const CombineArgs a)
{
    constexpr int SRC = F32 ? 4 : 2;
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = a.cols == 8 ? at : a.by_row.of(at), p = at - row * (a.cols / 8);
    if (row >= a.tokens) return;
    const uint64_t t = (uint64_t)a.first + row;
    float sum[8] = {};
    if (a.add) {
        if (a.add_f32) load8<true>(a.add + (int64_t)t * a.add_row + (uint64_t)p * 32, sum);
        else load8<false>(a.add + (int64_t)t * a.add_row + (uint64_t)p * 16, sum);
    }
    // eight rows on their way at once (one after the other: 4096 tokens of 8 x 7168 121 us)
    for (uint32_t j0 = 0; j0 < a.top && a.y_rows; j0 += 8) {
        Eight<F32> y[8];
        float w[8];
        bool there[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; j++) {
            there[j] = false;
            if (j0 + j < a.top) {
                const uint32_t from = (uint32_t)a.place[t * a.top + j0 + j];
                w[j] = a.weights[t * a.top + j0 + j];
                there[j] = from < a.y_rows;
                y[j].load(a.y + (int64_t)(there[j] ? from : 0) * a.y_row + (uint64_t)p * 8 * SRC);
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < 8; j++)
            if (there[j])
                for (int i = 0; i < 8; i++) sum[i] = fmaf(w[j], y[j].at(i), sum[i]);
    }
    uint8_t *out = a.out + (int64_t)t * a.out_row;
    if (a.out_f32) {
        *(f32x4 *)(out + (uint64_t)p * 32) = f32x4{sum[0], sum[1], sum[2], sum[3]};
        *(f32x4 *)(out + (uint64_t)p * 32 + 16) = f32x4{sum[4], sum[5], sum[6], sum[7]};
    } else store8_bf16(out + (uint64_t)p * 16, sum);
}

int check_y(const ecfm_y *y, int64_t *row)
{
    if ((y->dtype != ECFA_F32 && y->dtype != ECFA_BF16) || y->rows > (1u << 28)) return ECF8_E_ARG;
    if (y->rows && !y->d) return ECF8_E_ARG;
    *row = apart(y->row_stride, y->dtype == ECFA_F32 ? 4 : 2, y->rows);
    return ((uintptr_t)y->d & 15) || (*row & 15) ? ECF8_E_ALIGN : ECF8_OK;
}

} // namespace
} // namespace ecfm

using namespace ecfm;

extern "C" {

int ecfm_gate(const void *d_g, const void *d_u, uint32_t dtype, uint64_t rows, uint64_t cols, int64_t g_stride, int64_t u_stride, uint32_t group,
              uint8_t *d_q, float *d_scale, void *stream)
{
    if ((dtype != ECFA_F32 && dtype != ECFA_BF16) || (group != 0 && group != 128) || cols == 0 || cols > (1u << 20) || cols % (group ? 128 : 16)) return ECF8_E_ARG;
    if (rows > 1ull << 40 || (rows && (!d_g || !d_u || !d_q || !d_scale))) return ECF8_E_ARG;
    GateArgs a{};
    const int64_t e = dtype == ECFA_F32 ? 4 : 2;
    a.g_row = ecfa::apart(g_stride, e, rows);
    a.u_row = ecfa::apart(u_stride, e, rows);
    if (((uintptr_t)d_g & 15) || ((uintptr_t)d_u & 15) || (a.g_row & 15) || (a.u_row & 15) || ((uintptr_t)d_q & 7) || ((uintptr_t)d_scale & 3)) return ECF8_E_ALIGN;
    a.g = (const uint8_t *)d_g;
    a.u = (const uint8_t *)d_u;
    a.q = d_q;
    a.scale = d_scale;
    a.cols = (uint32_t)cols;
    a.by_row = divide_by((uint32_t)cols / 8);
    const uint64_t pieces = 0x7fffff00u / (cols / 8);          // rows of a launch: its threads are counted in 32 bits, with the threads of a row
    const uint64_t most = pieces < 0x1fffff ? pieces : 0x1fffff;
    for (uint64_t left = rows; left; left -= a.rows) {
        a.rows = (uint32_t)(left < most ? left : most);
        if (dtype == ECFA_F32) launch_gate<true>(a, group, (hipStream_t)stream);
        else launch_gate<false>(a, group, (hipStream_t)stream);
        if (hipGetLastError() != hipSuccess) return ECF8_E_HIP;
        a.g += (int64_t)a.rows * a.g_row;
        a.u += (int64_t)a.rows * a.u_row;
        a.q += a.rows * cols;
        a.scale += a.rows * (group ? cols / 128 : 1);
    }
    return ECF8_OK;
}

int ecfm_combine(const ecfm_y *y, const int32_t *d_place, const float *d_weights, uint32_t n_tokens, uint32_t top, uint32_t cols, const ecfm_y *add,
                 const ecfm_y *out, void *stream)
{
    if (!y || !out || top == 0 || top > 32 || cols == 0 || cols % 8 || cols > (1u << 20) || n_tokens > (1u << 22) || out->rows != n_tokens) return ECF8_E_ARG;
    CombineArgs a{};
    int rc = check_y(y, &a.y_row);
    if (!rc) rc = check_y(out, &a.out_row);
    if (!rc && add && add->d) rc = add->rows != n_tokens ? ECF8_E_ARG : check_y(add, &a.add_row);
    if (rc) return rc;
    if (n_tokens && (!d_place || !d_weights)) return ECF8_E_ARG;
    if (((uintptr_t)d_place & 3) || ((uintptr_t)d_weights & 3)) return ECF8_E_ALIGN;
    a.y = (const uint8_t *)y->d;
    a.y_rows = y->rows;
    a.out = (uint8_t *)out->d;
    a.out_f32 = out->dtype == ECFA_F32;
    if (add) {
        a.add = (const uint8_t *)add->d;
        a.add_f32 = add->dtype == ECFA_F32;
    }
    a.place = d_place;
    a.weights = d_weights;
    a.top = top;
    a.cols = cols;
    if (cols > 8) a.by_row = divide_by(cols / 8);
    const uint32_t most = 0x7fffff00u / (cols / 8);            // tokens of a launch: its threads are counted in 32 bits
    for (uint32_t t = 0; t < n_tokens; t += a.tokens) {
        a.first = t;
        a.tokens = n_tokens - t < most ? n_tokens - t : most;
        const dim3 grid((unsigned)(((uint64_t)a.tokens * (cols / 8) + 255) / 256));
        if (y->dtype == ECFA_F32) hipLaunchKernelGGL(ecfm_combine_kernel<true>, grid, dim3(256), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(ecfm_combine_kernel<false>, grid, dim3(256), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return ECF8_E_HIP;
    }
    return ECF8_OK;
}

} // extern "C"
