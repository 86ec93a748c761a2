// Attention of new tokens over a paged cache, the parts that its kernels and its host side share.
//
//   x_j = scale q . k_j (capped, less slope |p - j|),   out = sum_j e^(x_j - m) v_j / sum_j e^(x_j - m)
//
// The rows that meet the keys of one key/value head are the pairs (token, query head of that head), token by token: row r is
// query head r % share of token r / share.  Tokens of a sequence with the same keys thus share one pass over them.  A
// tile of rows walks over its keys 32 (or 64) at a time with a running maximum m and sum l.
//
// Products are computed transposed, S^T = K Q^T and O^T = V^T P^T: then a lane holds one row's scores (column lane % 16 or
// lane % 32 of the result), its statistics are the lane's own, and the scores leave the matrix cores in the order in which
// they have to enter them again as P^T, eight keys a lane, so that P never goes through LDS.  V^T comes from row-major V
// by the transposing LDS reads.
#pragma once
#include "ecfa_device.h"

namespace ecfa {

struct AttendArgs {
    CacheView c;
    BatchView b;
    const uint8_t *q;
    uint8_t *out;
    int64_t q_tok, q_head, o_tok, o_head;    // bytes
    const float *slopes;
    const int32_t *prefix;
    float *part;                             // partial sums: [row of (token, head)][split][head_dim], then (m, l) pairs
    float *part_ml;
    float scale_log2;                        // scale * log2(e)
    float cap;                               // softcap, 0: none
    uint32_t head_dim, heads, kv_heads, share, causal, window;
    uint32_t splits, row_tiles, tile_rows, split_unit;   // of a launch
};

constexpr float LOG2E = 1.4426950408889634f;
constexpr float NONE = -__builtin_huge_valf();

// What keys a tile of rows sees.  [lo, hi) is seen by some row, [full_lo, full_hi) by every one.
struct KeyRange {
    int32_t lo, hi, full_lo, full_hi;
};

__device__ inline KeyRange keys_of(const AttendArgs &a, const Seq &sq, int32_t prefix, int32_t first, int32_t last)   // tokens of the sequence
{
    const int32_t p0 = sq.place0 + first, p1 = sq.place0 + last;
    KeyRange r{0, sq.len, 0, sq.len};
    if (a.causal) {
        r.hi = p1 + 1 > prefix ? p1 + 1 : prefix;
        r.full_hi = p0 + 1 > prefix ? p0 + 1 : prefix;
        r.hi = r.hi < sq.len ? r.hi : sq.len;
        r.full_hi = r.full_hi < sq.len ? r.full_hi : sq.len;
    }
    if (a.window) {
        const int64_t w = a.window;                            // up to 2^32 - 1
        r.lo = p0 + 1 > w ? (int32_t)(p0 + 1 - w) : 0;
        r.full_lo = p1 + 1 > w ? (int32_t)(p1 + 1 - w) : 0;
    }
    return r;
}

__device__ inline int32_t prefix_of(const AttendArgs &a, uint32_t s, const Seq &sq)
{
    if (!a.prefix) return 0;
    const int32_t n = a.prefix[s];
    return n < sq.len ? n : sq.len;
}

// How the steps of 32 keys that a tile of rows sees are dealt to the splits of the launch: [first, first + count) of step numbers,
// `per` to a split, a multiple of `unit`.  `used` splits have work; none if the tile sees nothing.
struct Split {
    int32_t first, count, per, used;
};

__device__ inline Split split_of(const KeyRange &r, uint32_t splits, int32_t unit)
{
    Split p{0, 0, unit, 0};
    if (r.hi <= r.lo) return p;
    p.first = r.lo / 32;
    p.count = (r.hi + 31) / 32 - p.first;
    p.per = (int32_t)(((uint32_t)p.count + splits - 1) / splits);
    p.per = (p.per + unit - 1) / unit * unit;
    p.used = (p.count + p.per - 1) / p.per;
    return p;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline float max_f(float a, float b) { return __builtin_fmaxf(a, b); }      // a NaN loses: it comes back through the weights

// The larger of, or the sum of, a lane's value and that of the lane 32 (16) away.  The instructions swap halves (rows of 16
// lanes) of two registers, so that for the same value in both one of them ends with either partner's.
template <int LANES>
__device__ inline void partners(float x, float *y, float *z)
{
    if constexpr (LANES == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
        const uint32_t a = r[0], b = r[1];
        *y = __builtin_bit_cast(float, a), *z = __builtin_bit_cast(float, b);
    } else {
        const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(x), f32_bits(x), false, false);
        const uint32_t a = r[0], b = r[1];
        *y = __builtin_bit_cast(float, a), *z = __builtin_bit_cast(float, b);
    }
}
template <int LANES>
__device__ inline float max_xor(float x)
{
    float y, z;
    partners<LANES>(x, &y, &z);
    return max_f(y, z);
}
template <int LANES>
__device__ inline float sum_xor(float x)
{
    float y, z;
    partners<LANES>(x, &y, &z);
    return y + z;
}

// softcap * tanh(x / softcap), x in units of ln 2 as everything here: tanh(y) = 1 - 2 / (e^(2 y) + 1), and for small y, where that
// loses digits, y - y^3 / 3 + 2 y^5 / 15 (error below 2^-26 |y| for |y| < 0.06).
__device__ inline float capped(float x_log2, float cap)
{
    const float y = x_log2 / (cap * LOG2E);
    const float t = 1.f - 2.f / (exp2_fast(y * (2.f * LOG2E)) + 1.f);
    const float y2 = y * y;
    const float small = y * (1.f + y2 * (-0.33333333f + y2 * 0.13333333f));
    return (__builtin_fabsf(y) < 0.06f ? small : t) * (cap * LOG2E);
}

// Eight E4M3 bytes as BF16, which holds each of them.
__device__ inline bf16x8 bf16_of_e4m3(uint32_t lo, uint32_t hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Order between the LDS accesses of a wave's lanes where no other wave is concerned.
__device__ inline void lds_fence_wave()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Launches, one per cache type; kc = 32-element pieces of a head that the kernels are compiled for.
int launch_few_rows_bf16(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s);
int launch_few_rows_e4m3(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s);

} // namespace ecfa
