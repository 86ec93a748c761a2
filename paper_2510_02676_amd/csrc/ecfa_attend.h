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
    float *part;                             // partial sums of a row's splits, head_dim each: see few_part, many_part
    float *part_ml;                          // (m, l) of each
    int64_t many_part0;                      // where those of the tiles of many rows begin
    float scale_log2;                        // scale * log2(e)
    float cap;                               // softcap, 0: none
    uint32_t head_dim, heads, kv_heads, share, causal, window;
    int32_t few_rows;                        // sequences of up to so many rows are the few-rows kernel's, the others the many-rows kernel's
    uint32_t few_tile, few_splits;           // rows of a tile; splits of the first tile of a sequence (others, where there are any, have one)
    uint32_t many_tiles, many_splits;
};

// The partial sums of a row's first split.
__device__ inline int64_t few_part(const AttendArgs &a, uint32_t s, uint32_t kvh, int32_t row)
{
    return (((int64_t)s * a.kv_heads + kvh) * a.few_tile + row) * a.few_splits;
}
__device__ inline int64_t many_part(const AttendArgs &a, int64_t t, uint32_t head) { return a.many_part0 + (t * a.heads + head) * a.many_splits; }

constexpr int FEW_WAVES = 4, FEW_UNIT = FEW_WAVES;               // steps of 32 keys that a split is a multiple of
constexpr int MANY_WAVES = 4, MANY_ROWS = 32 * MANY_WAVES, MANY_KEYS = 64, MANY_UNIT = MANY_KEYS / 32;

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

// Two numbers to BF16, nearest even, in one instruction.
__device__ inline bf16x2 bf16_pair(float x, float y)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_convertvector((f32x2{x, y}), bf16x2);
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

// The slow way for one row: key by key, in fp32, from memory.  Taken where a value that some rows of a tile see and others do not
// is NaN or infinite: the matrix cores would multiply it by the zero weight of the rows that do not see it.  PARTS lanes
// (lane / (64 / PARTS) of them) share a row; element 8 (PARTS c + part) + .. of q and k is a lane's in dot products, and `element(n)`
// names the n-th group of four elements of the result that it holds, in y[4 n ..].  Steps [step_a, step_b) of 32 keys.
template <bool F8, int PARTS, int GROUPS, class Element>
__device__ inline void attend_slowly(const AttendArgs &a, const uint8_t *q, const uint8_t *k0, const uint8_t *v0, const int32_t *table, int32_t step_a,
                                     int32_t step_b, KeyRange seen, int32_t place, float to_log2, float slope, int part, Element element, float *y, float &m, float &l)
{
    const uint32_t in_page = (1u << a.c.page_shift) - 1;
    const auto eight = [](const uint8_t *p, float *x) {        // of the cache, from the place of the first
        bf16x8 b;
        if constexpr (F8) b = bf16_of_e4m3(((const uint32_t *)p)[0], ((const uint32_t *)p)[1]);
        else b = *(const bf16x8 *)p;
        for (int i = 0; i < 8; i++) x[i] = (float)b[i];
    };
    constexpr int E = F8 ? 1 : 2;
    m = NONE;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * GROUPS; i++) y[i] = 0.f;
#pragma unroll 1
    for (int32_t key = 32 * step_a; key < 32 * step_b; key++) {
        const bool in = key >= seen.lo && key < seen.hi;
        const uint32_t page = in ? (uint32_t)table[(uint32_t)key >> a.c.page_shift] : 0xffffffffu;
        const bool use = page < a.c.n_pages;
        if (!__any(use)) continue;
        const int64_t pg = use ? page : 0u, at = (uint32_t)key & in_page;
        const uint8_t *k = k0 + pg * a.c.k_page + at * a.c.k_tok, *v = v0 + pg * a.c.v_page + at * a.c.v_tok;
        float x = 0.f;
#pragma unroll 1
        for (int e = 8 * part; e < (int)a.head_dim; e += 8 * PARTS) {
            float kk[8];
            eight(k + e * E, kk);
            const bf16x8 qq = *(const bf16x8 *)(q + 2 * e);
            for (int i = 0; i < 8; i++) x += kk[i] * (float)qq[i];
        }
        for (int n = 64 / PARTS; n < 64; n *= 2) x += __shfl_xor(x, n);
        x *= to_log2;
        if (a.cap > 0.f) x = capped(x, a.cap);
        const int32_t far = place - key;
        x -= slope * (float)(far < 0 ? -far : far);
        const float m_new = use ? max_f(m, x) : m, base = m_new == NONE ? 0.f : m_new;
        const float shrink = exp2_fast(m - base), w = use ? (float)(__bf16)exp2_fast(x - base) : 0.f;
        m = m_new;
        l = l * shrink + w;
#pragma unroll
        for (int n = 0; n < GROUPS; n++) {
            const int e = element(n);
            float vv[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (e < (int)a.head_dim) eight(v + (e & ~7) * E, vv);
            for (int i = 0; i < 4; i++) {
                const float z = y[4 * n + i] * shrink;
                y[4 * n + i] = use ? z + w * (e & 4 ? vv[4 + i] : vv[i]) : z;
            }
        }
    }
}

// Launches, one per cache type; kc = 32-element pieces of a head that the kernels are compiled for.
int launch_few_rows_bf16(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s);
int launch_few_rows_e4m3(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s);
int launch_many_rows_bf16(const AttendArgs &a, uint32_t kc, hipStream_t s);
int launch_many_rows_e4m3(const AttendArgs &a, uint32_t kc, hipStream_t s);

} // namespace ecfa
