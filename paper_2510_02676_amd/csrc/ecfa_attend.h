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
#include <type_traits>

#include "ecfa_device.h"

namespace ecfa {

// Division by a number that the host knows: exact for dividends below 2^31.
struct Divisor {
    uint32_t by, mul, shift;
};

inline Divisor divisor_of(uint32_t by)
{
    uint32_t shift = 0;
    while (shift < 31 && (1u << shift) < by) shift++;
    return Divisor{by, (uint32_t)((1ull << (31 + shift)) / by + 1), 31 + shift};
}

__device__ inline int32_t over(int32_t x, const Divisor &d) { return (int32_t)(((uint64_t)(uint32_t)x * d.mul) >> d.shift); }

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
    float cap, cap_inv;                      // softcap, 0: none; 1 / softcap
    uint32_t head_dim, heads, kv_heads, share, causal, window;
    Divisor by_share, by_kv_heads, by_goal, by_items;
    int32_t few_rows;                        // sequences of up to so many rows are the few-rows kernel's, the others the many-rows kernel's
    uint32_t few_tile;                       // rows of a tile
    uint32_t few_goal, few_unit, few_items;  // see few_plan
    uint32_t many_tiles, many_splits;
};

constexpr int FEW_WAVES = 4;
constexpr int MANY_WAVES = 4, MANY_ROWS = 32 * MANY_WAVES, MANY_KEYS = 64, MANY_UNIT = MANY_KEYS / 32;

// The partial sums of a row: of a piece of its keys, and of its first split.
__device__ inline int64_t few_part(const AttendArgs &a, uint32_t item, uint32_t kvh, int32_t row)
{
    return ((int64_t)item * a.kv_heads + kvh) * a.few_tile + row;
}
__device__ inline int64_t many_part(const AttendArgs &a, int64_t t, uint32_t head) { return a.many_part0 + (t * a.heads + head) * a.many_splits; }

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

// How the steps of 32 keys that a tile of many rows sees are dealt to the splits of the launch: [first, first + count) of step numbers,
// `per` to a split, a multiple of MANY_UNIT.  `used` splits have work; none if the tile sees nothing.
struct Split {
    int32_t first, count, per, used;
};

__device__ inline Split split_of(const KeyRange &r, uint32_t splits)
{
    Split p{0, 0, MANY_UNIT, 0};
    if (r.hi <= r.lo) return p;
    p.first = r.lo / 32;
    p.count = (r.hi + 31) / 32 - p.first;
    p.per = (int32_t)(((uint32_t)p.count + splits - 1) / splits);
    p.per = (p.per + MANY_UNIT - 1) / MANY_UNIT * MANY_UNIT;
    p.used = (p.count + p.per - 1) / p.per;
    return p;
}

// How the keys of the few-rows kernel's sequences are dealt to its workgroups.  All of them, in steps of 32 keys, are cut into about
// few_goal equal pieces (of few_unit steps at least, and a multiple of that): a sequence gets as many items as it has pieces, one if it
// has rows and sees nothing.  That is few_goal + n_seqs items at most, whatever the lengths are, which only the device knows.
// few_goal 0, or a sequence of over 2^25 keys: an item is a sequence.  Every wave works this out for itself: a lane a sequence, 64 at a time.
constexpr int32_t FEW_LONGEST = 1 << 20;     // steps of a sequence that is cut: sums over 1024 sequences stay in 32 bits

struct FewItem {
    bool there;
    uint32_t s, first_item;                  // of the sequence
    int32_t split, per, used;
};

__device__ inline int32_t few_steps(const AttendArgs &a, uint32_t s)           // -1: not this kernel's, or no rows
{
    const Seq sq = seq_of(a.b, s);
    const int32_t rows = sq.qn * (int32_t)a.share;
    if (rows <= 0 || rows > a.few_rows) return -1;
    const int32_t end = rows < (int32_t)a.few_tile ? rows : (int32_t)a.few_tile;
    const KeyRange r = keys_of(a, sq, prefix_of(a, s, sq), 0, over(end - 1, a.by_share));
    return r.hi > r.lo ? (r.hi + 31) / 32 - r.lo / 32 : 0;
}

// The item of a workgroup, or (by_seq) that of the first piece of a sequence.
__device__ inline FewItem few_plan(const AttendArgs &a, uint32_t wanted, bool by_seq = false)
{
    const uint32_t n = a.b.n_seqs, lane = threadIdx.x & 63;
    if (a.few_goal == 0) return FewItem{wanted < n && few_steps(a, wanted) >= 0, wanted, wanted, 0, 0x3fffffff, 1};
    const int32_t own = lane < n ? few_steps(a, lane) : -1;
    int32_t total = own > 0 ? own : 0;
    bool long_ones = own > FEW_LONGEST;
    for (uint32_t base = 64; base < n; base += 64) {
        const int32_t x = base + lane < n ? few_steps(a, base + lane) : -1;
        total += x > 0 ? x : 0;
        long_ones = long_ones || x > FEW_LONGEST;
    }
    FewItem it{false, 0, 0, 0, 0x3fffffff, 0};
    if (!__any(long_ones)) {
        if (n > 1)
            for (int k = 1; k < 64; k *= 2) total += __shfl_xor(total, k);
        total = __builtin_amdgcn_readfirstlane(total);         // at most 2^30: the host asks for pieces of up to 1024 sequences
        const int32_t unit = (int32_t)a.few_unit, piece = over(total + (int32_t)a.few_goal - 1, a.by_goal);
        it.per = piece > unit ? (piece + unit - 1) & -unit : unit;
    }
    const float per_inv = __builtin_amdgcn_rcpf((float)it.per);
    uint32_t before = 0;
    for (uint32_t base = 0; base < n; base += 64) {
        const int32_t x = base == 0 ? own : base + lane < n ? few_steps(a, base + lane) : -1;
        uint32_t mine = x < 0 ? 0u : 1u;
        if (x > it.per) {                                      // x / per, upwards: at most few_goal, where fp32 is off by less than one
            mine = (uint32_t)((float)x * per_inv);
            mine -= (int32_t)mine * it.per > x ? 1u : 0u;
            mine += (int32_t)mine * it.per < x ? 1u : 0u;
        }
        uint32_t sum = mine;                                   // of this lane and those before it
        if (n > 1)
            for (int k = 1; k < 64; k *= 2) {
                const uint32_t y = (uint32_t)__shfl_up((int)sum, k);
                sum += (int)lane >= k ? y : 0u;
            }
        const bool here = by_seq ? base + lane == wanted : before + sum > wanted && before + sum - mine <= wanted;
        const uint64_t hit = __ballot(here && mine > 0);
        if (hit) {
            const int i = __ffsll((unsigned long long)hit) - 1;
            it.there = true;
            it.s = base + (uint32_t)i;
            it.used = __builtin_amdgcn_readlane((int)mine, i);
            it.first_item = before + (uint32_t)__builtin_amdgcn_readlane((int)(sum - mine), i);
            it.split = by_seq ? 0 : (int32_t)(wanted - it.first_item);
            return it;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    }
    return it;
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

// What a dot product is multiplied by for a score in units of ln 2, kept within the normal numbers of fp32: zero would make NaN of what is masked, an
// infinity of a dot product of 0.
__device__ inline float factor_of(const AttendArgs &a, float k_scale) { return __builtin_amdgcn_fmed3f(a.scale_log2 * k_scale, 0x1p-126f, 0x1.fffffep127f); }

// The score of a dot product x, in units of ln 2, with the cap if there is one: softcap * tanh(y), y = scale x / softcap, and
// tanh(y) = 1 - 2 / (e^(2 y) + 1), which is off by 2^-23 of the cap at most.  That is all for caps up to SIMPLE_CAP (2^-16 of a score); beyond
// it small y, where that loses digits, take y - y^3 / 3 + 2 y^5 / 15 (error below 2^-26 |y| for |y| < 0.06),
// which costs 6 % of a mixed batch whose scores are capped (47.4 -> 50.3 us).  cap_in = to_log2 * 2 / softcap.
constexpr float SIMPLE_CAP = 64.f;
__device__ inline float capped_or_scaled(const AttendArgs &a, float x, float to_log2, float cap_in)
{
    if (!(a.cap > 0.f)) return x * to_log2;
    const float z = x * cap_in, c = a.cap * LOG2E;             // z = 2 y log2(e)
    const float t = __builtin_fmaf(-2.f * c, __builtin_amdgcn_rcpf(exp2_fast(z) + 1.f), c);
    if (a.cap <= SIMPLE_CAP) return t;
    const float y = z * (0.5f / LOG2E), y2 = y * y;
    const float small = __builtin_fmaf(y * y2, __builtin_fmaf(y2, 0.13333333f, -0.33333333f), y) * c;
    return __builtin_fabsf(y) < 0.06f ? small : t;
}
__device__ inline float less_distance(float x, float slope, int32_t far) { return __builtin_fmaf(-slope, (float)(far < 0 ? -far : far), x); }

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

// Transposing reads of V from LDS, several at a time, with the wait for them.  (As builtins each would first wait for all loads from memory
// to LDS that are on their way, those of the next step too: the compiler does not know that they go to the other buffer.)
// tr16: lane i of sixteen gives the place of four elements of row i / 4 and gets column i of the four rows; N fragments of eight keys from two
// reads each, at at0[n] and at1[n], both `OFFSET` bytes on.  tr8: eight bytes of row i / 2, column i of eight rows, for each fragment one read.
template <int OFFSET>
__device__ __forceinline__ void tr16(const int (&at0)[3], const int (&at1)[3], bf16x8 *f)
{
    u32x2 a[3], b[3];
    asm volatile("ds_read_b64_tr_b16 %0, %6 offset:%12\n\tds_read_b64_tr_b16 %1, %7 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %2, %8 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(b[0]), "=&v"(a[1]), "=&v"(b[1]), "=&v"(a[2]), "=&v"(b[2])
                 : "v"(at0[0]), "v"(at1[0]), "v"(at0[1]), "v"(at1[1]), "v"(at0[2]), "v"(at1[2]), "i"(OFFSET)
                 : "memory");
    for (int n = 0; n < 3; n++) f[n] = __builtin_bit_cast(bf16x8, u32x4{a[n][0], a[n][1], b[n][0], b[n][1]});
}
template <int OFFSET>
__device__ __forceinline__ void tr16(const int (&at0)[4], const int (&at1)[4], bf16x8 *f)
{
    u32x2 a[4], b[4];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %1, %9 offset:%16\n\t"
                 "ds_read_b64_tr_b16 %2, %10 offset:%16\n\tds_read_b64_tr_b16 %3, %11 offset:%16\n\t"
                 "ds_read_b64_tr_b16 %4, %12 offset:%16\n\tds_read_b64_tr_b16 %5, %13 offset:%16\n\t"
                 "ds_read_b64_tr_b16 %6, %14 offset:%16\n\tds_read_b64_tr_b16 %7, %15 offset:%16\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(b[0]), "=&v"(a[1]), "=&v"(b[1]), "=&v"(a[2]), "=&v"(b[2]), "=&v"(a[3]), "=&v"(b[3])
                 : "v"(at0[0]), "v"(at1[0]), "v"(at0[1]), "v"(at1[1]), "v"(at0[2]), "v"(at1[2]), "v"(at0[3]), "v"(at1[3]), "i"(OFFSET)
                 : "memory");
    for (int n = 0; n < 4; n++) f[n] = __builtin_bit_cast(bf16x8, u32x4{a[n][0], a[n][1], b[n][0], b[n][1]});
}
template <int OFFSET>
__device__ __forceinline__ void tr8(const int (&at)[3], u32x2 *f)
{
    asm volatile("ds_read_b64_tr_b8 %0, %3 offset:%6\n\tds_read_b64_tr_b8 %1, %4 offset:%6\n\tds_read_b64_tr_b8 %2, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "i"(OFFSET)
                 : "memory");
}
template <int OFFSET>
__device__ __forceinline__ void tr8(const int (&at)[4], u32x2 *f)
{
    asm volatile("ds_read_b64_tr_b8 %0, %4 offset:%8\n\tds_read_b64_tr_b8 %1, %5 offset:%8\n\t"
                 "ds_read_b64_tr_b8 %2, %6 offset:%8\n\tds_read_b64_tr_b8 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "i"(OFFSET)
                 : "memory");
}

// f(integral_constant) for 0 .. N - 1: offsets in instructions are constants.
template <int N, int I = 0, class F>
__device__ __forceinline__ void times(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        times<N, I + 1>(f);
    }
}

// The slow way for one row: key by key, in fp32, from memory.  Taken where a value that some rows of a tile see and others do not
// is NaN or infinite: the matrix cores would multiply it by the zero weight of the rows that do not see it.  PARTS lanes
// (lane / (64 / PARTS) of them) share a row; element 8 (PARTS c + part) + .. of q and k is a lane's in dot products, and `element(n)`
// names the n-th group of four elements of the result that it holds, in y[4 n ..].  Steps of 32 keys: `units` of them at every
// `stride`-th from step_a on, below step_b.
template <bool F8, int PARTS, int GROUPS, class Element>
__device__ inline void attend_slowly(const AttendArgs &a, const uint8_t *q, const uint8_t *k0, const uint8_t *v0, const int32_t *table, int32_t step_a,
                                     int32_t step_b, int32_t units, int32_t stride, KeyRange seen, int32_t place, float to_log2, float slope, int part, Element element, float *y, float &m, float &l)
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
        if (key == 32 * (step_a + units)) {
            step_a += stride;
            key = 32 * step_a;
            if (step_a >= step_b) break;
        }
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
        x = less_distance(capped_or_scaled(a, x, to_log2, to_log2 * 2.f * a.cap_inv), slope, place - key);
        const float m_new = use ? max_f(m, x) : m, base = m_new == NONE ? 0.f : m_new;
        const float shrink = exp2_fast(m - base), w = use ? (float)(__bf16)exp2_fast(x - base) : 0.f;
        m = m_new;
        l = l * shrink + w;
#pragma unroll
        for (int n = 0; n < GROUPS; n++) {
            const int e = element(n);
            bf16x4 vv{};
            if (e < (int)a.head_dim) {
                if constexpr (F8) {
                    const bf16x8 b = bf16_of_e4m3(*(const uint32_t *)(v + e), 0);
                    vv = bf16x4{b[0], b[1], b[2], b[3]};
                } else vv = *(const bf16x4 *)(v + 2 * e);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float z = y[4 * n + i] * shrink;
                y[4 * n + i] = use ? z + w * (float)vv[i] : z;
            }
        }
    }
}

// Launches, one per cache type; kc = 32-element pieces of a head that the kernels are compiled for.
int launch_attend_bf16(const AttendArgs &a, uint32_t kc, bool few, bool many, hipStream_t s);
int launch_attend_e4m3(const AttendArgs &a, uint32_t kc, bool few, bool many, hipStream_t s);

} // namespace ecfa
