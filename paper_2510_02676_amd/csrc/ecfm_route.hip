// From a router's logits to experts, their weights, and the pairs (token, expert) sorted by expert (ecfm.h).
#include "ecfm_device.h"

#include <cfloat>
#include <cmath>

namespace ecfm {
namespace {

constexpr uint32_t WAVES = 16, THREADS = 64 * WAVES, MAX_TOP = 32, MAX_EXPERTS = 1024;
constexpr uint32_t HALF_WAVE = 256;                // up to as many experts a token has 32 lanes, else 64
constexpr uint32_t MOST_TOKENS = 128;              // of a workgroup that chooses, or sorts
constexpr uint32_t ADD_UP = 512;                   // up to as many workgroups that choose, each one that sorts adds up all their counts by itself,
constexpr uint32_t SUMS_16 = 0xffff;               // two in a word: up to as many tokens
constexpr uint32_t CUS = 256;
constexpr uint32_t SLOTS = MOST_TOKENS * MAX_TOP, PER_WAVE = SLOTS / THREADS;

struct RouteArgs {
    const void *logits;
    const float *bias;
    int64_t stride;
    int32_t *ids, *starts, *rows, *place;
    float *weights;
    uint16_t *counts;                              // [workgroups that choose][padded]: pairs of each expert
    uint32_t *sums;                                // with many workgroups, [workgroups that sort + 1][padded]: pairs in those before; in all
    uint32_t tokens, experts, top, sigmoid, normalise, groups, top_groups, f32;
    uint32_t chosen_by, sorted_by;                 // workgroups
    uint32_t choose_tokens, sort_tokens;           // of a workgroup; the second is a multiple of the first
    uint32_t padded;                               // experts, rounded up to a multiple of 8
    uint32_t wide;                                 // logits and bias can be loaded by the 16 bytes (or what a lane has, if that is less)
    uint32_t size, per_size, lanes;                // of a group: experts, 2^20 / experts (rounded up), lanes if these are whole ones and 1, 2, 4, ..., else 0
    float scale;
};

// What sorting takes of LDS.  A pair without an expert has the number 0xffff.
struct SortSpace {
    uint16_t id[SLOTS];
    uint32_t start[MAX_EXPERTS], total[MAX_EXPERTS];
    uint32_t wave[WAVES];
};

// Lanes of a wave with the same number as this one, bit by bit.
__device__ inline uint64_t same_as_mine(uint32_t v, uint32_t bits)
{
    uint64_t m = ~0ull;
    for (uint32_t i = 0; i < bits; i++) {
        const bool one = v >> i & 1;
        const uint64_t b = __ballot(one);
        m &= one ? b : ~b;
    }
    return m;
}

// The pairs s.id[0 .. pairs) to their places, pair `first` of all the first of them.  s.start: pairs of the same expert in workgroups before, s.total: in all.
// A wave has a run of the pairs, 64 at a time: a pair's rank is the number of lanes below with the same expert, on top of what the wave had of it
// before.  No atomics, so the order is that of the tokens (8192 x 8 pairs with the sums before 7.6 us; each expert looking through all pairs 49).  counts: [WAVES][padded] of LDS.
__device__ inline void place_pairs(const RouteArgs &a, SortSpace &s, uint32_t *counts, uint32_t first, uint32_t pairs)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bits = 32 - __builtin_clz(a.experts);
    for (uint32_t i = threadIdx.x; i < WAVES * a.padded; i += THREADS) counts[i] = 0;
    // where each expert's pairs begin
    const uint32_t own = threadIdx.x < a.experts ? s.total[threadIdx.x] : 0;
    uint32_t upto = own;
    for (uint32_t d = 1; d < 64; d *= 2) {
        const uint32_t v = __shfl_up(upto, d);
        upto += lane >= d ? v : 0;
    }
    if (lane == 63) s.wave[wave] = upto;
    __syncthreads();
    uint32_t start = upto - own, all = 0;
    for (uint32_t w = 0; w < WAVES; w++) {
        start += w < wave ? s.wave[w] : 0;
        all += s.wave[w];
    }
    if (blockIdx.x == 0) {
        if (threadIdx.x < a.experts) a.starts[threadIdx.x] = (int32_t)start;
        if (threadIdx.x == 0) a.starts[a.experts] = (int32_t)all;
    }
    if (threadIdx.x < a.experts) start += s.start[threadIdx.x];
    // ranks within the wave's run
    const uint32_t each = (pairs + THREADS - 1) / THREADS * 64;
    uint32_t id[PER_WAVE], rank[PER_WAVE];
#pragma unroll
    for (uint32_t q = 0; q < PER_WAVE; q++) {
        const uint32_t i = wave * each + 64 * q + lane;
        if (64 * q >= each) break;
        id[q] = i < pairs ? s.id[i] : 0xffff;
        const bool there = id[q] < a.experts;
        const uint64_t same = same_as_mine(there ? id[q] : a.experts, bits), below = same & ((1ull << lane) - 1);
        rank[q] = 0;
        if (there) {
            rank[q] = counts[wave * a.padded + id[q]] + (uint32_t)__popcll(below);
            if (!(same >> lane >> 1)) counts[wave * a.padded + id[q]] = rank[q] + 1;
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (threadIdx.x < a.experts)
        for (uint32_t w = 0; w < WAVES; w++) {
            const uint32_t n = counts[w * a.padded + threadIdx.x];
            counts[w * a.padded + threadIdx.x] = start;
            start += n;
        }
    __syncthreads();
#pragma unroll
    for (uint32_t q = 0; q < PER_WAVE; q++) {
        const uint32_t i = wave * each + 64 * q + lane;
        if (64 * q >= each || i >= pairs) break;
        int32_t at = -1;
        if (id[q] < a.experts) {
            at = (int32_t)(counts[wave * a.padded + id[q]] + rank[q]);
            a.rows[at] = (int32_t)((first + i) / a.top);
        }
        a.place[first + i] = at;
    }
    for (uint32_t i = all + blockIdx.x * THREADS + threadIdx.x; i < a.tokens * a.top; i += gridDim.x * THREADS) a.rows[i] = -1;
}

// Over the 32 or 64 lanes of a token, the result in all of them: pairs, pairs of pairs, ... exchange what they have, so sums too are the same bits in every
// lane (turning the rows would add up in another order in each, and equal logits would get unequal scores).
template <int CTRL>
__device__ inline uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

template <int CTRL>
__device__ inline double moved(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)moved<CTRL>((uint32_t)(b >> 32)) << 32 | moved<CTRL>((uint32_t)b));
}

// The neighbour's row (HALF false) or half of the wave, in either place of the two results.
template <bool HALF>
__device__ inline void exchanged(uint32_t v, uint32_t &one, uint32_t &other)
{
    const auto r = HALF ? __builtin_amdgcn_permlane32_swap(v, v, false, false) : __builtin_amdgcn_permlane16_swap(v, v, false, false);
    one = r[0];
    other = r[1];
}

template <bool HALF>
__device__ inline void exchanged(double v, double &one, double &other)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    uint32_t lo[2], hi[2];
    exchanged<HALF>((uint32_t)b, lo[0], lo[1]);
    exchanged<HALF>((uint32_t)(b >> 32), hi[0], hi[1]);
    one = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]);
    other = __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}

template <int LANES, class T, class F>
__device__ inline T join(T v, F f)
{
    v = f(v, moved<0xb1>(v));
    v = f(v, moved<0x4e>(v));
    v = f(v, moved<0x141>(v));
    v = f(v, moved<0x140>(v));
    T one, other;
    exchanged<false>(v, one, other);
    v = f(one, other);
    if (LANES == 64) {
        exchanged<true>(v, one, other);
        v = f(one, other);
    }
    return v;
}

template <int LANES>
__device__ inline uint32_t most_of(uint32_t v)
{
    return join<LANES>(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}

template <int LANES>
__device__ inline double sum_of(double v)
{
    return join<LANES>(v, [](double x, double y) { return x + y; });
}

// Numbers as whole numbers of the same order, above 0.
__device__ inline uint32_t ordered(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);      // (-0 as 0)
    return b >> 31 ? ~b : b | 0x80000000u;
}

__device__ inline uint64_t ordered(double v)                           // (not -0)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t hi = (uint32_t)(b >> 32), sign = (uint32_t)((int32_t)hi >> 31);
    return (uint64_t)(hi ^ (sign | 0x80000000u)) << 32 | ((uint32_t)b ^ sign);
}

constexpr uint32_t LEAST = 0x00100000;             // no finite number's upper 32 bits are below, -infinity's are

__device__ inline float finite(float v) { return v != v ? -INFINITY : v > FLT_MAX ? FLT_MAX : v; }

// (The reciprocal by two steps of Newton's from an estimate of 2^-22 or better; the last instruction puts 0 for infinity.)
__device__ inline double sigmoid(float v)
{
    const double y = 1.0 + exp(-(double)v);
    double r = __builtin_amdgcn_rcp(y);
    r = fma(fma(-y, r, 1.0), r, r);
    r = fma(fma(-y, r, 1.0), r, r);
    return __builtin_amdgcn_div_fixup(r, y, 1.0);
}

// The two best of a group.
struct Two {
    double best = -INFINITY, second = -INFINITY;

    __device__ void add(double v)
    {
        second = fmax(second, fmin(best, v));
        best = fmax(best, v);
    }

    template <int CTRL>
    __device__ void add_moved()
    {
        const double b = moved<CTRL>(best), s = moved<CTRL>(second);
        add(b);
        second = fmax(second, s);
    }

    template <bool HALF>
    __device__ void add_exchanged()
    {
        double b0, b1, s0, s1;
        exchanged<HALF>(best, b0, b1);
        exchanged<HALF>(second, s0, s1);
        best = fmax(b0, b1);
        second = fmax(fmin(b0, b1), fmax(s0, s1));
    }

    // over the 2, 4, ... lanes in a row that have a group together
    __device__ void over(uint32_t lanes)
    {
        if (lanes > 1) add_moved<0xb1>();
        if (lanes > 2) add_moved<0x4e>();
        if (lanes > 4) add_moved<0x141>();
        if (lanes > 8) add_moved<0x140>();
        if (lanes > 16) add_exchanged<false>();
        if (lanes > 32) add_exchanged<true>();
    }

    __device__ double worth() const { return second == -INFINITY ? best : best + second; }
};

// PER numbers of a row from the lane's first on, -infinity (`none`) behind the last expert.
template <int PER, class T>
__device__ inline void load_row(const T *row, uint32_t first, uint32_t experts, bool wide, float none, float (&v)[PER])
{
    constexpr int BYTES = PER * sizeof(T) < 16 ? PER * sizeof(T) : 16, EACH = BYTES / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(EACH)));
    if (wide) {                                                // (the experts end where a lane's do)
        const uint32_t from = first < experts ? first : 0;
#pragma unroll
        for (int p = 0; p < PER / EACH; p++) {
            const Piece w = *(const Piece *)(row + from + p * EACH);
#pragma unroll
            for (int i = 0; i < EACH; i++) v[p * EACH + i] = first < experts ? (float)w[i] : none;
        }
    } else
#pragma unroll
        for (int q = 0; q < PER; q++) {
            const uint32_t e = first + q;
            const float w = (float)row[e < experts ? e : experts - 1];
            v[q] = e < experts ? w : none;
        }
}

// Groups: none, of whole lanes (1, 2, 4, ...), of any size.
enum Groups { NONE, LANES_WHOLE, ANY };

// A token has 32 lanes, with more than 256 experts 64; lane l has the experts PER l ... PER l + PER - 1.  Scores and choices are taken in 64 bits, since neighbouring
// choices decide whole numbers: in 32, two libraries' exponentials would send a token to different experts now and then.  The largest choice
// is looked for by its upper 32 bits; the lower ones and the number decide only where several have the same (BF16 logits leave the lower half of a word
// free, so there the number is part of the key).  Weights are taken for the chosen ones alone, at the end.
// 8192 tokens, eight of 256 experts in groups: 12.0 us, bound by its instructions: 2.4 the rounds, 1.5 the groups, 2.1 the exponentials, 2 the launch; the rest loads and stores.
// One token a wave with the lane's experts 64 apart took 17.3, and both kinds of scores and of groups in one kernel 14.4 (spilled registers).
// 16 tokens, six of 64 experts, with the sorting: 5.7 us, one step after the other.
template <int LANES, int PER, Groups GROUPS, bool SIGMOID>
__global__ __launch_bounds__(THREADS) void ecfm_choose_kernel(const RouteArgs a)
{
    constexpr uint32_t AT_ONCE = THREADS / LANES, WORTHS = GROUPS != NONE ? AT_ONCE * 64 * 8 : 0;
    constexpr uint32_t VALUES = GROUPS == ANY ? AT_ONCE * LANES * PER * 8 : 0, COUNTS = WAVES * LANES * PER * 4;
    __shared__ SortSpace s;
    __shared__ __attribute__((aligned(16))) uint8_t room[(VALUES > COUNTS ? VALUES : COUNTS) + WORTHS];
    const uint32_t l = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const bool alone = a.chosen_by == 1;
    const uint32_t first = blockIdx.x * a.choose_tokens, n = a.tokens - first < a.choose_tokens ? a.tokens - first : a.choose_tokens;
    if (threadIdx.x < a.padded) s.total[threadIdx.x] = s.start[threadIdx.x] = 0;
    for (uint32_t i = threadIdx.x; i < n * a.top; i += THREADS) s.id[i] = 0xffff;
    __syncthreads();
    for (uint32_t i = slot; i < (n + 1) / 2 * 2; i += AT_ONCE) {        // (a wave's two tokens go together)
        const bool there = i < n;
        const int64_t line = (int64_t)(first + (there ? i : n - 1)) * a.stride;
        float x[PER];
        if (a.f32) load_row<PER>((const float *)a.logits + line, PER * l, a.experts, a.wide, -INFINITY, x);
        else load_row<PER>((const __bf16 *)a.logits + line, PER * l, a.experts, a.wide, -INFINITY, x);
        uint32_t hi[PER], lo[PER];
        for (int q = 0; q < PER; q++) {
            // the logits' order; two BF16 numbers differ in the upper half, and the lower one has the expert's number
            const uint32_t key = ordered(x[q]), e = PER * l + q;
            x[q] = finite(x[q]);
            hi[q] = x[q] == -INFINITY ? 0 : a.f32 ? ordered(x[q]) : (key & 0xffff0000u) | (0xffff - e);
            lo[q] = 0;
        }
        float most = 0;
        double sum = 1;
        if (!SIGMOID) {
            most = -FLT_MAX;
            for (int q = 0; q < PER; q++) most = fmaxf(most, x[q]);
            const uint32_t m = most_of<LANES>(ordered(most));
            most = __builtin_bit_cast(float, m >> 31 ? m & 0x7fffffffu : ~m);
        }
        if (a.bias || GROUPS != NONE || !SIGMOID) {
            double score[PER];
            if (SIGMOID)
                for (int q = 0; q < PER; q++) score[q] = sigmoid(x[q]);
            else {
                sum = 0;
                for (int q = 0; q < PER; q++) {
                    score[q] = x[q] == -INFINITY ? 0 : exp((double)x[q] - (double)most);
                    sum += score[q];
                }
                sum = sum_of<LANES>(sum);
                if (a.bias || GROUPS != NONE)
                    for (int q = 0; q < PER; q++) score[q] = score[q] / sum;
            }
            if (a.bias || GROUPS != NONE) {
                float bias[PER] = {};
                if (a.bias) load_row<PER>(a.bias, PER * l, a.experts, a.wide, 0.f, bias);
                for (int q = 0; q < PER; q++) {
                    // (a score is 0 or more, so the sum is not -0; -infinity for NaN)
                    score[q] = fmax(score[q] + (double)(x[q] == -INFINITY ? -INFINITY : bias[q]), -INFINITY);
                    const uint64_t key = ordered(score[q]);
                    hi[q] = (uint32_t)(key >> 32);
                    lo[q] = (uint32_t)key;
                }
            }
            if constexpr (GROUPS != NONE) {
                double *worths = (double *)(room + (VALUES > COUNTS ? VALUES : COUNTS)) + slot * 64;
                Two two;
                if (GROUPS == LANES_WHOLE) {                                 // a group is 1, 2, 4, ... lanes
                    for (int q = 0; q < PER; q++) two.add(score[q]);
                    two.over(a.lanes);
                    const uint32_t group = PER * l * a.per_size >> 20;
                    if ((l & (a.lanes - 1)) == 0 && group < a.groups) worths[group] = two.worth();
                } else {
                    double *values = (double *)room + slot * LANES * PER;
                    for (int q = 0; q < PER; q++) values[PER * l + q] = score[q];
                    __builtin_amdgcn_wave_barrier();
                    __threadfence_block();
                    const uint32_t share = a.groups >= LANES ? 1 : LANES >> (32 - __builtin_clz(a.groups - 1));
                    for (uint32_t g0 = 0; g0 < a.groups; g0 += LANES / share) {
                        const uint32_t g = g0 + l / share;
                        two = Two();
                        if (g < a.groups)
                            for (uint32_t j = l % share; j < a.size; j += share) two.add(values[g * a.size + j]);
                        two.over(share);
                        if (l % share == 0 && g < a.groups) worths[g] = two.worth();
                    }
                }
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
                // lane l looks at group l, and at l + 32
                uint64_t open = 0;
                for (uint32_t g0 = 0; g0 < a.groups; g0 += LANES) {
                    const uint32_t g = g0 + l;
                    const double own = worths[g < a.groups ? g : 0];
                    uint32_t better = 0;
                    for (uint32_t o = 0; o < a.groups; o++) {
                        const double v = worths[o];
                        better += (v > own) | ((v == own) & (o < g));
                    }
                    uint64_t m = __ballot(g < a.groups && better < a.top_groups);
                    if (LANES == 32) m = (threadIdx.x & 32 ? m >> 32 : m & 0xffffffffu) << g0;
                    open |= m;
                }
                if (GROUPS == LANES_WHOLE) {
                    const bool shut = !(open >> (PER * l * a.per_size >> 20 & 63) & 1);
                    for (int q = 0; q < PER; q++) hi[q] = shut ? 0 : hi[q];
                } else
                    for (int q = 0; q < PER; q++) hi[q] = open >> ((PER * l + q) * a.per_size >> 20 & 63) & 1 ? hi[q] : 0;
                __builtin_amdgcn_wave_barrier();
            }
        }
        // Round after round the largest key, whose place then holds the number of the round.
        for (uint32_t j = 1; j <= a.top; j++) {
            uint32_t best = hi[0];
            for (int q = 1; q < PER; q++) best = hi[q] > best ? hi[q] : best;
            best = most_of<LANES>(best);
            const uint64_t live = __ballot(best >= LEAST);
            if (!live) break;                                  // nobody is left
            best = best >= LEAST ? best : ~0u;                // (which nobody has)
            uint32_t found = 0;
            for (int q = 0; q < PER; q++) found += (uint32_t)__popcll(__ballot(hi[q] == best));
            if (found * LANES != (uint32_t)__popcll(live)) {   // several: by the lower halves, then the lowest number
                uint32_t low = 0;
                for (int q = 0; q < PER; q++) low = hi[q] == best && lo[q] > low ? lo[q] : low;
                low = most_of<LANES>(low);
                uint32_t at = 0;
                for (int q = PER - 1; q >= 0; q--) at = hi[q] == best && lo[q] == low ? MAX_EXPERTS - (PER * l + q) : at;
                at = MAX_EXPERTS - most_of<LANES>(at);
                for (int q = 0; q < PER; q++) hi[q] = at == PER * l + q ? j : hi[q];
            } else
                for (int q = 0; q < PER; q++) hi[q] = hi[q] == best ? j : hi[q];
        }
        for (int q = 0; q < PER; q++)
            if (hi[q] - 1 < a.top && there) s.id[i * a.top + hi[q] - 1] = (uint16_t)(PER * l + q);
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
        const bool mine = there && l < a.top;
        const uint32_t id = mine ? s.id[i * a.top + l] : 0xffff;
        double w = 0;
        if (id < a.experts) {
            const float v = finite(a.f32 ? ((const float *)a.logits)[line + id] : (float)((const __bf16 *)a.logits)[line + id]);
            w = SIGMOID ? sigmoid(v) : exp((double)v - (double)most) / sum;
        }
        if (a.normalise) {
            const double total = sum_of<LANES>(w);
            w = total > 0 ? w / total : 0;
        }
        if (mine) {
            const uint64_t at = (uint64_t)(first + i) * a.top + l;
            a.ids[at] = id < a.experts ? (int32_t)id : -1;
            a.weights[at] = (float)(w * (double)a.scale);
            if (id < a.experts) atomicAdd(&s.total[id], 1u);   // (whole numbers: in any order)
        }
    }
    __syncthreads();
    if (alone) place_pairs(a, s, (uint32_t *)room, 0, n * a.top);
    else if (threadIdx.x < a.padded) a.counts[(uint64_t)blockIdx.x * a.padded + threadIdx.x] = (uint16_t)s.total[threadIdx.x];
}

// Where many workgroups chose (MOST_TOKENS each, as many as sort): of each expert, the pairs before each workgroup that sorts, and of all.
__global__ __launch_bounds__(THREADS) void ecfm_sum_kernel(const RouteArgs a)
{
    __shared__ uint32_t part[WAVES][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const uint32_t each = (a.sorted_by + WAVES - 1) / WAVES, lo = wave * each < a.sorted_by ? wave * each : a.sorted_by, hi = lo + each < a.sorted_by ? lo + each : a.sorted_by;
    uint32_t n = 0;
    if (e < a.experts)
#pragma unroll 16
        for (uint32_t b = lo; b < hi; b++) n += a.counts[(uint64_t)b * a.padded + e];
    part[wave][lane] = n;
    __syncthreads();
    uint32_t at = 0, all = 0;
    for (uint32_t w = 0; w < WAVES; w++) {
        at += w < wave ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (e >= a.experts) return;
#pragma unroll 16
    for (uint32_t b = lo; b < hi; b++) {
        a.sums[(uint64_t)b * a.padded + e] = at;
        at += a.counts[(uint64_t)b * a.padded + e];
    }
    if (wave == 0) a.sums[(uint64_t)a.sorted_by * a.padded + e] = all;
}

template <bool SUMMED>
__global__ __launch_bounds__(THREADS) void ecfm_sort_kernel(const RouteArgs a)
{
    __shared__ SortSpace s;
    __shared__ uint32_t counts[WAVES * MAX_EXPERTS];
    const uint32_t token = blockIdx.x * a.sort_tokens, pairs = (a.tokens - token < a.sort_tokens ? a.tokens - token : a.sort_tokens) * a.top;
    for (uint32_t i = threadIdx.x; i < pairs; i += THREADS) s.id[i] = (uint16_t)a.ids[token * a.top + i];
    if (SUMMED) {
        if (threadIdx.x < a.experts) {
            s.start[threadIdx.x] = a.sums[(uint64_t)blockIdx.x * a.padded + threadIdx.x];
            s.total[threadIdx.x] = a.sums[(uint64_t)a.sorted_by * a.padded + threadIdx.x];
        }
    } else {
        // Eight experts a thread, every so many workgroups' counts, two to a word as they were written: an expert has at most one of a token's
        // pairs, so up to SUMS_16 tokens no sum passes 16 bits.  Words of neighbouring threads lie side by side in LDS.
        const uint32_t eights = a.padded / 8, lines = THREADS / eights, line = threadIdx.x / eights, e = threadIdx.x % eights;
        uint32_t *all = counts, *before = counts + 4 * eights;
        for (uint32_t i = threadIdx.x; i < 8 * eights; i += THREADS) counts[i] = 0;
        __syncthreads();
        if (line < lines) {
            const uint32_t mine = blockIdx.x * (a.sort_tokens / a.choose_tokens);
            u32x4 sum = {}, below = {};
#pragma unroll 4
            for (uint32_t b = line; b < a.chosen_by; b += lines) {
                const u32x4 v = *(const u32x4 *)(a.counts + (uint64_t)b * a.padded + 8 * e);
                sum += v;
                below += b < mine ? v : u32x4{};
            }
            for (uint32_t i = 0; i < 4; i++) {                 // (whole numbers: in any order)
                if (sum[i]) atomicAdd(&all[i * eights + e], sum[i]);
                if (below[i]) atomicAdd(&before[i * eights + e], below[i]);
            }
        }
        __syncthreads();
        if (threadIdx.x < a.padded) {
            const uint32_t at = threadIdx.x % 8 / 2 * eights + threadIdx.x / 8, half = threadIdx.x % 2 * 16;
            s.total[threadIdx.x] = all[at] >> half & 0xffff;
            s.start[threadIdx.x] = before[at] >> half & 0xffff;
        }
    }
    __syncthreads();
    place_pairs(a, s, counts, token * a.top, pairs);
}

template <Groups GROUPS, bool SIGMOID>
void choose(const RouteArgs &a, hipStream_t s)
{
    const dim3 grid(a.chosen_by), block(THREADS);
    if (a.experts <= 64) hipLaunchKernelGGL((ecfm_choose_kernel<32, 2, GROUPS, SIGMOID>), grid, block, 0, s, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((ecfm_choose_kernel<32, 4, GROUPS, SIGMOID>), grid, block, 0, s, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((ecfm_choose_kernel<32, 8, GROUPS, SIGMOID>), grid, block, 0, s, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((ecfm_choose_kernel<64, 8, GROUPS, SIGMOID>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ecfm_choose_kernel<64, 16, GROUPS, SIGMOID>), grid, block, 0, s, a);
}

template <Groups GROUPS>
void choose(const RouteArgs &a, hipStream_t s)
{
    if (a.sigmoid) choose<GROUPS, true>(a, s);
    else choose<GROUPS, false>(a, s);
}

// Tokens of a workgroup that chooses.  Few where there are more compute units, of which each then is done sooner (512 tokens of 256 experts 17.2 -> 13.0 us),
// but not many workgroups of a few, since their counts are read again (1024 by 4: 15.4, by 8: 14.0).  Where there are more tokens than all take at
// once, as many times what one does that the compute units are done soonest: 12000 by 32 33.2, by 64 29.5.
uint32_t choose_tokens(uint32_t tokens, uint32_t experts)
{
    const uint32_t once = THREADS / (experts <= HALF_WAVE ? 32 : 64);
    if (tokens <= once) return once;
    for (uint32_t n = 4; n < once; n *= 2)
        if (tokens <= n * (n == 4 ? CUS / 2 : CUS)) return n;
    uint32_t best = MOST_TOKENS, least = ~0u;
    for (uint32_t n = once; n <= MOST_TOKENS; n += once) {
        const uint32_t groups = (tokens + n - 1) / n, passes = (groups + CUS - 1) / CUS * (n / once);
        if ((groups <= ADD_UP || n == MOST_TOKENS) && passes <= least) {
            least = passes;
            best = n;
        }
    }
    return best;
}

uint32_t choosers(uint32_t tokens, uint32_t experts)
{
    const uint32_t n = choose_tokens(tokens, experts);
    return tokens <= n ? 1 : (tokens + n - 1) / n;
}

uint32_t sort_tokens(uint32_t tokens, uint32_t experts)
{
    const uint32_t n = choose_tokens(tokens, experts);
    return n < 32 ? 32 : n;
}

uint32_t sorters(uint32_t tokens, uint32_t experts)
{
    const uint32_t n = sort_tokens(tokens, experts);
    return (tokens + n - 1) / n;
}

uint32_t padded(uint32_t experts) { return (experts + 7) / 8 * 8; }
uint64_t counts_bytes(uint32_t tokens, uint32_t experts) { return ((uint64_t)choosers(tokens, experts) * padded(experts) * 2 + 15) / 16 * 16; }

bool bad(uint32_t tokens, uint32_t experts, uint32_t top)
{
    return experts == 0 || experts > MAX_EXPERTS || top == 0 || top > MAX_TOP || top > experts || tokens > (1u << 22);
}

} // namespace
} // namespace ecfm

using namespace ecfm;

extern "C" {

uint64_t ecfm_route_workspace_bytes(uint32_t n_tokens, uint32_t experts, uint32_t top)
{
    if (bad(n_tokens, experts, top)) return 0;
    if (choosers(n_tokens, experts) == 1) return 0;
    return counts_bytes(n_tokens, experts) + (n_tokens > SUMS_16 ? (uint64_t)(sorters(n_tokens, experts) + 1) * padded(experts) * 4 : 0);
}

int ecfm_route(const ecfm_route_opts *o, int32_t *d_ids, float *d_weights, int32_t *d_starts, int32_t *d_rows, int32_t *d_place,
               void *d_workspace, uint64_t workspace_bytes, void *stream)
{
    if (!o || bad(o->n_tokens, o->experts, o->top) || (o->dtype != ECFA_F32 && o->dtype != ECFA_BF16) || o->sigmoid > 1 || o->normalise > 1
        || !std::isfinite(o->scale))
        return ECF8_E_ARG;
    if (o->groups == 0 || o->groups > 64 || o->experts % o->groups || o->top_groups == 0 || o->top_groups > o->groups
        || o->top > o->experts / o->groups * o->top_groups)
        return ECF8_E_ARG;
    if (!d_starts || (o->n_tokens && (!o->d_logits || !d_ids || !d_weights || !d_rows || !d_place))) return ECF8_E_ARG;
    const uintptr_t e = o->dtype == ECFA_F32 ? 4 : 2;
    if (((uintptr_t)o->d_logits & (e - 1)) || ((uintptr_t)o->d_bias & 3) || ((uintptr_t)d_ids & 3) || ((uintptr_t)d_weights & 3) || ((uintptr_t)d_starts & 3)
        || ((uintptr_t)d_rows & 3) || ((uintptr_t)d_place & 3) || ((uintptr_t)d_workspace & 15))
        return ECF8_E_ALIGN;
    const uint64_t need = ecfm_route_workspace_bytes(o->n_tokens, o->experts, o->top);
    if (need && (!d_workspace || workspace_bytes < need)) return ECF8_E_CAPACITY;
    RouteArgs a{};
    a.logits = o->d_logits;
    a.bias = o->d_bias;
    a.stride = o->n_tokens > 1 ? o->logit_stride : 0;
    a.ids = d_ids;
    a.starts = d_starts;
    a.rows = d_rows;
    a.place = d_place;
    a.weights = d_weights;
    a.counts = (uint16_t *)d_workspace;
    a.sums = (uint32_t *)((uint8_t *)d_workspace + counts_bytes(o->n_tokens, o->experts));
    a.tokens = o->n_tokens;
    a.experts = o->experts;
    a.top = o->top;
    a.sigmoid = o->sigmoid;
    a.normalise = o->normalise;
    a.groups = o->groups;
    a.top_groups = o->top_groups;
    a.f32 = o->dtype == ECFA_F32;
    a.scale = o->scale;
    a.chosen_by = choosers(o->n_tokens, o->experts);           // (no tokens: the starts are written all the same)
    a.choose_tokens = choose_tokens(o->n_tokens, o->experts);
    a.sort_tokens = sort_tokens(o->n_tokens, o->experts);
    a.sorted_by = sorters(o->n_tokens, o->experts);
    a.padded = padded(o->experts);
    // as many lanes a token and experts a lane as the kernel has
    const uint32_t per = a.experts <= 64 ? 2 : a.experts <= 128 ? 4 : a.experts <= 512 ? 8 : 16, bytes = per * (uint32_t)e < 16 ? per * (uint32_t)e : 16, bias_bytes = per * 4 < 16 ? per * 4 : 16;
    a.wide = a.experts % per == 0 && (uintptr_t)a.logits % bytes == 0 && a.stride * (int64_t)e % bytes == 0 && (uintptr_t)a.bias % bias_bytes == 0;
    a.size = a.experts / a.groups;
    a.per_size = ((1u << 20) + a.size - 1) / a.size;
    a.lanes = a.size % per ? 0 : a.size / per;
    if (a.lanes & (a.lanes - 1)) a.lanes = 0;
    hipStream_t s = (hipStream_t)stream;
    if (a.groups == 1) choose<NONE>(a, s);
    else if (a.lanes) choose<LANES_WHOLE>(a, s);
    else choose<ANY>(a, s);
    if (a.tokens > SUMS_16) {
        hipLaunchKernelGGL(ecfm_sum_kernel, dim3((a.experts + 63) / 64), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(ecfm_sort_kernel<true>, dim3(a.sorted_by), dim3(THREADS), 0, s, a);
    } else if (a.chosen_by > 1) hipLaunchKernelGGL(ecfm_sort_kernel<false>, dim3(a.sorted_by), dim3(THREADS), 0, s, a);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

} // extern "C"
