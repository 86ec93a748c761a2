// From a router's logits to experts, their weights, and the pairs (token, expert) sorted by expert (ecfm.h).
#include "ecfm_device.h"

#include <cfloat>
#include <cmath>

namespace ecfm {
namespace {

constexpr uint32_t WAVES = 16, THREADS = 64 * WAVES, MAX_TOP = 32, MAX_EXPERTS = 1024;
constexpr uint32_t ONE_BLOCK = 64;                 // up to as many tokens one workgroup does everything
constexpr uint32_t CHOOSE_TOKENS = 32;             // of a workgroup that chooses
constexpr uint32_t SORT_TOKENS = 128;              // of a workgroup that sorts
constexpr uint32_t ADD_UP = 512;                   // up to as many workgroups that choose, each one that sorts adds up all their counts by itself
constexpr uint32_t SLOTS = SORT_TOKENS * MAX_TOP, PER_WAVE = SLOTS / THREADS;

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
    uint32_t padded;                               // experts, rounded up to a multiple of 8
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
// before.  No atomics, so the order is that of the tokens (8192 x 8 pairs 8.5 us; each expert looking through all pairs 49).  counts: [WAVES][padded] of LDS.
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

// Over the lanes of a wave, by moves along the rows of 16 and from row to row; the result is lane 63's.
template <int CTRL, int ROWS>
__device__ inline uint32_t moved(uint32_t v, uint32_t none)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}

template <class F>
__device__ inline uint32_t wave_join(uint32_t v, uint32_t none, F join)
{
    v = join(v, moved<0x111, 0xf>(v, none));
    v = join(v, moved<0x112, 0xf>(v, none));
    v = join(v, moved<0x114, 0xf>(v, none));
    v = join(v, moved<0x118, 0xf>(v, none));
    v = join(v, moved<0x142, 0xa>(v, none));
    v = join(v, moved<0x143, 0xc>(v, none));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ inline uint32_t wave_most(uint32_t v)
{
    return wave_join(v, 0, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}

template <int CTRL, int ROWS>
__device__ inline double plus_moved(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t m = (uint64_t)moved<CTRL, ROWS>((uint32_t)(b >> 32), 0) << 32 | moved<CTRL, ROWS>((uint32_t)b, 0);
    return v + __builtin_bit_cast(double, m);
}

__device__ inline double of_lane(double v, uint32_t lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t r = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane);
    return __builtin_bit_cast(double, r);
}

__device__ inline double wave_sum(double v)
{
    v = plus_moved<0x111, 0xf>(v);
    v = plus_moved<0x112, 0xf>(v);
    v = plus_moved<0x114, 0xf>(v);
    v = plus_moved<0x118, 0xf>(v);
    v = plus_moved<0x142, 0xa>(v);
    v = plus_moved<0x143, 0xc>(v);
    return of_lane(v, 63);
}

// Numbers as whole numbers of the same order, above 0.
__device__ inline uint32_t ordered(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);      // (-0 as 0)
    return b >> 31 ? ~b : b | 0x80000000u;
}

__device__ inline uint64_t ordered(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);
    return b >> 63 ? ~b : b | 1ull << 63;
}

// A wave takes a token: lane l has the experts l, l + 64, ...  Scores and choices are taken in 64 bits, since neighbouring choices decide whole numbers: in
// 32, two libraries' exponentials would send a token to different experts now and then.  The largest choice is looked for by its upper 32 bits;
// the lower ones and the number decide only where lanes have the same.  8192 tokens, eight of 256 experts in groups: 17.9 us, bound by its instructions (exponentials in
// 64 bits, eight searches over the wave); 16 tokens, six of 64 experts, with the sorting: 6.2 us, one after the other.
template <int PER, bool GROUPS>
__global__ __launch_bounds__(THREADS) void ecfm_choose_kernel(const RouteArgs a)
{
    constexpr uint32_t KEYS = GROUPS ? WAVES * 64 * PER * 8 : 0, COUNTS = WAVES * 64 * PER * 4;
    __shared__ SortSpace s;
    __shared__ __attribute__((aligned(16))) uint8_t room[KEYS > COUNTS ? KEYS : COUNTS];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool alone = a.chosen_by == 1;
    const uint32_t first = blockIdx.x * CHOOSE_TOKENS, n = alone ? a.tokens : a.tokens - first < CHOOSE_TOKENS ? a.tokens - first : CHOOSE_TOKENS;
    if (threadIdx.x < a.padded) s.total[threadIdx.x] = s.start[threadIdx.x] = 0;
    float bias[PER], ahead[PER];
    for (int q = 0; q < PER; q++) bias[q] = a.bias && lane + 64 * q < a.experts ? a.bias[lane + 64 * q] : 0.f;
    const auto load = [&](uint32_t i) {
        for (int q = 0; q < PER; q++) {
            const uint32_t e = lane + 64 * q;
            const int64_t at = (int64_t)(first + i) * a.stride + e;
            ahead[q] = -INFINITY;
            if (e < a.experts && i < n) ahead[q] = a.f32 ? ((const float *)a.logits)[at] : (float)((const __bf16 *)a.logits)[at];
        }
    };
    load(wave);
    __syncthreads();
    for (uint32_t i = wave; i < n; i += WAVES) {
        const uint32_t t = first + i;
        double score[PER];
        uint64_t key[PER];
        float x[PER], most = -FLT_MAX;
        for (int q = 0; q < PER; q++) {
            x[q] = ahead[q] != ahead[q] ? -INFINITY : ahead[q] > FLT_MAX ? FLT_MAX : ahead[q];
            most = fmaxf(most, x[q]);
        }
        load(i + WAVES);
        double sum = 0;
        if (a.sigmoid)
            for (int q = 0; q < PER; q++) score[q] = 1.0 / (1.0 + exp(-(double)x[q]));
        else {
            const uint32_t m = wave_most(ordered(most));
            most = __builtin_bit_cast(float, m >> 31 ? m & 0x7fffffffu : ~m);
            for (int q = 0; q < PER; q++) {
                score[q] = x[q] == -INFINITY ? 0 : exp((double)x[q] - (double)most);
                sum += score[q];
            }
            sum = wave_sum(sum);
            for (int q = 0; q < PER; q++) score[q] = score[q] / sum;
        }
        for (int q = 0; q < PER; q++) {
            const double c = score[q] + (double)bias[q];
            key[q] = a.bias || GROUPS ? ordered(c) : (uint64_t)ordered(x[q]) << 32;
            if (x[q] == -INFINITY || c != c || c == -INFINITY) key[q] = 0;
        }
        if constexpr (GROUPS) {
            // Equal numbers of lanes look for a group's two best and compare notes
            double(*keys)[64 * PER] = (double(*)[64 * PER])room;
            for (int q = 0; q < PER; q++) keys[wave][lane + 64 * q] = key[q] ? score[q] + (double)bias[q] : -INFINITY;
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
            const uint32_t size = a.experts / a.groups, share = 64 >> (32 - __builtin_clz(a.groups - 1)), group = lane / share;
            double best = -INFINITY, second = -INFINITY;
            if (group < a.groups)
                for (uint32_t j = lane % share; j < size; j += share) {
                    const double v = keys[wave][group * size + j];
                    second = fmax(second, fmin(best, v));
                    best = fmax(best, v);
                }
            for (uint32_t d = 1; d < share; d *= 2) {
                const double b2 = __shfl_xor(best, d), s2 = __shfl_xor(second, d);
                second = fmax(fmin(best, b2), fmax(second, s2));
                best = fmax(best, b2);
            }
            const double worth = second == -INFINITY ? best : best + second;
            uint32_t better = 0;
            for (uint32_t o = 0; o < a.groups; o++) {
                const double v = of_lane(worth, o * share);
                better += v > worth || (v == worth && o < group);
            }
            const uint64_t open = __ballot(group < a.groups && better < a.top_groups);
            for (int q = 0; q < PER; q++) {
                const uint32_t e = lane + 64 * q;
                if (e >= a.experts || !(open >> (e / size * share) & 1)) key[q] = 0;
            }
            __builtin_amdgcn_wave_barrier();
        }
        int32_t id = -1;
        double got = 0, total = 0;
        for (uint32_t j = 0; j < a.top; j++) {
            uint64_t k = key[0];
            uint32_t e = lane;
            for (int q = 1; q < PER; q++)
                if (key[q] > k) {
                    k = key[q];
                    e = lane + 64 * q;
                }
            const uint32_t hi = (uint32_t)(k >> 32), hi_most = wave_most(hi);
            if (hi_most == 0) break;                           // nobody is left
            uint64_t who = __ballot(hi == hi_most);
            if (who & (who - 1)) {
                const uint32_t lo = hi == hi_most ? (uint32_t)k : 0, lo_most = wave_most(lo);
                who = __ballot(hi == hi_most && lo == lo_most);
                if (who & (who - 1)) {                         // the lowest number
                    const uint32_t low = ~wave_most(who >> lane & 1 ? ~e : 0);
                    who = 1ull << (low & 63);
                }
            }
            const uint32_t at_lane = (uint32_t)__ffsll((unsigned long long)who) - 1, at = (uint32_t)__builtin_amdgcn_readlane((int)e, at_lane);
            double w = 0;
            for (int q = 0; q < PER; q++)
                if (at / 64 == (uint32_t)q) {                  // (the same for all lanes)
                    w = of_lane(score[q], at_lane);
                    key[q] = lane == at_lane ? 0 : key[q];
                }
            total += w;
            if (lane == j) {
                id = (int32_t)at;
                got = w;
            }
        }
        if (a.normalise) got = total > 0 ? got / total : 0;
        if (lane < a.top) {
            a.ids[(uint64_t)t * a.top + lane] = id;
            a.weights[(uint64_t)t * a.top + lane] = (float)(got * (double)a.scale);
            s.id[i * a.top + lane] = id < 0 ? 0xffff : (uint16_t)id;
            if (id >= 0) atomicAdd(&s.total[id], 1u);          // (whole numbers: in any order)
        }
    }
    __syncthreads();
    if (alone) place_pairs(a, s, (uint32_t *)room, 0, n * a.top);
    else if (threadIdx.x < a.padded) a.counts[(uint64_t)blockIdx.x * a.padded + threadIdx.x] = (uint16_t)s.total[threadIdx.x];
}

// Where many workgroups chose: of each expert, the pairs before each workgroup that sorts, and of all.
__global__ __launch_bounds__(THREADS) void ecfm_sum_kernel(const RouteArgs a)
{
    constexpr uint32_t PER = SORT_TOKENS / CHOOSE_TOKENS;
    __shared__ uint32_t part[WAVES][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const uint32_t each = (a.sorted_by + WAVES - 1) / WAVES, lo = wave * each < a.sorted_by ? wave * each : a.sorted_by, hi = lo + each < a.sorted_by ? lo + each : a.sorted_by;
    const auto of_block = [&](uint32_t b) {
        uint32_t n = 0;
        for (uint32_t i = b * PER; i < (b + 1) * PER && i < a.chosen_by; i++) n += a.counts[(uint64_t)i * a.padded + e];
        return n;
    };
    uint32_t n = 0;
    if (e < a.experts)
        for (uint32_t b = lo; b < hi; b++) n += of_block(b);
    part[wave][lane] = n;
    __syncthreads();
    uint32_t at = 0, all = 0;
    for (uint32_t w = 0; w < WAVES; w++) {
        at += w < wave ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (e >= a.experts) return;
    for (uint32_t b = lo; b < hi; b++) {
        a.sums[(uint64_t)b * a.padded + e] = at;
        at += of_block(b);
    }
    if (wave == 0) a.sums[(uint64_t)a.sorted_by * a.padded + e] = all;
}

template <bool SUMMED>
__global__ __launch_bounds__(THREADS) void ecfm_sort_kernel(const RouteArgs a)
{
    constexpr uint32_t PER = SORT_TOKENS / CHOOSE_TOKENS;
    __shared__ SortSpace s;
    __shared__ uint32_t counts[WAVES * MAX_EXPERTS];
    const uint32_t token = blockIdx.x * SORT_TOKENS, pairs = (a.tokens - token < SORT_TOKENS ? a.tokens - token : SORT_TOKENS) * a.top;
    for (uint32_t i = threadIdx.x; i < pairs; i += THREADS) s.id[i] = (uint16_t)a.ids[token * a.top + i];
    if (SUMMED) {
        if (threadIdx.x < a.experts) {
            s.start[threadIdx.x] = a.sums[(uint64_t)blockIdx.x * a.padded + threadIdx.x];
            s.total[threadIdx.x] = a.sums[(uint64_t)a.sorted_by * a.padded + threadIdx.x];
        }
    } else {
        if (threadIdx.x < a.padded) s.start[threadIdx.x] = s.total[threadIdx.x] = 0;
        __syncthreads();
        // eight experts a thread, every so many workgroups' counts
        const uint32_t eights = a.padded / 8, lines = THREADS / eights, line = threadIdx.x / eights, e = threadIdx.x % eights * 8;
        uint32_t before[8] = {}, all[8] = {};
        if (line < lines) {
#pragma unroll 4
            for (uint32_t b = line; b < a.chosen_by; b += lines) {
                const u32x4 v = *(const u32x4 *)(a.counts + (uint64_t)b * a.padded + e);
                for (uint32_t i = 0; i < 8; i++) {
                    const uint32_t n = v[i / 2] >> i % 2 * 16 & 0xffff;
                    all[i] += n;
                    before[i] += b < blockIdx.x * PER ? n : 0;
                }
            }
            for (uint32_t i = 0; i < 8; i++) {                 // (whole numbers: in any order)
                if (all[i]) atomicAdd(&s.total[e + i], all[i]);
                if (before[i]) atomicAdd(&s.start[e + i], before[i]);
            }
        }
    }
    __syncthreads();
    place_pairs(a, s, counts, token * a.top, pairs);
}

template <bool GROUPS>
void choose(const RouteArgs &a, hipStream_t s)
{
    const dim3 grid(a.chosen_by), block(THREADS);
    if (a.experts <= 64) hipLaunchKernelGGL((ecfm_choose_kernel<1, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((ecfm_choose_kernel<2, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((ecfm_choose_kernel<4, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((ecfm_choose_kernel<8, GROUPS>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ecfm_choose_kernel<16, GROUPS>), grid, block, 0, s, a);
}

uint32_t choosers(uint32_t tokens) { return tokens <= ONE_BLOCK ? 1 : (tokens + CHOOSE_TOKENS - 1) / CHOOSE_TOKENS; }
uint32_t sorters(uint32_t tokens) { return (tokens + SORT_TOKENS - 1) / SORT_TOKENS; }
uint32_t padded(uint32_t experts) { return (experts + 7) / 8 * 8; }
uint64_t counts_bytes(uint32_t tokens, uint32_t experts) { return ((uint64_t)choosers(tokens) * padded(experts) * 2 + 15) / 16 * 16; }

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
    if (choosers(n_tokens) == 1) return 0;
    return counts_bytes(n_tokens, experts) + (choosers(n_tokens) > ADD_UP ? (uint64_t)(sorters(n_tokens) + 1) * padded(experts) * 4 : 0);
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
    a.chosen_by = choosers(o->n_tokens);           // (no tokens: the starts are written all the same)
    a.sorted_by = sorters(o->n_tokens);
    a.padded = padded(o->experts);
    hipStream_t s = (hipStream_t)stream;
    if (a.groups > 1) choose<true>(a, s);
    else choose<false>(a, s);
    if (a.chosen_by > ADD_UP) {
        hipLaunchKernelGGL(ecfm_sum_kernel, dim3((a.experts + 63) / 64), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL(ecfm_sort_kernel<true>, dim3(a.sorted_by), dim3(THREADS), 0, s, a);
    } else if (a.chosen_by > 1) hipLaunchKernelGGL(ecfm_sort_kernel<false>, dim3(a.sorted_by), dim3(THREADS), 0, s, a);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

} // extern "C"
