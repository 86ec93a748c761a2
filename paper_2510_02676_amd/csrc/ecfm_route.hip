// From a router's logits to experts, their weights, and the pairs (token, expert) sorted by expert (ecfm.h).
#include "ecfm_device.h"

#include <cfloat>
#include <cmath>

namespace ecfm {
namespace {

constexpr uint32_t ROUTE_WAVES = 16, ROUTE_THREADS = 64 * ROUTE_WAVES, ROUTE_TOKENS = 64, MAX_TOP = 32, MAX_EXPERTS = 1024;
constexpr uint32_t SLOTS = ROUTE_TOKENS * MAX_TOP;

struct RouteArgs {
    const void *logits;
    const float *bias;
    int64_t stride;
    int32_t *ids, *starts, *rows, *place;
    float *weights;
    uint32_t *counts;                              // [blocks][experts]: pairs of a block of tokens; behind them [experts]: of all
    uint32_t tokens, experts, top, sigmoid, normalise, groups, top_groups, f32;
    uint32_t per_block, blocks;                    // tokens of a workgroup, workgroups
    uint32_t log_bins;                             // experts, rounded up to a power of two from 64 on
    float scale;
};

// Shared by the workgroup that sorts its tokens' pairs.
struct SortSpace {
    uint16_t id[SLOTS];
    uint32_t count[ROUTE_THREADS];                 // [segment][bin]
    uint32_t wave[ROUTE_WAVES];
};

// Pairs of a workgroup by expert, without atomics: thread (segment, expert) looks through its segment of the pairs.  Leaves the counts in
// s.count and returns this thread's segment.
__device__ inline void segment_of(const RouteArgs &a, uint32_t pairs, uint32_t *lo, uint32_t *hi)
{
    const uint32_t segments = ROUTE_THREADS >> a.log_bins, seg = threadIdx.x >> a.log_bins, each = (pairs + segments - 1) / segments;
    *lo = seg * each < pairs ? seg * each : pairs;
    *hi = *lo + each < pairs ? *lo + each : pairs;
}

__device__ inline void count_pairs(const RouteArgs &a, SortSpace &s, uint32_t pairs)
{
    const uint32_t e = threadIdx.x & ((1u << a.log_bins) - 1);
    uint32_t lo, hi, n = 0;
    segment_of(a, pairs, &lo, &hi);
    for (uint32_t i = lo; i < hi; i++) n += s.id[i] == e;
    s.count[threadIdx.x] = n;
    __syncthreads();
}

// The pairs of this workgroup to their places.  `before`: pairs of the same expert in workgroups before it, `total`: in all, both for the
// expert of threads below 2^log_bins.
__device__ inline void place_pairs(const RouteArgs &a, SortSpace &s, uint32_t first, uint32_t pairs, uint32_t before, uint32_t total)
{
    const uint32_t bins = 1u << a.log_bins, e = threadIdx.x & (bins - 1), seg = threadIdx.x >> a.log_bins, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = threadIdx.x < a.experts ? total : 0;
    const uint32_t own = upto;
    for (uint32_t d = 1; d < 64; d *= 2) {
        const uint32_t v = __shfl_up(upto, d);
        upto += lane >= d ? v : 0;
    }
    if (lane == 63) s.wave[wave] = upto;
    __syncthreads();
    uint32_t waves_before = 0, all = 0;
    for (uint32_t w = 0; w < ROUTE_WAVES; w++) {
        waves_before += w < wave ? s.wave[w] : 0;
        all += s.wave[w];
    }
    const uint32_t start = waves_before + upto - own;
    if (blockIdx.x == 0) {
        if (threadIdx.x < a.experts) a.starts[threadIdx.x] = (int32_t)start;
        if (threadIdx.x == 0) a.starts[a.experts] = (int32_t)all;
    }
    // counts become places: of a segment's first pair of an expert
    if (threadIdx.x < bins) {
        uint32_t at = start + before;
        for (uint32_t g = 0; g < ROUTE_THREADS >> a.log_bins; g++) {
            const uint32_t n = s.count[(g << a.log_bins) + e];
            s.count[(g << a.log_bins) + e] = at;
            at += n;
        }
    }
    __syncthreads();
    uint32_t lo, hi, at = s.count[(seg << a.log_bins) + e];
    segment_of(a, pairs, &lo, &hi);
    for (uint32_t i = lo; i < hi; i++)
        if (s.id[i] == e && e < a.experts) {
            a.rows[at] = (int32_t)((first + i) / a.top);
            a.place[first + i] = (int32_t)at++;
        }
    // pairs without an expert
    for (uint32_t i = threadIdx.x; i < pairs; i += ROUTE_THREADS)
        if (s.id[i] >= a.experts) a.place[first + i] = -1;
    const uint32_t slots = a.tokens * a.top;
    for (uint32_t i = all + blockIdx.x * ROUTE_THREADS + threadIdx.x; i < slots; i += a.blocks * ROUTE_THREADS) a.rows[i] = -1;
}

__device__ inline double wave_sum(double v)
{
    for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
    return v;
}

// A wave takes a token: lane l has the experts l, l + 64, ...  Scores and choices are taken in 64 bits, since neighbouring choices decide whole numbers: in
// 32, two libraries' exponentials would send a token to different experts now and then.
template <int PER, bool GROUPS>
__global__ __launch_bounds__(ROUTE_THREADS) void ecfm_choose_kernel(const RouteArgs a)
{
    __shared__ SortSpace s;
    __shared__ double keys[GROUPS ? ROUTE_WAVES : 1][GROUPS ? 64 * PER : 1];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = blockIdx.x * a.per_block, n = a.tokens - first < a.per_block ? a.tokens - first : a.per_block;
    for (uint32_t i = wave; i < n; i += ROUTE_WAVES) {
        const uint32_t t = first + i;
        double score[PER], key[PER];
        float x[PER], most = -INFINITY;
        for (int q = 0; q < PER; q++) {
            const uint32_t e = lane + 64 * q;
            x[q] = -INFINITY;
            if (e < a.experts) x[q] = a.f32 ? ((const float *)a.logits)[(int64_t)t * a.stride + e] : (float)((const __bf16 *)a.logits)[(int64_t)t * a.stride + e];
            x[q] = x[q] != x[q] ? -INFINITY : x[q] > FLT_MAX ? FLT_MAX : x[q];
            most = fmaxf(most, x[q]);
        }
        for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
        double sum = 0;
        for (int q = 0; q < PER; q++) {
            if (x[q] == -INFINITY) score[q] = 0;
            else if (a.sigmoid) score[q] = 1.0 / (1.0 + exp(-(double)x[q]));
            else score[q] = exp((double)x[q] - (double)most);
            sum += score[q];
        }
        if (!a.sigmoid) {
            sum = wave_sum(sum);
            for (int q = 0; q < PER; q++) score[q] = sum > 0 ? score[q] / sum : 0;
        }
        for (int q = 0; q < PER; q++) {
            const uint32_t e = lane + 64 * q;
            key[q] = a.bias ? score[q] + (double)(e < a.experts ? a.bias[e] : 0.f) : GROUPS ? score[q] : (double)x[q];
            if (x[q] == -INFINITY || key[q] != key[q]) key[q] = -INFINITY;
        }
        if constexpr (GROUPS) {
            for (int q = 0; q < PER; q++) keys[wave][lane + 64 * q] = key[q];
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
            const uint32_t size = a.experts / a.groups;
            double best = -INFINITY, second = -INFINITY;
            if (lane < a.groups)
                for (uint32_t j = 0, o = lane % size; j < size; j++, o = o + 1 == size ? 0 : o + 1) {     // lanes begin at unlike places: unlike banks
                    const double v = keys[wave][lane * size + o];
                    second = fmax(second, fmin(best, v));
                    best = fmax(best, v);
                }
            const double worth = second == -INFINITY ? best : best + second;
            uint32_t better = 0;
            for (uint32_t o = 0; o < a.groups; o++) {
                const double v = __shfl(worth, o);
                better += v > worth || (v == worth && o < lane);
            }
            const uint64_t open = __ballot(lane < a.groups && better < a.top_groups);
            for (int q = 0; q < PER; q++) {
                const uint32_t e = lane + 64 * q;
                if (e >= a.experts || !(open >> (e / size) & 1)) key[q] = -INFINITY;
            }
            __builtin_amdgcn_wave_barrier();
        }
        int32_t id = -1;
        double got = 0;
        for (uint32_t j = 0; j < a.top; j++) {
            double k = key[0], v = score[0];
            uint32_t e = lane;
            for (int q = 1; q < PER; q++)
                if (key[q] > k) {
                    k = key[q];
                    v = score[q];
                    e = lane + 64 * q;
                }
            double top = k;
            uint32_t at = e;
            for (int d = 32; d; d /= 2) {
                const double k2 = __shfl_xor(top, d);
                const uint32_t e2 = __shfl_xor(at, d);
                if (k2 > top || (k2 == top && e2 < at)) {
                    top = k2;
                    at = e2;
                }
            }
            v = __shfl(v, at & 63);                            // of the lane whose best it is
            if (lane == j && top != -INFINITY) {
                id = (int32_t)at;
                got = v;
            }
            for (int q = 0; q < PER; q++)
                if (lane + 64 * q == at) key[q] = -INFINITY;
        }
        if (a.normalise) {
            double total = 0;
            for (uint32_t j = 0; j < a.top; j++) total += __shfl(got, j);
            got = total > 0 ? got / total : 0;
        }
        if (lane < a.top) {
            a.ids[(uint64_t)t * a.top + lane] = id;
            a.weights[(uint64_t)t * a.top + lane] = (float)(got * (double)a.scale);
            s.id[i * a.top + lane] = id < 0 ? 0xffff : (uint16_t)id;
        }
    }
    __syncthreads();
    count_pairs(a, s, n * a.top);
    uint32_t mine = 0;
    if (threadIdx.x < a.experts)
        for (uint32_t g = 0; g < ROUTE_THREADS >> a.log_bins; g++) mine += s.count[(g << a.log_bins) + threadIdx.x];
    if (a.blocks == 1) place_pairs(a, s, 0, n * a.top, 0, mine);
    else if (threadIdx.x < a.experts) a.counts[(uint64_t)blockIdx.x * a.experts + threadIdx.x] = mine;
}

// Where there are many workgroups: each expert's counts become sums over the workgroups before; behind the last, the sums of all.
__global__ __launch_bounds__(ROUTE_THREADS) void ecfm_sum_kernel(const RouteArgs a)
{
    __shared__ uint32_t part[ROUTE_WAVES][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const uint32_t each = (a.blocks + ROUTE_WAVES - 1) / ROUTE_WAVES, lo = wave * each < a.blocks ? wave * each : a.blocks, hi = lo + each < a.blocks ? lo + each : a.blocks;
    uint32_t n = 0;
    if (e < a.experts)
        for (uint32_t b = lo; b < hi; b++) n += a.counts[(uint64_t)b * a.experts + e];
    part[wave][lane] = n;
    __syncthreads();
    uint32_t at = 0, all = 0;
    for (uint32_t w = 0; w < ROUTE_WAVES; w++) {
        at += w < wave ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (e >= a.experts) return;
    for (uint32_t b = lo; b < hi; b++) {
        const uint32_t c = a.counts[(uint64_t)b * a.experts + e];
        a.counts[(uint64_t)b * a.experts + e] = at;
        at += c;
    }
    if (wave == 0) a.counts[(uint64_t)a.blocks * a.experts + e] = all;
}

template <bool SUMMED>
__global__ __launch_bounds__(ROUTE_THREADS) void ecfm_sort_kernel(const RouteArgs a)
{
    __shared__ SortSpace s;
    const uint32_t first = blockIdx.x * a.per_block * a.top, n = a.tokens - blockIdx.x * a.per_block < a.per_block ? a.tokens - blockIdx.x * a.per_block : a.per_block;
    for (uint32_t i = threadIdx.x; i < n * a.top; i += ROUTE_THREADS) s.id[i] = (uint16_t)a.ids[first + i];
    uint32_t before = 0, total = 0;
    if (threadIdx.x < a.experts) {
        if (SUMMED) {
            before = a.counts[(uint64_t)blockIdx.x * a.experts + threadIdx.x];
            total = a.counts[(uint64_t)a.blocks * a.experts + threadIdx.x];
        } else
            for (uint32_t b = 0; b < a.blocks; b++) {
                const uint32_t c = a.counts[(uint64_t)b * a.experts + threadIdx.x];
                before += b < blockIdx.x ? c : 0;
                total += c;
            }
    }
    __syncthreads();
    count_pairs(a, s, n * a.top);
    place_pairs(a, s, first, n * a.top, before, total);
}

template <bool GROUPS>
void choose(const RouteArgs &a, hipStream_t s)
{
    const dim3 grid(a.blocks), block(ROUTE_THREADS);
    if (a.experts <= 64) hipLaunchKernelGGL((ecfm_choose_kernel<1, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((ecfm_choose_kernel<2, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((ecfm_choose_kernel<4, GROUPS>), grid, block, 0, s, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((ecfm_choose_kernel<8, GROUPS>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ecfm_choose_kernel<16, GROUPS>), grid, block, 0, s, a);
}

constexpr uint32_t ADD_UP_BLOCKS = 256;            // up to here each workgroup adds up the counts of all by itself

uint32_t tokens_of_block(uint32_t tokens)
{
    (void)tokens;
    return ROUTE_TOKENS;
}

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
    const uint32_t per = tokens_of_block(n_tokens), blocks = (n_tokens + per - 1) / per;
    return blocks <= 1 ? 0 : (uint64_t)(blocks + 1) * experts * 4;
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
        || ((uintptr_t)d_rows & 3) || ((uintptr_t)d_place & 3) || ((uintptr_t)d_workspace & 3))
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
    a.counts = (uint32_t *)d_workspace;
    a.tokens = o->n_tokens;
    a.experts = o->experts;
    a.top = o->top;
    a.sigmoid = o->sigmoid;
    a.normalise = o->normalise;
    a.groups = o->groups;
    a.top_groups = o->top_groups;
    a.f32 = o->dtype == ECFA_F32;
    a.scale = o->scale;
    a.per_block = tokens_of_block(o->n_tokens);
    a.blocks = o->n_tokens ? (o->n_tokens + a.per_block - 1) / a.per_block : 1;      // no tokens: the starts are written all the same
    a.log_bins = 6;
    while ((1u << a.log_bins) < a.experts) a.log_bins++;
    hipStream_t s = (hipStream_t)stream;
    if (a.groups > 1) choose<true>(a, s);
    else choose<false>(a, s);
    if (a.blocks > 1) {
        if (a.blocks > ADD_UP_BLOCKS) {
            hipLaunchKernelGGL(ecfm_sum_kernel, dim3((a.experts + 63) / 64), dim3(ROUTE_THREADS), 0, s, a);
            hipLaunchKernelGGL(ecfm_sort_kernel<true>, dim3(a.blocks), dim3(ROUTE_THREADS), 0, s, a);
        } else hipLaunchKernelGGL(ecfm_sort_kernel<false>, dim3(a.blocks), dim3(ROUTE_THREADS), 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

} // extern "C"
