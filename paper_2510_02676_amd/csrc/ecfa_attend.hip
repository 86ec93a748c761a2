// Attention over a paged cache: the host side, and the kernel that joins the splits of long sequences.
#include <cmath>

#include "ecf8_device.h"
#include "ecfa_attend.h"
#include "ecfa_host.h"

namespace {
using namespace ecfa;

constexpr int JOIN_THREADS = 256, JOIN_FEW = 8;

// The pieces' (m, l, O) of a row to one row: a thread four elements of it, from piece `first` on every `by`-th one, four pieces' at once.
struct Joined {
    float top, all;
    f32x4 y;
};
__device__ inline Joined join(const AttendArgs &a, int64_t part, int64_t stride, int32_t used, int32_t first, int32_t by, uint32_t quad)
{
    Joined j{NONE, 0.f, f32x4{0, 0, 0, 0}};
    for (int32_t i = first; i < used; i += 4 * by) {
        float m[4], l[4], top = j.top;
        f32x4 y[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t at = part + stride * (i + k * by < used ? i + k * by : i);
            m[k] = a.part_ml[2 * at];
            l[k] = a.part_ml[2 * at + 1];
            y[k] = *(const f32x4 *)(a.part + at * a.head_dim + 4 * quad);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) top = max_f(top, m[k]);    // (one twice does not matter here)
        const float base = top == NONE ? 0.f : top, old = exp2_fast(j.top - base);
        j.all *= old;
        j.y *= old;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (i + k * by >= used) break;
            const float w = exp2_fast(m[k] - base);
            j.all += l[k] * w;
            j.y += y[k] * w;
        }
        j.top = top;
    }
    return j;
}

__device__ inline void write_joined(const AttendArgs &a, const Joined &j, int64_t t, int64_t head, uint32_t quad)
{
    const float inv = j.all == 0.f ? 0.f : 1.f / j.all;
    bf16x4 z;
    for (int i = 0; i < 4; i++) z[i] = (__bf16)(j.all == 0.f ? 0.f : j.y[i] * inv);
    *(bf16x4 *)(a.out + t * a.o_tok + head * a.o_head + 8 * quad) = z;
}

// Reads what the pieces have written, 4 head_dim + 8 bytes a row and piece, once.  The first few_blocks workgroups are for rows of the few-rows
// kernel's first tiles, few_joined of them for each sequence and key/value head.  Such a row may have hundreds of pieces: then the groups of
// head_dim / 4 threads of a workgroup share them; up to JOIN_FEW pieces are one group's work.  The others are for a token of the
// other kernel each, with few pieces: head_dim / 4 threads a row.  Bound by its chain: lengths, plan, pieces, rows take 4.9 us for one
// token of 4096 keys and 5.9 for 64 of up to 8192.
__global__ __launch_bounds__(JOIN_THREADS) void ecfa_attend_join_kernel(const AttendArgs a, uint32_t few_blocks, uint32_t few_joined)
{
    __shared__ f32x4 sums[JOIN_THREADS];
    __shared__ float alls[JOIN_THREADS], tops[JOIN_THREADS];
    const int32_t share = (int32_t)a.share;
    const uint32_t quads = a.head_dim / 4, groups = JOIN_THREADS / quads, group = threadIdx.x / quads, quad = threadIdx.x % quads;
    if (blockIdx.x >= few_blocks) {
        const uint32_t t = blockIdx.x - few_blocks, s = seq_of_row(a.b, t);
        const Seq sq = seq_of(a.b, s);
        const int32_t tok = (int32_t)t - sq.q0, rows = sq.qn * share, prefix = prefix_of(a, s, sq);
        if (tok < 0 || tok >= sq.qn || rows <= a.few_rows || group >= groups) return;
        for (uint32_t head = group; head < a.heads; head += groups) {
            const int32_t row = tok * share + (int32_t)(head - (uint32_t)over((int32_t)head, a.by_share) * a.share);
            const int32_t row0 = row / MANY_ROWS * MANY_ROWS, row_end = row0 + MANY_ROWS < rows ? row0 + MANY_ROWS : rows;
            const int32_t used = split_of(keys_of(a, sq, prefix, over(row0, a.by_share), over(row_end - 1, a.by_share)), a.many_splits).used;
            if (used <= 1) continue;                           // written already
            const int64_t part = many_part(a, t, head);
            write_joined(a, join(a, part, 1, used, 0, 1, quad), t, head, quad);
        }
        return;
    }
    const uint32_t kvh = blockIdx.x / few_joined % a.kv_heads, s = blockIdx.x / few_joined / a.kv_heads;
    const FewItem it = few_plan(a, s, true);
    if (!it.there || it.used <= 1) return;                     // not this kernel's, or written already
    const Seq sq = seq_of(a.b, s);
    const int32_t rows = sq.qn * share < (int32_t)a.few_tile ? sq.qn * share : (int32_t)a.few_tile;
    const int64_t stride = (int64_t)a.kv_heads * a.few_tile;
    if (it.used <= JOIN_FEW) {                                 // few pieces: a row for each group of threads
        if (group >= groups) return;
        for (int32_t row = (int32_t)(blockIdx.x % few_joined * groups + group); row < rows; row += (int32_t)(few_joined * groups)) {
            const int32_t tok = over(row, a.by_share);
            write_joined(a, join(a, few_part(a, it.first_item, kvh, row), stride, it.used, 0, 1, quad), (int64_t)sq.q0 + tok,
                         (int64_t)kvh * a.share + (row - tok * share), quad);
        }
        return;
    }
    for (int32_t row = (int32_t)(blockIdx.x % few_joined); row < rows; row += (int32_t)few_joined) {
        const int64_t part = few_part(a, it.first_item, kvh, row);
        Joined j{NONE, 0.f, f32x4{0, 0, 0, 0}};
        if (group < groups) j = join(a, part, stride, it.used, (int32_t)group, (int32_t)groups, quad);
        __syncthreads();
        sums[threadIdx.x] = j.y;
        alls[threadIdx.x] = j.all;
        tops[threadIdx.x] = j.top;
        __syncthreads();
        if (threadIdx.x < quads) {
            float top = NONE;
            for (uint32_t k = 0; k < groups; k++) top = max_f(top, tops[k * quads + quad]);
            const float base = top == NONE ? 0.f : top;
            j = Joined{top, 0.f, f32x4{0, 0, 0, 0}};
            for (uint32_t k = 0; k < groups; k++) {
                const float w = exp2_fast(tops[k * quads + quad] - base);
                j.all += alls[k * quads + quad] * w;
                j.y += sums[k * quads + quad] * w;
            }
            const int32_t tok = over(row, a.by_share);
            write_joined(a, j, (int64_t)sq.q0 + tok, (int64_t)kvh * a.share + (row - tok * share), quad);
        }
    }
}

// What a call launches: decided by shapes, the hints and the window alone.
struct Shape {
    uint32_t kc;                   // 32-element pieces of a head in the kernels
    bool few, many;                // which kernels
    int32_t few_rows;
    uint32_t few_tiles, few_goal, few_unit, few_items, few_joined, many_tiles, many_splits;
    uint64_t few_parts, many_parts;          // partial rows in the workspace
};

// Pieces of the keys of each tile of many rows.  Where the tiles leave compute units free, in as many pieces, of 512 keys at least, as make the
// last workgroup end first: rounds of two workgroups on each compute unit (one for heads of more than 128 elements, by registers), each
// the steps of 64 keys of a piece and a start of about four steps' time; for the second kernel as much again, and a little for each piece.
// (192 tiles of 8768 keys: 5 pieces 136 us, 3 pieces 160; 300 tiles of 9200: 3 pieces 204, 2 pieces 234.)  More tiles than
// that are of unlike length and fill one another's gaps (512 tiles of 8192 keys: whole 255 us, in two 272).
uint32_t splits_of(uint64_t tiles, uint64_t slots, uint64_t keys)
{
    if (tiles > slots || keys <= 512) return 1;
    const double steps = (double)keys / 64, piece = 0.3;
    double best = steps + 4;
    uint64_t best_n = 1;
    for (uint64_t rounds = 1; rounds <= 4; rounds++) {         // the most pieces that so many rounds hold, or the best number if it is less
        uint64_t n = rounds * slots / tiles;
        const uint64_t enough = (uint64_t)std::sqrt(steps * (double)rounds / piece), most = (keys + 511) / 512;
        n = n < enough ? n : enough;
        n = n < most ? n : most;
        if (n < 2) continue;
        const double t = (double)((n * tiles + slots - 1) / slots) * (steps / (double)n + 4) + 4 + piece * (double)n;
        if (t < best) best = t, best_n = n;
    }
    return (uint32_t)best_n;
}

// Up to 32 rows of a sequence (the heads that share their keys, times its new tokens) go to the few-rows kernel, which reads K and V without
// waiting for other waves and cuts the keys in equal pieces; more go to 128-row tiles.  At 32 rows, heads of 128, BF16: one
// sequence of 4096 keys 18.8 us (tiles 31.1), 64 of them with 8 heads 232 (236), E4M3 143 (177).  17 to 32 rows that meet no more
// than 512 keys go to tiles as well, which need no second kernel then: 64 sequences of 512 keys 29.3 us (few-rows kernel 44.0), E4M3 25.5 (31.3).
// `window`: 0 if there is none; with one, no more is asked for than without.
Shape shape_of(const ecfa_cache *c, const ecfa_batch *b, uint32_t heads, uint32_t cus, uint64_t window)
{
    Shape p{};
    const uint32_t kc = (c->head_dim + 31) / 32, share = heads / c->kv_heads;
    p.kc = kc <= 2 ? 2 : kc <= 4 ? kc : kc <= 6 ? 6 : 8;
    const uint32_t max_q = !b->d_q_start ? 1 : b->max_q && b->max_q < b->n_tokens ? b->max_q : b->n_tokens;
    const uint64_t keys = (uint64_t)b->table_width * c->page_size;
    const uint64_t max_kv = b->max_kv && b->max_kv < keys ? b->max_kv : keys;
    const auto seen = [&](uint64_t rows) { return window && window + rows < max_kv ? window + rows : max_kv; };    // keys of a tile
    const uint64_t rows = (uint64_t)max_q * share;
    if (rows <= 16 || (rows <= 32 && max_kv > 512)) {          // few rows everywhere
        p.few = true;
        p.few_rows = 0x7fffffff;
        p.few_tiles = rows <= 16 ? 1 : 2;
    } else {                       // many in some sequence; single tokens of others, if there may be any, in the other kernel
        p.many = true;
        p.few = share <= 32 && (uint64_t)b->n_seqs * max_q != b->n_tokens;
        p.few_tiles = share <= 16 ? 1 : 2;
        p.few_rows = p.few ? 16 * (int32_t)p.few_tiles : 0;
    }
    p.many_splits = 1;
    if (p.few) {
        // As many pieces as make two workgroups on each compute unit, with a step for each wave at least (two for 32 rows), of up to 1024
        // sequences: every workgroup reads all of their lengths.  One of 32768 keys among 1023 of 32: 327 us, among 1024 (none cut) 435; but 1024 of 512
        // keys 549 us, 1025 372.  One token of 131072 keys, 64 of up to 8192, 16 times 8 tokens of 4096: two workgroups 108, 49, 77 us; one 131, 52,
        // 88; four 111, 49, 94.  Twice as many steps at least: 2048 keys of one token 12.7 us, 11.4 with one; 8 tokens after 4088 keys 18.8 us,
        // 21.6 with one.
        const uint32_t bytes = p.kc * 32 * (c->dtype == ECFA_E4M3 ? 1 : 2);
        p.few_unit = FEW_WAVES * (p.few_tiles > 1 ? 2 : bytes <= 64 ? 4 : bytes <= 128 ? 2 : 1);        // KU of FewShape, of two sub-tiles twice that
        const uint64_t want = (2ull * cus + c->kv_heads - 1) / c->kv_heads, pieces = (seen(16 * p.few_tiles) + 32 * p.few_unit - 1) / (32 * p.few_unit);
        const uint64_t most = pieces * b->n_seqs;
        p.few_goal = pieces <= 1 || b->n_seqs > 1024 ? 0 : (uint32_t)(want < most ? want : most);
        p.few_items = p.few_goal + b->n_seqs;
        // In the second kernel a workgroup a row while all of them are on the card at once, and then a group of its threads a row (16 times 8
        // tokens of 4096 keys, 4096 rows and heads: 77.0 -> 67.5 us; 15 times 16 rows of a head of 256, 1920: 32.5, by groups 35.3).
        const uint32_t joined = (uint32_t)(rows < 16 * p.few_tiles ? rows : 16 * p.few_tiles), groups = JOIN_THREADS / (c->head_dim / 4);
        p.few_joined = (uint64_t)b->n_seqs * c->kv_heads * joined < 8ull * cus ? joined : (joined + groups - 1) / groups;
        if (p.few_goal) p.few_parts = (uint64_t)p.few_items * c->kv_heads * 16 * p.few_tiles;
    }
    if (p.many) {
        p.many_tiles = (uint32_t)((uint64_t)b->n_tokens * share / MANY_ROWS) + b->n_seqs;
        const uint64_t slots = (kc <= 4 ? 2ull : 1ull) * cus, tiles = ((uint64_t)b->n_tokens * share + MANY_ROWS - 1) / MANY_ROWS * c->kv_heads;
        p.many_splits = splits_of(tiles, slots, max_kv);
        const uint32_t n = splits_of(tiles, slots, seen(MANY_ROWS));
        if (n < p.many_splits) p.many_splits = n;              // with a window no more than without: the workspace is sized without
        if (p.many_splits > 1) p.many_parts = (uint64_t)b->n_tokens * heads * p.many_splits;
    }
    return p;
}

uint64_t workspace_of(const Shape &p, uint32_t head_dim) { return (p.few_parts + p.many_parts) * (head_dim + 2) * 4; }

uint64_t few_join_blocks(const ecfa_cache *c, const ecfa_batch *b, const Shape &p) { return p.few_goal ? (uint64_t)b->n_seqs * c->kv_heads * p.few_joined : 0; }

uint64_t join_blocks(const ecfa_cache *c, const ecfa_batch *b, const Shape &p) { return few_join_blocks(c, b, p) + (p.many_parts ? b->n_tokens : 0u); }

int check_heads(const ecfa_cache *c, uint32_t heads)
{
    return heads == 0 || heads > (1u << 20) || heads % c->kv_heads ? ECF8_E_ARG : ECF8_OK;
}

// Rows of a sequence are counted in 32 bits, and a launch's threads, 256 a workgroup, too.
int check_counts(const ecfa_cache *c, const ecfa_batch *b, uint32_t heads, const Shape &p)
{
    if ((uint64_t)b->n_tokens * (heads / c->kv_heads) > (1u << 30)) return ECF8_E_ARG;
    const uint64_t most = 0xffffff;
    if ((uint64_t)(p.few ? p.few_items : 0) * c->kv_heads + (p.many ? (uint64_t)p.many_tiles * c->kv_heads * p.many_splits : 0) > most) return ECF8_E_ARG;
    return join_blocks(c, b, p) > most ? ECF8_E_ARG : ECF8_OK;
}

int check_attend_rows(const ecfa_rows *r, uint32_t n_tokens)
{
    if (r->dtype != ECFA_BF16) return ECF8_E_ARG;
    if (n_tokens && !r->d) return ECF8_E_ARG;
    if (((uintptr_t)r->d & 15) || (apart(r->token_stride, 2, n_tokens) & 15) || (apart(r->head_stride, 2, r->heads) & 15)) return ECF8_E_ALIGN;
    return ECF8_OK;
}

} // namespace

extern "C" {

uint64_t ecfa_attend_workspace_bytes(const ecfa_cache *cache, const ecfa_batch *batch, uint32_t heads)
{
    CacheView c{};
    BatchView b{};
    if (!cache || !batch || cache_view(cache, true, &c) || batch_view(cache, batch, true, &b) || check_heads(cache, heads) || !batch->n_tokens) return 0;
    const int cus = device_cus();
    const Shape p = shape_of(cache, batch, heads, cus > 0 ? (uint32_t)cus : 256u, 0);
    return check_counts(cache, batch, heads, p) ? 0 : workspace_of(p, cache->head_dim);
}

int ecfa_attend(const ecfa_cache *cache, const ecfa_batch *batch, const ecfa_attend_opts *opts, const ecfa_rows *q, const ecfa_rows *out,
                void *d_workspace, uint64_t workspace_bytes, void *stream)
{
    AttendArgs a{};
    if (!cache || !batch || !opts || !q || !out) return ECF8_E_ARG;
    int rc = cache_view(cache, true, &a.c);
    if (!rc) rc = batch_view(cache, batch, true, &a.b);
    if (!rc) rc = check_heads(cache, q->heads);
    if (!rc && out->heads != q->heads) rc = ECF8_E_ARG;
    if (!rc) rc = check_attend_rows(q, batch->n_tokens);
    if (!rc) rc = check_attend_rows(out, batch->n_tokens);
    if (rc) return rc;
    if (!(opts->scale > 0) || !std::isfinite(opts->scale) || !(opts->softcap >= 0) || !std::isfinite(opts->softcap) || opts->causal > 1) return ECF8_E_ARG;
    if (opts->window && opts->d_prefix_len) return ECF8_E_ARG;
    if (((uintptr_t)opts->d_slopes & 3) || ((uintptr_t)opts->d_prefix_len & 3)) return ECF8_E_ALIGN;
    if (batch->n_tokens == 0) return ECF8_OK;
    const int cus = device_cus();
    if (cus <= 0) return ECF8_E_HIP;
    const Shape p = shape_of(cache, batch, q->heads, (uint32_t)cus, opts->causal ? opts->window : 0);
    if ((rc = check_counts(cache, batch, q->heads, p))) return rc;
    const uint64_t need = workspace_of(p, cache->head_dim);
    if (need) {
        if (!d_workspace) return ECF8_E_ARG;
        if ((uintptr_t)d_workspace & 15) return ECF8_E_ALIGN;
        if (workspace_bytes < need) return ECF8_E_CAPACITY;
        a.part = (float *)d_workspace;
        a.part_ml = a.part + (p.few_parts + p.many_parts) * cache->head_dim;
        a.many_part0 = (int64_t)p.few_parts;
    }
    a.q = (const uint8_t *)q->d;
    a.out = (uint8_t *)out->d;
    a.q_tok = apart(q->token_stride, 2, batch->n_tokens);
    a.q_head = apart(q->head_stride, 2, q->heads);
    a.o_tok = apart(out->token_stride, 2, batch->n_tokens);
    a.o_head = apart(out->head_stride, 2, out->heads);
    a.slopes = opts->d_slopes;
    a.prefix = opts->d_prefix_len;
    a.scale_log2 = opts->scale * LOG2E;
    // A cap above 2^100 changes no score that fp32 tells from its neighbours (below 2^88 by less than 2^-24 of it); below 2^-100 all weights are alike.
    // So what the kernels work with has a reciprocal and stays finite times log2(e).
    a.cap = opts->softcap > 0x1p100f ? 0.f : opts->softcap > 0 && opts->softcap < 0x1p-100f ? 0x1p-100f : opts->softcap;
    a.cap_inv = a.cap > 0 ? 1.f / a.cap : 0.f;
    a.head_dim = cache->head_dim;
    a.heads = q->heads;
    a.kv_heads = cache->kv_heads;
    a.share = q->heads / cache->kv_heads;
    a.by_share = divisor_of(a.share);
    a.by_kv_heads = divisor_of(a.kv_heads);
    a.by_items = divisor_of(p.few_items ? p.few_items : 1);
    a.by_goal = divisor_of(p.few_goal ? p.few_goal : 1);
    a.causal = opts->causal;
    a.window = opts->window;
    a.few_rows = p.few_rows;
    a.few_tile = 16 * p.few_tiles;
    a.few_goal = p.few_goal;
    a.few_unit = p.few_unit;
    a.few_items = p.few_items;
    a.many_tiles = p.many_tiles;
    a.many_splits = p.many_splits;
    hipStream_t s = (hipStream_t)stream;
    const bool f8 = cache->dtype == ECFA_E4M3;
    rc = f8 ? launch_attend_e4m3(a, p.kc, p.few, p.many, s) : launch_attend_bf16(a, p.kc, p.few, p.many, s);
    if (rc || !need) return rc;
    hipLaunchKernelGGL(ecfa_attend_join_kernel, dim3((unsigned)join_blocks(cache, batch, p)), dim3(JOIN_THREADS), 0, s, a,
                       (uint32_t)few_join_blocks(cache, batch, p), p.few_joined ? p.few_joined : 1u);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

} // extern "C"
