// Attention over a paged cache: the host side, and the kernel that joins the splits of long sequences.
#include <cmath>

#include "ecf8_device.h"
#include "ecfa_attend.h"
#include "ecfa_host.h"

namespace {
using namespace ecfa;

constexpr int JOIN_THREADS = 256;

// One workgroup for a (token, query head): the splits' (m, l, O) to one row.  The splits are dealt to groups of head_dim / 4 threads, so
// that all partial rows are on their way at once.  Reads what the splits have written, 4 head_dim + 8 bytes each, once.
__global__ __launch_bounds__(JOIN_THREADS) void ecfa_attend_join_kernel(const AttendArgs a)
{
    __shared__ f32x4 sums[JOIN_THREADS];
    const uint32_t t = blockIdx.x / a.heads, head = blockIdx.x % a.heads;
    const uint32_t s = seq_of_row(a.b, t);
    const Seq sq = seq_of(a.b, s);
    const int32_t tok = (int32_t)t - sq.q0;
    if (tok < 0 || tok >= sq.qn) return;
    const int32_t rows = sq.qn * (int32_t)a.share, tile = (int32_t)a.tile_rows;
    const int32_t row0 = (tok * (int32_t)a.share + (int32_t)(head % a.share)) / tile * tile;
    const int32_t row_end = row0 + tile < rows ? row0 + tile : rows;
    const KeyRange kr = keys_of(a, sq, prefix_of(a, s, sq), row0 / (int32_t)a.share, (row_end - 1) / (int32_t)a.share);
    const int32_t used = split_of(kr, a.splits, (int32_t)a.split_unit).used;
    if (used <= 1) return;                                     // the row is written already
    const int64_t part = ((int64_t)t * a.heads + head) * a.splits;
    const float *ml = a.part_ml + part * 2;
    float top = NONE;
    for (int32_t i = threadIdx.x & 63; i < used; i += 64) top = max_f(top, ml[2 * i]);
    for (int k = 1; k < 64; k *= 2) top = max_f(top, __shfl_xor(top, k));
    const float base = top == NONE ? 0.f : top;
    const uint32_t quads = a.head_dim / 4, groups = JOIN_THREADS / quads, group = threadIdx.x / quads, quad = threadIdx.x % quads;
    f32x4 y{0, 0, 0, 0};
    float all = 0.f;
    if (group < groups)
        for (int32_t i = (int32_t)group; i < used; i += (int32_t)groups) {
            const float w = exp2_fast(ml[2 * i] - base);
            all += ml[2 * i + 1] * w;
            y += *(const f32x4 *)(a.part + (part + i) * a.head_dim + 4 * quad) * w;
        }
    __shared__ float alls[JOIN_THREADS];
    sums[threadIdx.x] = y;
    alls[threadIdx.x] = all;
    __syncthreads();
    if (threadIdx.x >= quads) return;
    for (uint32_t k = 1; k < groups; k++) {
        y += sums[k * quads + quad];
        all += alls[k * quads + quad];
    }
    const float inv = all == 0.f ? 0.f : 1.f / all;
    bf16x4 z;
    for (int i = 0; i < 4; i++) z[i] = (__bf16)(all == 0.f ? 0.f : y[i] * inv);
    *(bf16x4 *)(a.out + (int64_t)t * a.o_tok + (int64_t)head * a.o_head + 8 * quad) = z;
}

// What a call launches: decided by shapes and the hints alone.
struct Shape {
    uint32_t kc;                   // 32-element pieces of a head in the kernel
    uint32_t tiles;                // sub-tiles of 16 rows
    uint32_t row_tiles, splits, tile_rows, split_unit;
    uint64_t part_floats;          // partial sums in the workspace, then two floats for each of part_rows
    uint64_t part_rows;
};

Shape shape_of(const ecfa_cache *c, const ecfa_batch *b, uint32_t heads, uint32_t cus)
{
    Shape p{};
    const uint32_t kc = (c->head_dim + 31) / 32;
    p.kc = kc <= 2 ? 2 : kc <= 4 ? kc : kc <= 6 ? 6 : 8;
    const uint32_t max_q = !b->d_q_start ? 1 : b->max_q && b->max_q < b->n_tokens ? b->max_q : b->n_tokens;
    const uint64_t keys = (uint64_t)b->table_width * c->page_size;
    const uint64_t max_kv = b->max_kv && b->max_kv < keys ? b->max_kv : keys;
    const uint64_t rows = (uint64_t)max_q * (heads / c->kv_heads);
    p.tiles = rows <= 16 ? 1 : 2;
    p.tile_rows = 16 * p.tiles;
    p.row_tiles = (uint32_t)((rows + p.tile_rows - 1) / p.tile_rows);
    p.split_unit = 4;
    // enough workgroups for four on each compute unit, of 128 keys at least
    const uint64_t whole = (uint64_t)b->n_seqs * c->kv_heads * p.row_tiles;
    const uint64_t want = whole ? (4ull * cus + whole - 1) / whole : 1, most = (max_kv + 127) / 128;
    const uint64_t n = want < most ? want : most;
    p.splits = (uint32_t)(n < 1 ? 1 : n > 256 ? 256 : n);
    if (p.splits > 1) {
        p.part_rows = (uint64_t)b->n_tokens * heads * p.splits;
        p.part_floats = p.part_rows * c->head_dim;
    }
    return p;
}

int check_heads(const ecfa_cache *c, uint32_t heads)
{
    return heads == 0 || heads > (1u << 20) || heads % c->kv_heads ? ECF8_E_ARG : ECF8_OK;
}

int check_attend_rows(const ecfa_rows *r, uint32_t n_tokens)
{
    if (r->dtype != ECFA_BF16) return ECF8_E_ARG;
    if (n_tokens && !r->d) return ECF8_E_ARG;
    if (((uintptr_t)r->d & 15) || (r->token_stride * 2 & 15) || (r->head_stride * 2 & 15)) return ECF8_E_ALIGN;
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
    const Shape p = shape_of(cache, batch, heads, cus > 0 ? (uint32_t)cus : 256u);
    return (p.part_floats + 2 * p.part_rows) * 4;
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
    const Shape p = shape_of(cache, batch, q->heads, (uint32_t)cus);
    const uint64_t need = (p.part_floats + 2 * p.part_rows) * 4;
    if (need) {
        if (!d_workspace) return ECF8_E_ARG;
        if ((uintptr_t)d_workspace & 15) return ECF8_E_ALIGN;
        if (workspace_bytes < need) return ECF8_E_CAPACITY;
        a.part = (float *)d_workspace;
        a.part_ml = a.part + p.part_floats;
    }
    a.q = (const uint8_t *)q->d;
    a.out = (uint8_t *)out->d;
    a.q_tok = q->token_stride * 2;
    a.q_head = q->head_stride * 2;
    a.o_tok = out->token_stride * 2;
    a.o_head = out->head_stride * 2;
    a.slopes = opts->d_slopes;
    a.prefix = opts->d_prefix_len;
    a.scale_log2 = opts->scale * LOG2E;
    a.cap = opts->softcap;
    a.head_dim = cache->head_dim;
    a.heads = q->heads;
    a.kv_heads = cache->kv_heads;
    a.share = q->heads / cache->kv_heads;
    a.causal = opts->causal;
    a.window = opts->window;
    a.splits = p.splits;
    a.row_tiles = p.row_tiles;
    a.tile_rows = p.tile_rows;
    a.split_unit = p.split_unit;
    hipStream_t s = (hipStream_t)stream;
    // a launch counts its threads, 256 a workgroup, in 32 bits
    if ((uint64_t)batch->n_seqs * p.row_tiles * a.kv_heads * p.splits > 0xffffff || (p.splits > 1 && (uint64_t)batch->n_tokens * a.heads > 0xffffff)) return ECF8_E_ARG;
    rc = cache->dtype == ECFA_E4M3 ? launch_few_rows_e4m3(a, p.kc, p.tiles, s) : launch_few_rows_bf16(a, p.kc, p.tiles, s);
    if (rc || p.splits <= 1) return rc;
    hipLaunchKernelGGL(ecfa_attend_join_kernel, dim3(batch->n_tokens * a.heads), dim3(JOIN_THREADS), 0, s, a);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

} // extern "C"
