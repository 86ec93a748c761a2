// Rows on their way into and out of attention: keys and values appended to a paged cache with the rotation applied on the way
// (ecfa_append), and rows rounded to E4M3 with scales (ecfa_quant).  Both are one pass over their data and bound by memory, or, for a
// single token, by the launch.
#include <cmath>

#include "ecfa_device.h"
#include "ecfa_host.h"

namespace {
using namespace ecfa;

constexpr int APPEND_THREADS = 256;

struct RowsView {                            // strides in bytes
    uint8_t *d;
    int64_t tok, head;
};

struct AppendArgs {
    CacheView c;
    BatchView b;
    RowsView q, k, v, q_out;
    const uint64_t *freq;
    const int32_t *pos;
    float rope_scale;
    uint32_t rot_units;                      // rot_dim / 16
    uint32_t units;                          // head_dim / 16
    uint32_t slots;                          // heads that a workgroup holds at once
    uint32_t q_heads, kv_heads;
};

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

// x / by in fp32.  The product with the reciprocal alone would lose ties of E4M3.  It is put right by what is left of x: with r the reciprocal to the
// nearest and q within a unit of the quotient, q + (x - q by) r in two fused operations is the quotient to the nearest (Markstein, 1990), as
// long as x - q by is a number of fp32, which scales from 2^-90 on see to for quotients from 2^-11 on.  Smaller ones are zeros in E4M3, and in BF16 a unit
// of fp32 is of no account.  Infinities stay.  Other scales: divisions.  6472 tokens, BF16 rows, E4M3, 32 + 2 x 8 heads of 128: 2 % more than the product
// alone takes, sixteen divisions 10 %, which also take registers: 84 instead of 63, and with them 64 prompts of up to 100 tokens 11.1 us instead of 9.3.
__device__ inline void divide16(float *x, float by)
{
    if (by >= 0x1p-90f && by <= 0x1p90f) {
        const float r = 1.f / by;
        for (int j = 0; j < 16; j++) {
            const float q = x[j] * r, y = __builtin_fmaf(__builtin_fmaf(-q, by, x[j]), r, q);
            x[j] = __builtin_fabsf(q) < 0x1p127f ? __builtin_copysignf(y, q) : q;
        }
    } else
#pragma unroll 1
        for (int j = 0; j < 16; j++) x[j] /= by;
}

// A workgroup takes one token.  A thread keeps its 16 elements' place within a head (eight pairs: 8 u .. and rot / 2 + 8 u .. by
// halves, 16 u .. interleaved) and walks over the heads of q, k and v, so that its eight sines and cosines are made once.  The angle
// is position times frequency modulo 2^64 of a turn: the upper 32 bits go to the sine unit, which takes turns, and the
// error stays below 2^-24 of a turn at any position.
// Bound by memory: 6472 tokens of BF16 rows with 32 + 2 x 8 heads of 128 elements, 80 MB in and 80 out, take 35 us (4.6 TB/s); a single
// token 3.6 us, the time of a launch and of three loads that follow one another (length, page, row).  128 and 512 threads a token: 37.8 and
// 41.4 us where 256 took 37.4.  Results written past the caches make the call alone faster, 27.4 us, but the attention that reads them loses
// more than that: both together take 221 us this way and 229 past the caches for 16384 tokens in sequences of 512 (E4M3 220.6 and 227.5), 89.0 and 90.6 for 6400 in
// sequences of 100 (E4M3 86.2 and 90.8), 411 and 413 for a sequence of 6472; only at 65536 tokens in BF16, 800 MB of results, 760 and 748.
template <bool F32, bool F8, bool INTERLEAVED>
__global__ __launch_bounds__(APPEND_THREADS) void ecfa_append_kernel(const AppendArgs a)
{
    const uint32_t t = blockIdx.x;
    const uint32_t s = seq_of_row(a.b, t);
    const Seq sq = seq_of(a.b, s);
    const int32_t i = (int32_t)t - sq.q0;
    if (i < 0 || i >= sq.qn) return;                           // a row of no sequence
    const uint32_t u = threadIdx.x % a.units, slot = threadIdx.x / a.units;
    if (slot >= a.slots) return;
    const int32_t place = sq.place0 + i;
    const bool turns = u < a.rot_units;
    uint32_t e0 = 16 * u, e1 = 16 * u + 8;                     // elements of the two halves of this thread's 16
    if (!INTERLEAVED && turns) e0 = 8 * u, e1 = 8 * a.rot_units + 8 * u;
    float c[8], sn[8];
    if (turns) {
        const int64_t pos = a.pos ? a.pos[t] : place;
        for (int j = 0; j < 8; j++) {
            const int32_t turn = (int32_t)((uint64_t)pos * a.freq[8 * u + j] >> 32);
            const float x = (float)turn * 0x1p-32f;
            c[j] = __builtin_amdgcn_cosf(x) * a.rope_scale;
            sn[j] = __builtin_amdgcn_sinf(x) * a.rope_scale;
        }
    }
    // where the token's keys and values go
    uint32_t page = 0xffffffffu;
    const uint32_t at = (uint32_t)place & ((1u << a.c.page_shift) - 1);
    if (a.k.d && place >= 0 && place < sq.len) page = (uint32_t)a.b.table[(int64_t)s * a.b.table_stride + ((uint32_t)place >> a.c.page_shift)];
    const bool kept = page < a.c.n_pages;
    constexpr int SRC = F32 ? 4 : 2, DST = F8 ? 1 : 2;
    const uint32_t heads = a.q_heads + 2 * a.kv_heads;
    for (uint32_t h = slot; h < heads; h += a.slots) {
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
        if (!is_q && !kept) continue;
        const RowsView &r = is_q ? a.q : is_v ? a.v : a.k;
        const uint32_t hh = is_q ? h : is_v ? h - a.q_heads - a.kv_heads : h - a.q_heads;
        const uint8_t *src = r.d + (int64_t)t * r.tok + (int64_t)hh * r.head;
        float x[16];
        if (is_v) {                                            // v lies as it came: 16 elements in a row
            load8<F32>(src + 16 * u * SRC, x);
            load8<F32>(src + (16 * u + 8) * SRC, x + 8);
        } else {
            load8<F32>(src + e0 * SRC, x);
            load8<F32>(src + e1 * SRC, x + 8);
            if (turns)
                for (int j = 0; j < 8; j++) {
                    float &p = INTERLEAVED ? x[2 * j] : x[j], &q = INTERLEAVED ? x[2 * j + 1] : x[8 + j];
                    const float y = p * c[j] - q * sn[j];
                    q = q * c[j] + p * sn[j];
                    p = y;
                }
        }
        if (is_q) {
            uint8_t *dst = a.q_out.d + (int64_t)t * a.q_out.tok + (int64_t)hh * a.q_out.head;
            store8_bf16(dst + e0 * 2, x);
            store8_bf16(dst + e1 * 2, x + 8);
            continue;
        }
        const uint32_t d0 = is_v ? 16 * u : e0, d1 = is_v ? 16 * u + 8 : e1;
        uint8_t *dst = is_v ? a.c.v + (int64_t)page * a.c.v_page + (int64_t)at * a.c.v_tok + (int64_t)hh * a.c.v_head
                            : a.c.k + (int64_t)page * a.c.k_page + (int64_t)at * a.c.k_tok + (int64_t)hh * a.c.k_head;
        const float *scales = is_v ? a.c.v_scale : a.c.k_scale;
        if (scales) {
            divide16(x, scales[hh]);
        }
        if constexpr (F8) {
            *(u32x2 *)(dst + d0 * DST) = pack8_e4m3(x);
            *(u32x2 *)(dst + d1 * DST) = pack8_e4m3(x + 8);
        } else {
            store8_bf16(dst + d0 * DST, x);
            store8_bf16(dst + d1 * DST, x + 8);
        }
    }
}

struct QuantArgs {
    const uint8_t *x;
    uint8_t *q;
    float *scale;
    int64_t row_bytes;                       // between rows of x
    uint64_t rows;
    uint32_t cols, per_row;                  // per_row: workgroups of a row (groups of 128 only)
};

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

// A scale per row: THREADS threads a row (four rows to a workgroup of 256 if they are 64), the row held in registers between its
// two uses up to HELD pieces of eight a thread, fetched again beyond that.
template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void ecfa_quant_rows_kernel(const QuantArgs a)
{
    constexpr int SRC = F32 ? 4 : 2, HELD = 4, BLOCK = THREADS == 64 ? 256 : THREADS, WAVES = BLOCK / 64;
    const uint64_t row = THREADS == 64 ? (uint64_t)blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x;
    const uint32_t t = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
    const bool there = row < a.rows;
    const uint8_t *x = a.x + (int64_t)(there ? row : 0) * a.row_bytes;
    const uint32_t pieces = a.cols / 8;
    float held[HELD][8];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < HELD; k++)
        if (t + k * THREADS < pieces) {
            load8<F32>(x + (uint64_t)(t + k * THREADS) * 8 * SRC, held[k]);
            const uint32_t o = most8(held[k]);
            m = o > m ? o : m;
        }
    for (uint32_t p = t + HELD * THREADS; p < pieces; p += THREADS) {
        float y[8];
        load8<F32>(x + (uint64_t)p * 8 * SRC, y);
        const uint32_t o = most8(y);
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
    uint8_t *q = a.q + row * a.cols;
#pragma unroll
    for (int k = 0; k < HELD; k++)
        if (t + k * THREADS < pieces) store_e4m3(q + (uint64_t)(t + k * THREADS) * 8, held[k], inv);
    for (uint32_t p = t + HELD * THREADS; p < pieces; p += THREADS) {
        float y[8];
        load8<F32>(x + (uint64_t)p * 8 * SRC, y);
        store_e4m3(q + (uint64_t)p * 8, y, inv);
    }
}

// A scale per 128 columns: sixteen lanes a group, eight columns a lane, 2048 columns a workgroup.  Bound by memory: 4096 x 14336 fp32 take 49 us
// (6.0 TB/s of 235 MB in, 60 out); with two and four times as many columns a workgroup 52 and 54 us, since fewer are in flight at the end.
template <bool F32>
__global__ __launch_bounds__(256) void ecfa_quant_groups_kernel(const QuantArgs a)
{
    constexpr int SRC = F32 ? 4 : 2;
    const uint64_t row = blockIdx.x / a.per_row;
    const uint32_t p = (uint32_t)(blockIdx.x % a.per_row) * 256 + threadIdx.x;
    if (p >= a.cols / 8) return;                               // the sixteen lanes of a group together: there is a multiple of 16 pieces
    float y[8];
    load8<F32>(a.x + (int64_t)row * a.row_bytes + (uint64_t)p * 8 * SRC, y);
    const uint32_t m = most_of_lanes<16>(most8(y));
    float scale;
    const float inv = inverse_and_scale(m, &scale);
    if ((threadIdx.x & 15) == 0) a.scale[row * (a.cols / 128) + p / 16] = scale;
    store_e4m3(a.q + row * a.cols + (uint64_t)p * 8, y, inv);
}

// Strides and addresses of rows of `dim` elements, `heads` of them a token.
int check_rows(const ecfa_rows *r, uint32_t n_tokens)
{
    if (r->dtype != ECFA_F32 && r->dtype != ECFA_BF16) return ECF8_E_ARG;
    if (n_tokens && !r->d) return ECF8_E_ARG;
    const int64_t e = r->dtype == ECFA_F32 ? 4 : 2;
    if (((uintptr_t)r->d & 15) || (apart(r->token_stride, e, n_tokens) & 15) || (apart(r->head_stride, e, r->heads) & 15)) return ECF8_E_ALIGN;
    return ECF8_OK;
}

RowsView rows_view(const ecfa_rows *r, uint32_t n_tokens)
{
    if (!r) return RowsView{nullptr, 0, 0};
    const int64_t e = r->dtype == ECFA_F32 ? 4 : 2;
    return RowsView{(uint8_t *)r->d, apart(r->token_stride, e, n_tokens), apart(r->head_stride, e, r->heads)};
}

template <bool F32, bool F8>
void launch_append(const AppendArgs &a, bool interleaved, hipStream_t s)
{
    if (interleaved) hipLaunchKernelGGL((ecfa_append_kernel<F32, F8, true>), dim3(a.b.n_tokens), dim3(APPEND_THREADS), 0, s, a);
    else hipLaunchKernelGGL((ecfa_append_kernel<F32, F8, false>), dim3(a.b.n_tokens), dim3(APPEND_THREADS), 0, s, a);
}

// Threads for a row so that it fits four pieces of eight a thread and rows are spread over the card.  BF16, 4096 rows: 512 columns with 64 threads
// 4.8 us, with 256 5.2, with 1024 13.5; 8192 columns with 256 17.8, with 64 24.6, with 1024 20.2; 16384 columns with 1024
// 32.3, with 256 37.7.
template <bool F32>
void launch_quant(const QuantArgs &a, uint32_t group, hipStream_t s)
{
    if (group) hipLaunchKernelGGL((ecfa_quant_groups_kernel<F32>), dim3((unsigned)(a.rows * a.per_row)), dim3(256), 0, s, a);
    else if (a.cols <= 1024) hipLaunchKernelGGL((ecfa_quant_rows_kernel<F32, 64>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, s, a);
    else if (a.cols <= 8192) hipLaunchKernelGGL((ecfa_quant_rows_kernel<F32, 256>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((ecfa_quant_rows_kernel<F32, 1024>), dim3((unsigned)a.rows), dim3(1024), 0, s, a);
}

} // namespace

extern "C" {

int ecfa_rope_freq(uint32_t rot_dim, double base, uint32_t kind, double factor, double original_len, double beta_fast,
                   double beta_slow, uint64_t *freq, float *scale)
{
    if (!freq || rot_dim == 0 || rot_dim % 2 || !(base > 1) || !std::isfinite(base) || kind > ECFA_ROPE_RAMP) return ECF8_E_ARG;
    if (kind == ECFA_ROPE_PLAIN) factor = 1;
    if (!(factor >= 1) || !std::isfinite(factor)) return ECF8_E_ARG;
    const double d = rot_dim;
    if (kind == ECFA_ROPE_BASE) {
        if (rot_dim == 2) return ECF8_E_ARG;
        base *= std::pow(factor, d / (d - 2));
        if (!std::isfinite(base)) return ECF8_E_ARG;
    }
    if (kind == ECFA_ROPE_RAMP && !(original_len > 0 && beta_slow > 0 && beta_fast > beta_slow && std::isfinite(original_len) && std::isfinite(beta_fast)))
        return ECF8_E_ARG;
    // The ramp is that of YaRN (arXiv 2309.00071), with its limits: index at which a pair turns `n` times within original_len,
    // original_len * base^(-2 j / d) / (2 pi) = n
    const double two_pi = 6.283185307179586476925;
    const auto index_of = [&](double n) { return d * std::log(original_len / (n * two_pi)) / (2 * std::log(base)); };
    double lo = 0, hi = 0;
    if (kind == ECFA_ROPE_RAMP) {
        lo = std::floor(index_of(beta_fast));
        hi = std::ceil(index_of(beta_slow));
        lo = lo < 0 ? 0 : lo;
        hi = hi > d - 1 ? d - 1 : hi;
        if (!(hi > lo)) hi = lo + 0.001;                       // one step at lo
    }
    for (uint32_t j = 0; j < rot_dim / 2; j++) {
        double turns = std::pow(base, -2.0 * j / d) / two_pi;
        if (kind == ECFA_ROPE_LINEAR) turns /= factor;
        if (kind == ECFA_ROPE_RAMP) {
            double w = (j - lo) / (hi - lo);                   // 0: stays, 1: divided
            w = w < 0 ? 0 : w > 1 ? 1 : w;
            turns = turns * (1 - w) + turns / factor * w;
        }
        freq[j] = (uint64_t)(turns * 18446744073709551616.0);  // below 2^62
    }
    if (scale) *scale = kind == ECFA_ROPE_RAMP ? (float)(1 + 0.1 * std::log(factor)) : 1.f;
    return ECF8_OK;
}

int ecfa_append(const ecfa_cache *cache, const ecfa_batch *batch, const ecfa_rope *rope, const ecfa_rows *q, const ecfa_rows *k,
                const ecfa_rows *v, const ecfa_rows *q_out, void *stream)
{
    AppendArgs a{};
    if (!cache || !batch || !k != !v || !q != !q_out || (!q && !k)) return ECF8_E_ARG;
    int rc = cache_view(cache, k != nullptr, &a.c);
    if (!rc) rc = batch_view(cache, batch, k != nullptr, &a.b);
    if (rc) return rc;
    const ecfa_rows *src = q ? q : k;
    for (const ecfa_rows *r : {q, k, v})
        if (r) {
            if (r->dtype != src->dtype) return ECF8_E_ARG;
            if ((rc = check_rows(r, batch->n_tokens))) return rc;
        }
    if (q) {
        if (q_out->dtype != ECFA_BF16 || q_out->heads != q->heads || q->heads == 0 || q->heads > (1u << 20)) return ECF8_E_ARG;
        if ((rc = check_rows(q_out, batch->n_tokens))) return rc;
        a.q_heads = q->heads;
    }
    if (k) {
        if (k->heads != cache->kv_heads || v->heads != cache->kv_heads) return ECF8_E_ARG;
        a.kv_heads = cache->kv_heads;
    }
    a.units = cache->head_dim / 16;
    bool interleaved = false;
    if (rope) {
        if (!rope->d_freq || rope->rot_dim == 0 || rope->rot_dim % 16 || rope->rot_dim > cache->head_dim || rope->interleaved > 1 || !std::isfinite(rope->scale))
            return ECF8_E_ARG;
        if (((uintptr_t)rope->d_freq & 7) || ((uintptr_t)rope->d_pos & 3)) return ECF8_E_ALIGN;
        a.freq = rope->d_freq;
        a.pos = rope->d_pos;
        a.rope_scale = rope->scale;
        a.rot_units = rope->rot_dim / 16;
        interleaved = rope->interleaved != 0;
    }
    a.slots = APPEND_THREADS / a.units;
    a.q = rows_view(q, batch->n_tokens);
    a.k = rows_view(k, batch->n_tokens);
    a.v = rows_view(v, batch->n_tokens);
    a.q_out = rows_view(q_out, batch->n_tokens);
    if (batch->n_tokens == 0) return ECF8_OK;
    const bool f32 = src->dtype == ECFA_F32, f8 = cache->dtype == ECFA_E4M3;
    hipStream_t s = (hipStream_t)stream;
    if (f32) f8 ? launch_append<true, true>(a, interleaved, s) : launch_append<true, false>(a, interleaved, s);
    else f8 ? launch_append<false, true>(a, interleaved, s) : launch_append<false, false>(a, interleaved, s);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

int ecfa_quant(const void *d_x, uint32_t dtype, uint64_t rows, uint64_t cols, int64_t row_stride, uint32_t group, uint8_t *d_q,
               float *d_scale, void *stream)
{
    if ((dtype != ECFA_F32 && dtype != ECFA_BF16) || (group != 0 && group != 128) || cols == 0 || cols > (1u << 20) || cols % (group ? 128 : 16)) return ECF8_E_ARG;
    if (rows && (!d_x || !d_q || !d_scale)) return ECF8_E_ARG;
    const int64_t e = dtype == ECFA_F32 ? 4 : 2;
    if (((uintptr_t)d_x & 15) || (apart(row_stride, e, rows) & 15) || ((uintptr_t)d_q & 7) || ((uintptr_t)d_scale & 3)) return ECF8_E_ALIGN;
    QuantArgs a{};
    a.x = (const uint8_t *)d_x;
    a.q = d_q;
    a.scale = d_scale;
    a.row_bytes = apart(row_stride, e, rows);
    a.rows = rows;
    a.cols = (uint32_t)cols;
    a.per_row = (uint32_t)((cols / 8 + 255) / 256);
    if (rows > 1ull << 40) return ECF8_E_ARG;
    const uint64_t most = 0x3fffff / a.per_row;                // rows of a launch: its threads are counted in 32 bits, 1024 a row at most
    for (uint64_t left = rows; left; left -= a.rows) {
        a.rows = left < most ? left : most;
        if (dtype == ECFA_F32) launch_quant<true>(a, group, (hipStream_t)stream);
        else launch_quant<false>(a, group, (hipStream_t)stream);
        if (hipGetLastError() != hipSuccess) return ECF8_E_HIP;
        a.x += (int64_t)a.rows * a.row_bytes;
        a.q += a.rows * cols;
        a.scale += a.rows * (group ? cols / 128 : 1);
    }
    return ECF8_OK;
}

} // extern "C"
