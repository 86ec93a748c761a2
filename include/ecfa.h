/*
 * ecfa.h -- C ABI of the attention between a layer's compressed projections.
 *
 * The fused products of ecf8.h give q, k and v of a layer as rows; its output
 * projection reads E4M3 rows with scales.  The calls here are what lies between:
 *
 *   ecfa_append   turns q and k by their positions (rotary embedding) and writes
 *                 k and v into a paged cache, in one launch
 *   ecfa_attend   lets the new tokens of every sequence (one, or a chunk) attend
 *                 to the keys and values of that sequence in the cache
 *   ecfa_quant    rounds rows to E4M3 with a scale per row or per 128 columns: X
 *                 and d_x_scale of ecf8_gemm_fp8_scaled
 *
 * Conventions are those of ecf8.h: plain pointers, DEVICE memory is the caller's,
 * nothing is allocated, nothing waits for the device, `stream` is a hipStream_t (NULL =
 * the default stream), all calls may be captured into a HIP graph, and every function
 * returns ECF8_OK or a negative ECF8_E_* code (ecf8_strerror).  Structures are HOST
 * memory and are read before the call returns.  What is in DEVICE memory (page
 * tables, lengths, starts) is read when the kernels run, so that a captured call
 * follows a loop that rewrites them; no value there makes a kernel access
 * memory outside of the buffers that the structures describe.
 */
#ifndef ECFA_H
#define ECFA_H

#include "ecf8.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ECFA_F32 = 1, ECFA_BF16 = 2, ECFA_E4M3 = 3 };

/* Rows of heads: element e of head h of token t is at d[t * token_stride + h * head_stride + e].
 * Strides are in elements; d, and both strides in bytes, are multiples of 16 (ECF8_E_ALIGN).
 * Here and below, a stride between things of which there is one does not count. */
typedef struct ecfa_rows {
    void *d;                       /* DEVICE                                            */
    int64_t token_stride, head_stride;
    uint32_t heads;
    uint32_t dtype;                /* ECFA_F32 or ECFA_BF16                             */
} ecfa_rows;

/* A pool of pages.  Element e of head h of the t-th token of page p is at
 * d_k[p * k_stride[0] + t * k_stride[1] + h * k_stride[2] + e], and so for d_v; strides
 * are in elements, so the pool may be ordered by token or by head.  Addresses and strides
 * in bytes are multiples of 16.  The value of an element is what is stored times the
 * scale of its head (NULL: 1); scales are positive.  E4M3 is OCP "fn". */
typedef struct ecfa_cache {
    void *d_k, *d_v;               /* DEVICE                                            */
    const float *d_k_scale;        /* DEVICE, kv_heads, or NULL                         */
    const float *d_v_scale;
    int64_t k_stride[3], v_stride[3];
    uint32_t n_pages;              /* 1 .. 2^31 - 1                                     */
    uint32_t page_size;            /* tokens of a page, a power of two up to 65536      */
    uint32_t kv_heads;
    uint32_t head_dim;             /* a multiple of 16, up to 256                       */
    uint32_t dtype;                /* ECFA_BF16 or ECFA_E4M3                            */
    uint32_t reserved;
} ecfa_cache;

/* One step of a serving loop.  Sequence s owns the new tokens q_start[s] .. q_start[s + 1]
 * (rows of q, k, v, out); its cache holds kv_len[s] tokens, the new ones among them (they
 * are the last ones), and key j of it is token j % page_size of page
 * page_table[s * table_stride + j / page_size].  A page number outside of the pool is a
 * hole: nothing is written there, and its keys are seen by nobody.  Keys beyond the
 * table's width are holes too.  Rows before the first start and from the last one on belong
 * to no sequence: what they would give is not written. */
typedef struct ecfa_batch {
    const int32_t *d_page_table;   /* DEVICE, n_seqs x table_width                      */
    const int32_t *d_kv_len;       /* DEVICE, n_seqs                                    */
    const int32_t *d_q_start;      /* DEVICE, n_seqs + 1, rising from 0; NULL: one new token each (n_tokens = n_seqs) */
    int64_t table_stride;          /* elements                                          */
    uint32_t table_width;          /* pages; table_width * page_size <= 2^30            */
    uint32_t n_seqs;               /* up to 2^22                                        */
    uint32_t n_tokens;             /* rows that there are, up to 2^22; starts outside are cut */
    uint32_t max_q;                /* hints for the launch, 0 = not known: the most new tokens and  */
    uint32_t max_kv;               /* the most keys of a sequence.  Results do not depend on them   */
    uint32_t reserved;
} ecfa_batch;

/* Rotary positions.  freq[j] is what position 1 turns pair j by, in 2^-64 of a full
 * turn; the angle of position p is p * freq[j] modulo one turn, in integers, so it is
 * as exact at position 10^6 as at 1.  Pair j is elements (j, j + rot_dim / 2), or (2 j,
 * 2 j + 1) if interleaved; elements from rot_dim on stay as they are.  (a, b) becomes
 * scale * (a cos - b sin, b cos + a sin). */
typedef struct ecfa_rope {
    const uint64_t *d_freq;        /* DEVICE, rot_dim / 2                               */
    const int32_t *d_pos;          /* DEVICE, n_tokens, or NULL: the place in the cache */
    uint32_t rot_dim;              /* a multiple of 16, up to head_dim                  */
    uint32_t interleaved;
    float scale;                   /* 1 unless the long-context scaling asks for more   */
    uint32_t reserved;
} ecfa_rope;

/*
 * ecfa_rope_freq (HOST): fills freq[rot_dim / 2] with base^(-2 j / rot_dim) / (2 pi) turns
 * and *scale (may be NULL) with the factor of ecfa_rope, stretched for contexts longer than
 * a model was trained on (RAMP with the steps and the limits of YaRN, arXiv 2309.00071, which
 * checkpoints that were stretched that way expect):
 *   ECFA_ROPE_PLAIN   as it is; factor and the others are ignored
 *   ECFA_ROPE_LINEAR  all frequencies divided by factor
 *   ECFA_ROPE_BASE    base * factor^(rot_dim / (rot_dim - 2)): the fastest pair stays, the
 *                     slowest is divided by factor
 *   ECFA_ROPE_RAMP    pairs that turn more than beta_fast times within original_len stay,
 *                     those of less than beta_slow turns are divided by factor, the ones
 *                     between are blended linearly by index; scale = 1 + 0.1 ln(factor)
 * ECF8_E_ARG: rot_dim 0 or odd, base <= 1, factor < 1, an unknown kind, a ramp without
 * original_len > 0 and beta_fast > beta_slow > 0, BASE with rot_dim 2.
 */
enum { ECFA_ROPE_PLAIN = 0, ECFA_ROPE_LINEAR = 1, ECFA_ROPE_BASE = 2, ECFA_ROPE_RAMP = 3 };
int ecfa_rope_freq(uint32_t rot_dim, double base, uint32_t kind, double factor, double original_len,
                   double beta_fast, double beta_slow, uint64_t *freq, float *scale);

/*
 * ecfa_append: for each new token, k turned and v go to the cache, at the token's place, and
 * q turned goes to q_out (BF16).  Angles and products are fp32; one rounding to the
 * cache's type, E4M3 after division by the head's scale and limited to +-448.  q and
 * q_out may be NULL (no q), k and v may both be NULL (q only; `cache` then gives head_dim
 * and page_size, its buffers are not touched); rope may be NULL (nothing turns).  q_out may be q itself
 * if q is BF16.  Tokens whose place is before 0 or in a hole are not written to the cache.
 * Two tokens with the same place (a page in two sequences) leave either one's values.
 */
int ecfa_append(const ecfa_cache *cache, const ecfa_batch *batch, const ecfa_rope *rope, const ecfa_rows *q,
                const ecfa_rows *k, const ecfa_rows *v, const ecfa_rows *q_out, void *stream);

/*
 * ecfa_attend: out[t][h] = sum over keys j of softmax_j(x_j) * v_j, with key/value head
 * h / (q->heads / kv_heads), place p = kv_len - (new tokens of the sequence) + (index of t among them),
 *   x_j = scale * q . k_j;  softcap > 0: x_j = softcap * tanh(x_j / softcap);  d_slopes: x_j -= slopes[h] * |p - j|
 * over the keys j < kv_len that are no holes and
 *   causal: j <= p, or j < prefix_len[s];   window > 0: j > p - window (not together with prefix_len).
 * A token that sees no key gets zeros.  What is stored in keys and values that a token does
 * not see (NaN, infinities) does not reach it.  q and out are BF16; products of BF16, sums
 * and softmax in fp32, so that scores have to lie within fp32; the weights are rounded to BF16
 * before they meet the values, and their sum is taken of the rounded ones.  With a cap of up to
 * 64 a score is off by 2^-23 of the cap at most, with a larger one only in proportion to itself.
 *
 * Where there are few rows, long sequences are split among workgroups that leave partial sums in
 * d_workspace (DEVICE, 16-byte aligned, of ecfa_attend_workspace_bytes(), which serves any options
 * of a call with this batch; NULL where that is 0), and a second kernel joins them; the split
 * depends on shapes, options and lengths alone, so the same call gives the same bits.  Calls that
 * overlap in time need a workspace each.
 * ECF8_E_ARG also: over 2^30 rows to a key/value head (n_tokens * q->heads / kv_heads) or over 2^24
 * workgroups, which 2^20 single tokens with 8 key/value heads come near; ecfa_attend_workspace_bytes
 * is 0 then.
 */
typedef struct ecfa_attend_opts {
    float scale;                   /* > 0                                               */
    float softcap;                 /* 0: none                                           */
    const float *d_slopes;         /* DEVICE, q->heads, or NULL                         */
    const int32_t *d_prefix_len;   /* DEVICE, n_seqs, or NULL                           */
    uint32_t causal;               /* 0 or 1                                            */
    uint32_t window;               /* 0: all keys                                       */
} ecfa_attend_opts;

uint64_t ecfa_attend_workspace_bytes(const ecfa_cache *cache, const ecfa_batch *batch, uint32_t heads);
int ecfa_attend(const ecfa_cache *cache, const ecfa_batch *batch, const ecfa_attend_opts *opts, const ecfa_rows *q,
                const ecfa_rows *out, void *d_workspace, uint64_t workspace_bytes, void *stream);

/*
 * ecfa_quant: x (rows x cols, BF16 or fp32, row_stride elements between rows) to E4M3 bytes d_q
 * (rows x cols, dense) and scales: per row (group = 0, d_scale[rows]) or per 128 columns
 * (group = 128, d_scale[rows][cols / 128]).  With a = max(|x| of the row or group, 2^-100):
 * scale = a / 448, q = x * (448 / a) rounded to the nearest, ties to even; q * scale is x again within
 * half a step.  A group with an infinity or a NaN has that as its scale.
 * cols: a multiple of 16 (of 128 with groups), up to 2^20.
 */
int ecfa_quant(const void *d_x, uint32_t dtype, uint64_t rows, uint64_t cols, int64_t row_stride, uint32_t group,
               uint8_t *d_q, float *d_scale, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECFA_H */
