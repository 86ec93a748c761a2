// Host side that the attention calls share: checks of a cache and a batch, and the kernels' view of them.
#pragma once
#include "ecfa_device.h"

namespace ecfa {

constexpr uint32_t MAX_TOKENS = 1u << 22;      // of a step: a launch counts its threads in 32 bits, 256 to 512 a token

// The bytes from one of n to the next, 0 where there is no next: then the caller's stride does not count, whatever it is.
inline int64_t apart(int64_t stride, int64_t bytes, uint64_t n) { return n > 1 ? stride * bytes : 0; }

// `used`: whether the call touches the pool (else only head_dim, page_size and dtype count).
inline int cache_view(const ecfa_cache *c, bool used, CacheView *o)
{
    if ((c->dtype != ECFA_BF16 && c->dtype != ECFA_E4M3) || c->head_dim == 0 || c->head_dim % 16 || c->head_dim > 256) return ECF8_E_ARG;
    if (c->page_size == 0 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return ECF8_E_ARG;
    o->page_shift = (uint32_t)__builtin_ctz(c->page_size);
    if (!used) return ECF8_OK;
    if (!c->d_k || !c->d_v || c->n_pages == 0 || c->n_pages > 0x7fffffffu || c->kv_heads == 0 || c->kv_heads > (1u << 20)) return ECF8_E_ARG;
    const int64_t e = c->dtype == ECFA_BF16 ? 2 : 1;
    if (((uintptr_t)c->d_k & 15) || ((uintptr_t)c->d_v & 15) || ((uintptr_t)c->d_k_scale & 3) || ((uintptr_t)c->d_v_scale & 3)) return ECF8_E_ALIGN;
    const uint32_t n[3] = {c->n_pages, c->page_size, c->kv_heads};
    int64_t k[3], v[3];
    for (int i = 0; i < 3; i++) {
        k[i] = apart(c->k_stride[i], e, n[i]);
        v[i] = apart(c->v_stride[i], e, n[i]);
        if ((k[i] & 15) || (v[i] & 15)) return ECF8_E_ALIGN;
    }
    o->k = (uint8_t *)c->d_k;
    o->v = (uint8_t *)c->d_v;
    o->k_scale = c->d_k_scale;
    o->v_scale = c->d_v_scale;
    o->k_page = k[0];
    o->k_tok = k[1];
    o->k_head = k[2];
    o->v_page = v[0];
    o->v_tok = v[1];
    o->v_head = v[2];
    o->n_pages = c->n_pages;
    o->near = o->k_tok >= 0 && o->v_tok >= 0 && o->k_tok < (1 << 25) && o->v_tok < (1 << 25);
    return ECF8_OK;
}

// `paged`: whether the call looks at the page table.
inline int batch_view(const ecfa_cache *c, const ecfa_batch *b, bool paged, BatchView *o)
{
    if (b->n_tokens > MAX_TOKENS || b->n_seqs > MAX_TOKENS || (b->n_tokens && b->n_seqs == 0)) return ECF8_E_ARG;
    if (!b->d_q_start && b->n_tokens != b->n_seqs) return ECF8_E_ARG;
    if (b->n_tokens && (!b->d_kv_len || (paged && (!b->d_page_table || b->table_width == 0)))) return ECF8_E_ARG;
    if (paged && (uint64_t)b->table_width * c->page_size > MAX_KEYS) return ECF8_E_ARG;
    if (((uintptr_t)b->d_page_table & 3) || ((uintptr_t)b->d_kv_len & 3) || ((uintptr_t)b->d_q_start & 3)) return ECF8_E_ALIGN;
    o->table = b->d_page_table;
    o->kv_len = b->d_kv_len;
    o->q_start = b->d_q_start;
    o->table_stride = b->table_stride;
    o->keys_max = paged ? b->table_width * c->page_size : MAX_KEYS;
    o->n_seqs = b->n_seqs;
    o->n_tokens = b->n_tokens;
    return ECF8_OK;
}

} // namespace ecfa
