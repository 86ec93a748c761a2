// What the attention kernels share: the kernel's view of a cache and a batch, and where a token stands in them.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "ecfa.h"

namespace ecfa {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr uint32_t MAX_KEYS = 1u << 30;      // of a sequence: places and their ends stay well inside 32 signed bits

struct CacheView {                           // strides in bytes
    uint8_t *k, *v;
    const float *k_scale, *v_scale;
    int64_t k_page, k_tok, k_head, v_page, v_tok, v_head;
    uint32_t n_pages, page_shift;
    uint32_t near;                           // tokens of a page lie less than 2^25 bytes apart: offsets over 16 of them fit 32 bits
                                             // (2048 tokens of 8192 keys 262 us, with an address a lane 286; 131072 keys 109.4, 111.2)
};

struct BatchView {
    const int32_t *table, *kv_len, *q_start;
    int64_t table_stride;
    uint32_t keys_max;                       // table_width * page_size
    uint32_t n_seqs, n_tokens;
};

struct Seq {
    int32_t q0, qn;                          // its rows
    int32_t place0;                          // place of its first new token; may be negative
    int32_t len;                             // keys that the table has room for
};

__host__ __device__ inline Seq seq_of(const BatchView &b, uint32_t s)
{
    Seq r;
    int32_t kv = b.kv_len[s];
    kv = kv < 0 ? 0 : kv > (int32_t)MAX_KEYS ? (int32_t)MAX_KEYS : kv;
    if (b.q_start) {
        const int32_t n = (int32_t)b.n_tokens;
        int32_t x = b.q_start[s], y = b.q_start[s + 1];
        x = x < 0 ? 0 : x > n ? n : x;
        y = y < x ? x : y > n ? n : y;
        r.q0 = x;
        r.qn = y - x;
    } else {
        r.q0 = (int32_t)s;
        r.qn = 1;
    }
    r.place0 = kv - r.qn;
    r.len = kv > (int32_t)b.keys_max ? (int32_t)b.keys_max : kv;
    return r;
}

// The sequence that row t belongs to: the last one that begins at or before it, found by all lanes of a wave together,
// 64 starts at a time (one round trip to memory up to 64 sequences, two up to 4096).  Rows before the first start get 0.
__device__ inline uint32_t seq_of_row(const BatchView &b, uint32_t t)
{
    if (!b.q_start) return t;
    uint32_t lo = 0, n = b.n_seqs;                                   // the answer is in [lo, lo + n)
    while (n > 1) {
        const uint32_t step = (n + 63) / 64;
        const uint64_t at = (uint64_t)lo + (uint64_t)(threadIdx.x & 63) * step;
        const bool begun = (threadIdx.x & 63) * step < n && b.q_start[at] <= (int32_t)t;
        const uint64_t hit = __ballot(begun);
        const uint32_t c = hit ? 64 - __clzll((long long)hit) : 1;   // probes up to the last that has begun
        const uint32_t skip = (c - 1) * step;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    return lo;
}

__device__ inline uint32_t f32_bits(float x) { return __builtin_bit_cast(uint32_t, x); }

} // namespace ecfa
