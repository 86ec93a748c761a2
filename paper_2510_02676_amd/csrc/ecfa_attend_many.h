// Attention for sequences with many rows (prompts, chunks of them): bound by the matrix cores and the softmax beside them.
//
// A workgroup takes one (tile of 128 rows, key/value head, split of the keys); each of its four waves holds 32 rows, their Q and their
// O, and all of them walk over the same 64 keys at a time, whose K and V lie in LDS as BF16 (two buffers: the next 64 keys arrive
// while the present ones are worked on, one barrier a step).  BF16 goes from memory to LDS without touching registers, E4M3 is turned into BF16
// on the way, once for the four waves.  The 16-byte pieces of a row are permuted by the row's number, so that neither the reads
// of K (16 rows, one piece) nor the transposing reads of V (4 rows, two pieces) meet in a bank.
//
// Measured: 4680 x 4680 tokens of 40 heads of 128 in 482 to 536 us (930 to 840 TFLOP/s, where a large library product reaches 1330); 2048 tokens over
// 8192 keys, causal, 250 to 285 us (960 to 845): unlike cards, the clock under that load.  2048 over 2048 tokens, 32 heads of 128, 160, 192 and 256: 61, 115, 110 and 136 us (160 runs as 192, and
// heads of more than 128 have one workgroup on a compute unit).  The matrix cores are busy for 42 % of the time and the vector ALUs for half of it: a score costs
// a multiply-add, an exponential, a share of the maximum, of the sum and of the rounding to BF16 beside its 256 products, and two waves
// of a SIMD cover one another only in part.
#pragma once
#include "ecfa_attend.h"

namespace ecfa {

template <int KC>
struct ManyShape {
    static constexpr int ROW = KC <= 2 ? 128 : KC <= 4 ? 256 : 512;   // bytes of a key's row in LDS
    static constexpr int PIECES = ROW / 16;
    static constexpr int TILE = MANY_KEYS * ROW;                      // K or V
    static constexpr int BYTES = 4 * TILE;
};

// Which piece of a row stands where: piece p of row r at place p ^ spread(r).
template <int KC>
__device__ inline int spread(int r)
{
    return KC <= 2 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
}

// The first tile of a sequence among all tiles of the launch: rows before it, in whole tiles, and one more for each sequence before it,
// which is never less than they need.
__host__ __device__ inline uint32_t first_tile(const AttendArgs &a, uint32_t s)
{
    int32_t x = a.b.q_start ? a.b.q_start[s] : (int32_t)s;
    x = x < 0 ? 0 : x > (int32_t)a.b.n_tokens ? (int32_t)a.b.n_tokens : x;
    return (uint32_t)((uint64_t)x * a.share / MANY_ROWS) + s;
}

// The row of sequence s, of `rows`, that a tile of the launch begins with, or -1: behind the sequence's last row, or before its first tile.
// The latter is what tiles before the first sequence have where the first start is above 0 (the search gives them sequence 0).
__host__ __device__ inline int32_t first_row(const AttendArgs &a, uint32_t s, uint32_t tile, int32_t rows)
{
    const uint32_t first = first_tile(a, s);
    const uint64_t row = (uint64_t)(tile - first) * MANY_ROWS;
    return tile < first || row >= (uint64_t)rows ? -1 : (int32_t)row;
}

__device__ inline uint32_t seq_of_tile(const AttendArgs &a, uint32_t tile)     // as seq_of_row
{
    uint32_t lo = 0, n = a.b.n_seqs;
    while (n > 1) {
        const uint32_t step = (n + 63) / 64, i = (threadIdx.x & 63) * step;
        const uint64_t hit = __ballot(i < n && first_tile(a, lo + i) <= tile);
        const uint32_t c = hit ? 64 - __clzll((long long)hit) : 1;
        const uint32_t skip = (c - 1) * step;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    return lo;
}

// The work of workgroup `block`, with S::BYTES of LDS.
template <int KC, bool F8, bool EXTRA>
__device__ __forceinline__ void attend_many(const AttendArgs &a, uint32_t block, uint8_t *lds)
{
    using S = ManyShape<KC>;
    typedef __attribute__((address_space(3))) uint8_t lds_u8;
    typedef __attribute__((address_space(1))) const uint8_t hbm_u8;
    constexpr int NC = 2 * KC;                                 // pieces of 16 elements along a head
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int half = lane / 32, col = lane % 32;
    // heads of keys next to each other in launch order: workgroups with the same keys then land on the same XCD where the heads
    // are a multiple of eight.  The last tiles, which see the most keys, go first.
    uint32_t at = (uint32_t)over((int32_t)block, a.by_kv_heads);
    const uint32_t kvh = block - at * a.kv_heads;
    const uint32_t split = at % a.many_splits;
    at = a.many_tiles - 1 - at / a.many_splits;
    const uint32_t s = seq_of_tile(a, at);
    const Seq sq = seq_of(a.b, s);
    const int32_t rows = sq.qn * (int32_t)a.share;
    if (rows <= a.few_rows) return;                            // the other kernel's
    const int32_t row0 = first_row(a, s, at, rows);
    if (row0 < 0) return;
    const int32_t row_end = row0 + MANY_ROWS < rows ? row0 + MANY_ROWS : rows;
    const int32_t prefix = prefix_of(a, s, sq);
    const int32_t share = (int32_t)a.share;
    const int32_t tok_a = over(row0, a.by_share), tok_b = over(row_end - 1, a.by_share);
    const KeyRange kr = keys_of(a, sq, prefix, tok_a, tok_b);
    const Split sp = split_of(kr, a.many_splits);
    const bool alone = sp.used <= 1;
    if ((int32_t)split >= (sp.used > 1 ? sp.used : 1)) return;

    const uint8_t *k0 = a.c.k + (int64_t)kvh * a.c.k_head, *v0 = a.c.v + (int64_t)kvh * a.c.v_head;
    const int32_t *table = a.b.table + (int64_t)s * a.b.table_stride;
    const uint32_t in_page = (1u << a.c.page_shift) - 1;
    const float k_scale = a.c.k_scale ? a.c.k_scale[kvh] : 1.f, v_scale = a.c.v_scale ? a.c.v_scale[kvh] : 1.f;
    const float to_log2 = factor_of(a, k_scale), cap_in = to_log2 * 2.f * a.cap_inv;

    // this lane's row
    const int32_t r = row0 + 32 * wave + col;
    const bool there = r < row_end;
    const int32_t tok = there ? over(r, a.by_share) : tok_a;
    const uint32_t head = kvh * a.share + (there ? (uint32_t)(r - tok * share) : 0u);
    const int64_t t = sq.q0 + tok;
    const int32_t place = sq.place0 + tok;
    const float slope = EXTRA && a.slopes ? a.slopes[head] * LOG2E : 0.f;
    const KeyRange own = keys_of(a, sq, prefix, tok, tok);
    bf16x8 q[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const int d = 16 * c + 8 * half;
        u32x4 x{0, 0, 0, 0};
        if (there && d < (int)a.head_dim) x = *(const u32x4 *)(a.q + t * a.q_tok + (int64_t)head * a.q_head + 2 * d);
        q[c] = __builtin_bit_cast(bf16x8, x);
    }
    f32x16 o[KC];
#pragma unroll
    for (int d = 0; d < KC; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.f;
    float m = NONE, l = 0.f;
    int poison = 0;

    const int32_t step_a = sp.first + (int32_t)split * sp.per;
    const int32_t step_b = step_a + sp.per < sp.first + sp.count ? step_a + sp.per : sp.first + sp.count;

    // The page of key 32 * step + lane as the table has it.  It is looked at a step later, so that nothing waits for the table.
    const auto entry_of = [&](int32_t step) {
        const int32_t key = 32 * step + lane;
        uint32_t e = 0xffffffffu;
        if (step < step_b && key < sq.len) e = (uint32_t)table[(uint32_t)key >> a.c.page_shift];
        return e;
    };
    // Of each of the 64 keys, whether any row of the tile may look at it
    const auto seen_by_some = [&](int32_t step, uint32_t e) {
        const int32_t key = 32 * step + lane;
        return (uint64_t)__ballot(e < a.c.n_pages && key >= kr.lo && key < kr.hi);
    };
    // This wave's 16 of the 64 keys, from memory to LDS.  Pages of 16 tokens and more hold them together (the first of them is in the
    // table if any is), and then their place is worked out by the scalar unit; smaller ones are looked up row by row.
    constexpr int LOAD_PIECES = F8 ? S::ROW / 32 : S::PIECES;  // 16-byte pieces of a row in memory
    constexpr int PER = 64 / LOAD_PIECES, LOADS = 16 / PER;    // rows of a load, loads
    const int load_row = lane / LOAD_PIECES, load_piece = lane % LOAD_PIECES;
    u32x4 kx[F8 ? LOADS : 1], vx[F8 ? LOADS : 1];
    const auto fetch_rows = [&](int n, const uint8_t *ks, const uint8_t *vs, int buffer) {
        if constexpr (F8) {
            kx[n] = *(const u32x4 *)ks;
            vx[n] = *(const u32x4 *)vs;
        } else {
            uint8_t *dst = lds + buffer * 2 * S::TILE + (16 * wave + PER * n) * S::ROW;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)ks, (lds_u8 *)dst, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((hbm_u8 *)vs, (lds_u8 *)(dst + S::TILE), 16, 0, 0);
        }
    };
    const auto piece_of = [&](int n) {                         // bytes into a row; past the head's end its start again
        const int off = 16 * (F8 ? load_piece : load_piece ^ spread<KC>(PER * n + load_row));
        return off < (int)a.head_dim * (F8 ? 1 : 2) ? off : 0;
    };
    const bool near = a.c.page_shift >= 4 && a.c.near;         // sixteen keys lie in one page, and 32 bits reach over them
    const auto fetch = [&](int32_t step, uint32_t e, int buffer) {
        if (near) {
            const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)e, 16 * wave);
            const uint64_t pg = first < a.c.n_pages ? first : 0u, in = (uint32_t)(32 * step + 16 * wave) & in_page;
            const uint8_t *ks = k0 + pg * (uint64_t)a.c.k_page + in * (uint32_t)a.c.k_tok, *vs = v0 + pg * (uint64_t)a.c.v_page + in * (uint32_t)a.c.v_tok;
#pragma unroll
            for (int n = 0; n < LOADS; n++) {
                const uint32_t row = (uint32_t)(PER * n + load_row), piece = (uint32_t)piece_of(n);
                fetch_rows(n, ks + (row * (uint32_t)a.c.k_tok + piece), vs + (row * (uint32_t)a.c.v_tok + piece), buffer);
            }
        } else {
#pragma unroll
            for (int n = 0; n < LOADS; n++) {
                const int row = 16 * wave + PER * n + load_row;
                const uint32_t mine = (uint32_t)__shfl((int)e, row);
                const int64_t pg = mine < a.c.n_pages ? mine : 0u, in = (uint32_t)(32 * step + row) & in_page;
                fetch_rows(n, k0 + pg * a.c.k_page + in * a.c.k_tok + piece_of(n), v0 + pg * a.c.v_page + in * a.c.v_tok + piece_of(n), buffer);
            }
        }
    };
    const auto store = [&](int buffer) {
        if constexpr (F8) {
#pragma unroll
            for (int n = 0; n < LOADS; n++) {
                const int row = 16 * wave + PER * n + load_row, piece = load_piece;
                if (16 * piece < (int)a.head_dim) {
                    uint8_t *dst = lds + buffer * 2 * S::TILE + row * S::ROW;
                    const int p0 = (2 * piece ^ spread<KC>(row & 15)) * 16, p1 = ((2 * piece + 1) ^ spread<KC>(row & 15)) * 16;
                    *(bf16x8 *)(dst + p0) = bf16_of_e4m3(kx[n][0], kx[n][1]);
                    *(bf16x8 *)(dst + p1) = bf16_of_e4m3(kx[n][2], kx[n][3]);
                    *(bf16x8 *)(dst + S::TILE + p0) = bf16_of_e4m3(vx[n][0], vx[n][1]);
                    *(bf16x8 *)(dst + S::TILE + p1) = bf16_of_e4m3(vx[n][2], vx[n][3]);
                }
            }
        }
    };

    // where this lane reads K and V: bytes from the start of a tile; chunks of a head by exclusive or, keys by addition
    const int k_at = col * S::ROW + ((half ^ spread<KC>(col & 15)) << 4);
    const int vr = 4 * half + lane % 16 / 4, vp = 2 * (lane / 16 % 2) + lane % 4 / 2;
    const int v_at = vr * S::ROW + ((vp ^ spread<KC>(vr)) << 4) + 8 * (lane & 1);
    const int v_at8 = (vr + 8) * S::ROW + ((vp ^ spread<KC>(vr + 8)) << 4) + 8 * (lane & 1);
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
    // Eight keys of V: of 16 that begin at `keys`, elements 32 d .. of the head; `y0`, `y1`: this lane's places in the first 16 keys
    const auto v_frag = [&](int y0, int y1, int d, int keys) {
        const bf16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(uintptr_t)(uint32_t)((y0 ^ d << 6) + keys * S::ROW));
        const bf16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(uintptr_t)(uint32_t)((y1 ^ d << 6) + keys * S::ROW));
        return bf16x8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
    };
    const int lds0 = (int)(uint32_t)(uintptr_t)(lds_u8 *)lds;

    uint32_t entry = entry_of(step_a);
    uint64_t ok = seen_by_some(step_a, entry);
    if (step_a < step_b) fetch(step_a, entry, 0);
    store(0);
    entry = entry_of(step_a + 2);
    int buffer = 0;
    for (int32_t step = step_a; step < step_b; step += 2) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // loads into LDS are no loads to the barrier's own wait
        __syncthreads();                                       // this step's keys are here, and nobody reads the other buffer any more
        const uint64_t ok_now = ok;
        ok = seen_by_some(step + 2, entry);
        if (step + 2 < step_b) fetch(step + 2, entry, buffer ^ 1);
        entry = entry_of(step + 4);
        if (ok_now != ~0ull) {                                 // values that nobody may see, as zeros (the same for all waves)
            const int row = 16 * wave + lane / 4;
            if (!(ok_now >> row & 1))
#pragma unroll 1
                for (int i = 16 * (lane % 4); i < S::ROW; i += 64) *(u32x4 *)(lds + (2 * buffer + 1) * S::TILE + row * S::ROW + i) = u32x4{0, 0, 0, 0};
            __syncthreads();
        }
        // Made anew each step, from three registers instead of kept in sixteen
        int ka = lds0 + buffer * 2 * S::TILE + k_at, va = lds0 + buffer * 2 * S::TILE + S::TILE + v_at, va8 = lds0 + buffer * 2 * S::TILE + S::TILE + v_at8;
        asm volatile("" : "+v"(ka), "+v"(va), "+v"(va8));
        f32x16 x[2];
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 16; i++) x[u][i] = 0.f;
        const auto scores = [&](auto ends) {                   // `ends`: the head ends before the kernel's pieces do; zeros past its end
#pragma unroll
            for (int c = 0; c < NC; c++)
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    bf16x8 kf = *(lds_bf16x8 *)(uintptr_t)(uint32_t)((ka ^ c << 5) + u * 32 * S::ROW);
                    if (ends.value && 16 * c >= (int)a.head_dim) kf = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
                    x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[c], x[u], 0, 0, 0);
                }
            if constexpr (!ends.value) {                       // reads four ahead of the products (1 %)
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int i = 0; i < 2 * NC - 4; i++) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            }
        };
        if (a.head_dim == KC * 32) scores(std::false_type());
        else scores(std::true_type());
        const int32_t key0 = 32 * step;
        const bool whole = ok_now == ~0ull && key0 >= kr.full_lo && key0 + 64 <= kr.full_hi;
        // x[u][i]: row `col`, key 32 u + 8 (i / 4) + 4 half + i % 4
        float c_log2 = to_log2;
        if constexpr (EXTRA) {
            c_log2 = 1.f;
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int i = 0; i < 16; i++) x[u][i] = capped_or_scaled(a, x[u][i], to_log2, cap_in);
            if (a.slopes)
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int i = 0; i < 16; i++) x[u][i] = less_distance(x[u][i], slope, place - (key0 + 32 * u + 8 * (i / 4) + 4 * half + i % 4));
        }
        uint64_t seen = ~0ull;
        if (!whole) {
            const int32_t below = own.lo - key0, above = own.hi - key0;
            seen = ok_now;
            seen &= above >= 64 ? ~0ull : above <= 0 ? 0ull : (1ull << above) - 1;
            seen &= below <= 0 ? ~0ull : below >= 64 ? 0ull : ~((1ull << below) - 1);
            const uint32_t s0 = (uint32_t)seen >> (4 * half), s1 = (uint32_t)(seen >> 32) >> (4 * half);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const uint32_t bit = 1u << (8 * (i / 4) + i % 4);
                if (!(s0 & bit)) x[0][i] = NONE;
                if (!(s1 & bit)) x[1][i] = NONE;
            }
        }
        float top = NONE;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = max_f(top, x[u][i]);
        top = max_xor<32>(top) * c_log2;
        // The maximum follows only where a score has outgrown it by 2^8: weights up to there lose nothing in BF16 or in the sums
        if (__any(top > m + 8.f)) {
            const float m_new = max_f(m, top);
            const float shrink = exp2_fast(m - (m_new == NONE ? 0.f : m_new));
            m = m_new;
            l *= shrink;
#pragma unroll
            for (int d = 0; d < KC; d++)
                o[d] *= shrink;
        }
        const float base = m == NONE ? 0.f : m;
        u32x4 pw[4];
        float l0 = 0.f, l1 = 0.f;
        const bf16x2 ones{(__bf16)1.f, (__bf16)1.f};
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const bf16x2 w = bf16_pair(exp2_fast(__builtin_fmaf(x[u][i], c_log2, -base)), exp2_fast(__builtin_fmaf(x[u][i + 1], c_log2, -base)));
                pw[2 * u + i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, w);
                if (i % 4) l1 = __builtin_amdgcn_fdot2_f32_bf16(w, ones, l1, false);
                else l0 = __builtin_amdgcn_fdot2_f32_bf16(w, ones, l0, false);
            }
        l += l0 + l1;
        bf16x8 p[4];
#pragma unroll
        for (int n = 0; n < 4; n++) p[n] = __builtin_bit_cast(bf16x8, pw[n]);

        if (!whole && tok_b > tok_a) {                         // rows that see different keys: 0 * v is 0 unless v is NaN or infinite
            const bf16x8 zero = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
#pragma unroll 1
            for (int d = 0; d < KC; d++) {
                f32x16 z;
                for (int i = 0; i < 16; i++) z[i] = 0.f;
#pragma unroll
                for (int n = 0; n < 4; n++) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(va, va8, d, 16 * n), zero, z, 0, 0, 0);
                for (int i = 0; i < 16; i++)                   // (elements past the head's end are not its own)
                    poison |= z[i] != 0.f && 32 * d + 8 * (i / 4) + 4 * half < (int)a.head_dim ? 1 : 0;
            }
        }
        // O^T += V^T P^T.  (The first read also waits for the next step's keys, which have been on their way since the barrier by then: reads
        // that do not, as in the few-rows kernel, were 2 % slower here.)
#pragma unroll
        for (int n = 0; n < 4; n++)
#pragma unroll
            for (int d = 0; d < KC; d++) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(va, va8, d, 16 * n), p[n], o[d], 0, 0, 0);
        store(buffer ^ 1);
        buffer ^= 1;
    }

    float all = sum_xor<32>(l);
    if (__any(poison)) {
        float y[16 * KC];
        attend_slowly<F8, 2, 4 * KC>(a, a.q + t * a.q_tok + (int64_t)head * a.q_head, k0, v0, table, step_a, step_b, 1, 1, own, place, to_log2, slope, half,
                                     [&](int n) { return 8 * n + 4 * half; }, y, m, all);
#pragma unroll
        for (int d = 0; d < KC; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[d][i] = y[16 * d + i];
    }
    if (!there) return;
    if (alone) {
        const float inv = all == 0.f ? 0.f : v_scale / all;
        uint8_t *dst = a.out + t * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
        for (int d = 0; d < KC; d++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int e = 32 * d + 8 * j + 4 * half;
                bf16x4 y;
                for (int i = 0; i < 4; i++) y[i] = (__bf16)(all == 0.f ? 0.f : o[d][4 * j + i] * inv);
                if (e < (int)a.head_dim) *(bf16x4 *)(dst + 2 * e) = y;
            }
    } else {
        const int64_t part = many_part(a, t, head) + split;
#pragma unroll
        for (int d = 0; d < KC; d++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int e = 32 * d + 8 * j + 4 * half;
                f32x4 y;
                for (int i = 0; i < 4; i++) y[i] = o[d][4 * j + i] * v_scale;
                if (e < (int)a.head_dim) *(f32x4 *)(a.part + part * a.head_dim + e) = y;
            }
        if (half == 0) {
            a.part_ml[2 * part] = m;
            a.part_ml[2 * part + 1] = all;
        }
    }
}

template <int KC, bool F8, bool EXTRA>
__global__ __launch_bounds__(MANY_WAVES * 64, KC <= 4 ? 2 : 1) void ecfa_attend_many_kernel(const AttendArgs a)
{
    __shared__ __align__(16) uint8_t lds[ManyShape<KC>::BYTES];
    attend_many<KC, F8, EXTRA>(a, blockIdx.x, lds);
}

} // namespace ecfa
