// Attention for sequences with few rows (a decode step: the heads of one token that share their keys): bound by reading K and V once.
//
// A workgroup takes one (sequence, key/value head, split of its keys, tile of 16 NT rows); its four waves take every fourth step of
// 32 keys each and do not meet until the end, where their (m, l, O) are joined in LDS.  K goes from memory straight into the
// registers that the matrix cores read it from (lane l: key l % 16, eight elements of the head); V passes through a piece of LDS that
// belongs to the wave, which turns it (no barrier).  The next step's K and V are fetched while the present one is worked on.
#pragma once
#include "ecfa_attend.h"

namespace ecfa {

template <int KC, bool F8, int NT>
struct FewShape {
    static constexpr int E = F8 ? 1 : 2;
    static constexpr int ROW = KC * 32 * E, PAD = F8 ? 16 : 32;      // bytes; the pad spreads the rows that a transposing read touches over the banks
    static constexpr int STRIDE = ROW + PAD;
    static constexpr int V_BYTES = 32 * STRIDE;                      // of a wave
    static constexpr int O_STRIDE = KC * 32 + 4;                     // floats
    static constexpr int JOIN_BYTES = FEW_WAVES * 16 * (O_STRIDE + 2) * 4;
    static constexpr int MAIN_BYTES = FEW_WAVES * V_BYTES;
    static constexpr int BYTES = MAIN_BYTES > JOIN_BYTES ? MAIN_BYTES : JOIN_BYTES;
};

template <int KC, bool F8, int NT>
__global__ __launch_bounds__(FEW_WAVES * 64, 2) void ecfa_attend_few_kernel(const AttendArgs a)
{
    using S = FewShape<KC, F8, NT>;
    constexpr int E = S::E;
    __shared__ __align__(16) uint8_t lds[S::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, col = lane % 16;
    uint32_t at = blockIdx.x;
    const uint32_t split = at % a.few_splits;
    at /= a.few_splits;
    const uint32_t kvh = at % a.kv_heads, s = at / a.kv_heads;
    const Seq sq = seq_of(a.b, s);
    const int32_t prefix = prefix_of(a, s, sq);
    const int32_t rows = sq.qn * (int32_t)a.share;
    if (rows > a.few_rows) return;                             // the other kernel's
    const uint8_t *k0 = a.c.k + (int64_t)kvh * a.c.k_head, *v0 = a.c.v + (int64_t)kvh * a.c.v_head;
    const int32_t *table = a.b.table + (int64_t)s * a.b.table_stride;
    const uint32_t in_page = (1u << a.c.page_shift) - 1;
    const float k_scale = a.c.k_scale ? a.c.k_scale[kvh] : 1.f, v_scale = a.c.v_scale ? a.c.v_scale[kvh] : 1.f;
    const float to_log2 = a.scale_log2 * k_scale;
    uint8_t *my_v = lds + wave * S::V_BYTES;

    // max_q is a hint: if a sequence has more rows than a tile after all, the tiles follow one another
    for (int32_t row0 = 0; row0 < rows; row0 += 16 * NT) {
        const int32_t row_end = row0 + 16 * NT < rows ? row0 + 16 * NT : rows;
        const int32_t tok_a = row0 / (int32_t)a.share, tok_b = (row_end - 1) / (int32_t)a.share;
        const KeyRange kr = keys_of(a, sq, prefix, tok_a, tok_b);
        const Split sp = split_of(kr, row0 == 0 ? a.few_splits : 1, FEW_UNIT);
        const bool alone = sp.used <= 1;
        if ((int32_t)split >= (sp.used > 1 ? sp.used : 1)) continue;

        // this lane's rows, one of each sub-tile
        int64_t o_at[NT];
        int32_t lo[NT], hi[NT], place[NT];
        float slope[NT];
        bf16x8 q[NT][KC];
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const int32_t r = row0 + 16 * n + col;
            const bool there = r < row_end;
            const int32_t tok = there ? r / (int32_t)a.share : tok_a;
            const uint32_t head = kvh * a.share + (there ? (uint32_t)r % a.share : 0);
            const int64_t t = sq.q0 + tok;
            o_at[n] = t * a.o_tok + (int64_t)head * a.o_head;
            place[n] = sq.place0 + tok;
            slope[n] = a.slopes ? a.slopes[head] * LOG2E : 0.f;
            const KeyRange own = keys_of(a, sq, prefix, tok, tok);
            lo[n] = own.lo;
            hi[n] = own.hi;
            const uint8_t *src = a.q + t * a.q_tok + (int64_t)head * a.q_head;
#pragma unroll
            for (int c = 0; c < KC; c++) {
                const int d = F8 && c < (KC & ~1) ? 64 * (c / 2) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
                u32x4 x{0, 0, 0, 0};
                if (there && d < (int)a.head_dim) x = *(const u32x4 *)(src + 2 * d);
                q[n][c] = __builtin_bit_cast(bf16x8, x);
            }
        }

        f32x4 o[NT][2 * KC];
        float m[NT], l[NT];
        int poison = 0;
#pragma unroll
        for (int n = 0; n < NT; n++) {
            m[n] = NONE;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < 2 * KC; d++) o[n][d] = f32x4{0, 0, 0, 0};
        }

        const int32_t step_a = sp.first + (int32_t)split * sp.per;
        const int32_t step_b = step_a + sp.per < sp.first + sp.count ? step_a + sp.per : sp.first + sp.count;

        // the page of key 32 * step + lane % 32, and whether any row may look at that key
        const auto pages_of = [&](int32_t step, uint32_t &page, uint32_t &ok) {
            const int32_t key = 32 * step + (lane & 31);
            uint32_t e = 0xffffffffu;
            if (step < step_b && key >= kr.lo && key < kr.hi) e = (uint32_t)table[(uint32_t)key >> a.c.page_shift];
            const bool fine = e < a.c.n_pages;
            page = fine ? e : 0u;                              // page 0 exists: what is read of it for a hole is not used
            ok = (uint32_t)__ballot(fine);
        };
        uint32_t kx[2][KC][F8 ? 2 : 4];
        u32x4 vx[F8 ? KC : 2 * KC];
        constexpr int PIECES = S::ROW / 16;
        const auto fetch = [&](int32_t step, uint32_t page) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const uint32_t in = (uint32_t)(32 * step + 16 * u + col) & in_page;
                const uint8_t *src = k0 + (int64_t)(uint32_t)__shfl((int)page, 16 * u + col) * a.c.k_page + (int64_t)in * a.c.k_tok;
#pragma unroll
                for (int c = 0; c < KC; c++) {
                    if constexpr (F8) {
                        if (c + 1 < KC && c % 2 == 0) {
                            const int d = 64 * (c / 2) + 16 * g;
                            const u32x4 x = *(const u32x4 *)(src + (d < (int)a.head_dim ? d : 0));
                            kx[u][c][0] = x[0], kx[u][c][1] = x[1], kx[u][c + 1][0] = x[2], kx[u][c + 1][1] = x[3];
                        } else if (c % 2 == 0) {
                            const int d = 32 * c + 8 * g;
                            const u32x2 x = *(const u32x2 *)(src + (d < (int)a.head_dim ? d : 0));
                            kx[u][c][0] = x[0], kx[u][c][1] = x[1];
                        }
                    } else {
                        const int d = 32 * c + 8 * g;
                        const u32x4 x = *(const u32x4 *)(src + 2 * (d < (int)a.head_dim ? d : 0));
                        for (int i = 0; i < 4; i++) kx[u][c][i] = x[i];
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < (int)(sizeof(vx) / sizeof(vx[0])); n++) {
                const int row = (64 * n + lane) / PIECES, piece = (64 * n + lane) % PIECES;
                const uint32_t in = (uint32_t)(32 * step + row) & in_page;
                const uint8_t *src = v0 + (int64_t)(uint32_t)__shfl((int)page, row) * a.c.v_page + (int64_t)in * a.c.v_tok;
                vx[n] = *(const u32x4 *)(src + (16 * piece < (int)a.head_dim * E ? 16 * piece : 0));
            }
        };

        uint32_t page, ok, page_next, ok_next;
        int32_t step = step_a + wave;
        pages_of(step, page, ok);
        if (step < step_b) fetch(step, page);
        pages_of(step + FEW_WAVES, page_next, ok_next);
        for (; step < step_b; step += FEW_WAVES) {
            // V of this step to LDS; keys that nobody sees as zeros
            lds_fence_wave();                                  // the reads of the step before are done with
#pragma unroll
            for (int n = 0; n < (int)(sizeof(vx) / sizeof(vx[0])); n++) {
                const int row = (64 * n + lane) / PIECES, piece = (64 * n + lane) % PIECES;
                u32x4 x = vx[n];
                if (ok != 0xffffffffu && !(ok >> row & 1)) x = u32x4{0, 0, 0, 0};
                *(u32x4 *)(my_v + row * S::STRIDE + 16 * piece) = x;
            }
            lds_fence_wave();
            // scores: x[n][u][i] belongs to row `col` and key 32 step + 16 u + 4 g + i
            f32x4 x[NT][2];
#pragma unroll
            for (int u = 0; u < 2; u++) {
#pragma unroll
                for (int n = 0; n < NT; n++) x[n][u] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < KC; c++) {
                    bf16x8 kf;
                    if constexpr (F8) kf = bf16_of_e4m3(kx[u][c][0], kx[u][c][1]);
                    else kf = __builtin_bit_cast(bf16x8, u32x4{kx[u][c][0], kx[u][c][1], kx[u][c][2], kx[u][c][3]});
                    if (a.head_dim < KC * 32) {                // elements past the head's end: zero against zero
                        const int d = F8 && c < (KC & ~1) ? 64 * (c / 2) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
                        if (d >= (int)a.head_dim) kf = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
                    }
#pragma unroll
                    for (int n = 0; n < NT; n++) x[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[n][c], x[n][u], 0, 0, 0);
                }
            }
            const int32_t key0 = 32 * step;
            const bool whole = ok == 0xffffffffu && key0 >= kr.full_lo && key0 + 32 <= kr.full_hi;
            const uint32_t ok_now = ok;
            page = page_next;
            ok = ok_next;
            if (step + FEW_WAVES < step_b) fetch(step + FEW_WAVES, page);
            pages_of(step + 2 * FEW_WAVES, page_next, ok_next);

            bf16x8 p[NT];
#pragma unroll
            for (int n = 0; n < NT; n++) {
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int i = 0; i < 4; i++) x[n][u][i] *= to_log2;
                if (a.cap > 0.f)
                    for (int u = 0; u < 2; u++)
                        for (int i = 0; i < 4; i++) x[n][u][i] = capped(x[n][u][i], a.cap);
                if (a.slopes)
                    for (int u = 0; u < 2; u++)
                        for (int i = 0; i < 4; i++) {
                            const int32_t far = place[n] - (key0 + 16 * u + 4 * g + i);
                            x[n][u][i] -= slope[n] * (float)(far < 0 ? -far : far);
                        }
                if (!whole) {
                    const int32_t below = lo[n] - key0, above = hi[n] - key0;      // bits [below, above)
                    uint32_t bits = ok_now;
                    bits &= above >= 32 ? 0xffffffffu : above <= 0 ? 0u : (1u << above) - 1;
                    bits &= below <= 0 ? 0xffffffffu : below >= 32 ? 0u : ~((1u << below) - 1);
                    for (int u = 0; u < 2; u++)
                        for (int i = 0; i < 4; i++)
                            if (!(bits >> (16 * u + 4 * g + i) & 1)) x[n][u][i] = NONE;
                }
                float top = max_f(max_f(max_f(x[n][0][0], x[n][0][1]), max_f(x[n][0][2], x[n][0][3])),
                                  max_f(max_f(x[n][1][0], x[n][1][1]), max_f(x[n][1][2], x[n][1][3])));
                top = max_xor<32>(max_xor<16>(top));
                const float m_new = max_f(m[n], top);
                const float base = m_new == NONE ? 0.f : m_new;
                const float shrink = exp2_fast(m[n] - base);
                m[n] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const __bf16 w = (__bf16)exp2_fast(x[n][u][i] - base);
                        p[n][4 * u + i] = w;
                        sum += (float)w;
                    }
                l[n] = l[n] * shrink + sum;
#pragma unroll
                for (int d = 0; d < 2 * KC; d++) o[n][d] *= shrink;
            }

            // O^T += V^T P^T
            const bool apart = !whole && tok_b > tok_a;        // rows that see different keys of this step
#pragma unroll
            for (int d = 0; d < 2 * KC; d++) {
                bf16x8 vf;
                if constexpr (F8) {
                    typedef __attribute__((ext_vector_type(2))) int i32x2;
                    const int row = (col / 2 < 4 ? 0 : 12) + 4 * g + col / 2;          // keys 4 g .. and 16 + 4 g ..
                    const auto src = (__attribute__((address_space(3))) i32x2 *)(my_v + row * S::STRIDE + 16 * d + 8 * (col & 1));
                    const i32x2 y = __builtin_amdgcn_ds_read_tr8_b64_v2i32(src);
                    vf = bf16_of_e4m3((uint32_t)y[0], (uint32_t)y[1]);
                } else {
                    const uint8_t *src = my_v + (4 * g + col / 4) * S::STRIDE + 32 * d + 8 * (col % 4);
                    const bf16x4 y0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)src);
                    const bf16x4 y1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(src + 16 * S::STRIDE));
                    vf = bf16x8{y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
                }
                if (apart) {                                   // 0 * v is 0 unless v is NaN or infinite
                    const bf16x8 zero = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
                    const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, zero, f32x4{0, 0, 0, 0}, 0, 0, 0);
                    for (int i = 0; i < 4; i++) poison |= z[i] != 0.f ? 1 : 0;
                }
#pragma unroll
                for (int n = 0; n < NT; n++) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[n], o[n][d], 0, 0, 0);
            }
        }
        if (__any(poison)) {                                   // this wave's keys once more, for all its rows
#pragma unroll
            for (int n = 0; n < NT; n++) {
                const KeyRange own{lo[n], hi[n], 0, 0};
                float y[8 * KC], m_slow = NONE, l_slow = 0.f;
                const int32_t r = row0 + 16 * n + col < row_end ? row0 + 16 * n + col : row0;
                const uint8_t *src = a.q + (sq.q0 + r / (int32_t)a.share) * a.q_tok + (int64_t)(kvh * a.share + (uint32_t)r % a.share) * a.q_head;
                for (int32_t st = step_a + wave; st < step_b; st += FEW_WAVES) {
                    float z[8 * KC], m_step, l_step;
                    attend_slowly<F8, 4, 2 * KC>(a, src, k0, v0, table, st, st + 1, own, place[n], to_log2, slope[n], g, [&](int i) { return 16 * i + 4 * g; }, z,
                                                 m_step, l_step);
                    const float m_new = max_f(m_slow, m_step), base = m_new == NONE ? 0.f : m_new;
                    const float f0 = exp2_fast(m_slow - base), f1 = exp2_fast(m_step - base);
                    for (int i = 0; i < 8 * KC; i++) y[i] = st == step_a + wave ? z[i] : y[i] * f0 + z[i] * f1;
                    l_slow = l_slow * f0 + l_step * f1;
                    m_slow = m_new;
                }
                m[n] = m_slow;
                l[n] = g == 0 ? l_slow : 0.f;                  // the lanes of a row each have the whole sum
#pragma unroll
                for (int d = 0; d < 2 * KC; d++) o[n][d] = f32x4{y[4 * d], y[4 * d + 1], y[4 * d + 2], y[4 * d + 3]};
            }
        }

        // the waves' parts together, sixteen rows at a time
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const float sum = sum_xor<32>(sum_xor<16>(l[n]));
            __syncthreads();
            float *oj = (float *)lds, *mj = oj + FEW_WAVES * 16 * S::O_STRIDE, *lj = mj + FEW_WAVES * 16;
#pragma unroll
            for (int d = 0; d < 2 * KC; d++) *(f32x4 *)(oj + (wave * 16 + col) * S::O_STRIDE + 16 * d + 4 * g) = o[n][d];
            if (g == 0) mj[wave * 16 + col] = m[n], lj[wave * 16 + col] = sum;
            __syncthreads();
            // sixteen threads a row: threadIdx / 16 is the row, and a thread takes four elements of each 64
            const int r = threadIdx.x / 16, e = threadIdx.x % 16;
            float top = NONE;
            for (int w = 0; w < FEW_WAVES; w++) top = max_f(top, mj[w * 16 + r]);
            const float base = top == NONE ? 0.f : top;
            float share[FEW_WAVES], all = 0.f;
            for (int w = 0; w < FEW_WAVES; w++) {
                share[w] = exp2_fast(mj[w * 16 + r] - base);
                all += lj[w * 16 + r] * share[w];
            }
            const int64_t o_row = __shfl(o_at[n], r & 15);     // lane r % 16 of this wave holds row r
            const int64_t part = few_part(a, s, kvh, 16 * n + r) + split;      // of the first tile: the others are not split
            if (row0 + 16 * n + r < row_end) {
                for (int d = 4 * e; d < (int)a.head_dim; d += 64) {
                    f32x4 y{0, 0, 0, 0};
                    for (int w = 0; w < FEW_WAVES; w++) y += *(const f32x4 *)(oj + (w * 16 + r) * S::O_STRIDE + d) * share[w];
                    if (alone) {
                        const float inv = all == 0.f ? 0.f : v_scale / all;
                        bf16x4 z;
                        for (int i = 0; i < 4; i++) z[i] = (__bf16)(all == 0.f ? 0.f : y[i] * inv);
                        *(bf16x4 *)(a.out + o_row + 2 * d) = z;
                    } else {
                        for (int i = 0; i < 4; i++) y[i] *= v_scale;
                        *(f32x4 *)(a.part + part * a.head_dim + d) = y;
                    }
                }
                if (!alone && e == 0) {
                    float *ml = a.part_ml + part * 2;
                    ml[0] = top;
                    ml[1] = all;
                }
            }
        }
        __syncthreads();                                       // LDS is free for another tile of rows
    }
}

template <int KC, bool F8>
int launch_few_rows_kc(const AttendArgs &a, uint32_t tiles, hipStream_t s)
{
    const uint64_t grid = (uint64_t)a.b.n_seqs * a.kv_heads * a.few_splits;
    if (tiles == 1) hipLaunchKernelGGL((ecfa_attend_few_kernel<KC, F8, 1>), dim3((unsigned)grid), dim3(FEW_WAVES * 64), 0, s, a);
    else hipLaunchKernelGGL((ecfa_attend_few_kernel<KC, F8, 2>), dim3((unsigned)grid), dim3(FEW_WAVES * 64), 0, s, a);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

template <bool F8>
int launch_few_rows(const AttendArgs &a, uint32_t kc, uint32_t tiles, hipStream_t s)
{
    switch (kc) {
    case 2: return launch_few_rows_kc<2, F8>(a, tiles, s);
    case 3: return launch_few_rows_kc<3, F8>(a, tiles, s);
    case 4: return launch_few_rows_kc<4, F8>(a, tiles, s);
    case 6: return launch_few_rows_kc<6, F8>(a, tiles, s);
    default: return launch_few_rows_kc<8, F8>(a, tiles, s);
    }
}

} // namespace ecfa
