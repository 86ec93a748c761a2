// Attention for sequences with few rows (a decode step: the heads of one token that share their keys): bound by reading K and V once.
//
// A workgroup takes one item (a sequence and a piece of its keys, see few_plan) of one key/value head and the rows of it, 16 NT at a
// time; its four waves take every fourth step of 32 KU keys each and do not meet until the end, where their (m, l, O) are joined in
// LDS.  K goes from memory straight into the registers that the matrix cores read it from (lane l: key l % 16, eight elements of
// the head); V goes from memory into a piece of LDS that belongs to the wave, without touching registers, and is turned when it is read from there.  A step
// is as many keys as make 16 KB of K and V of a wave with 16 rows, so that the eight waves of a compute unit have 128 KB on their
// way: the next step's are fetched as soon as the present one's scores are made.  Two sub-tiles (NT = 2) do not fit the registers: heads of 65 to 128 in BF16 spill 55 of
// them to memory (11 up to 96), 26 in E4M3, and of more than 192 133 and 74.  Heads of more than 128 have one workgroup on a compute unit.  The 16-byte pieces of a row of V are permuted by
// the row's number so that the transposing reads (4 rows and 32 bytes, or 8 rows and 16 bytes, for 16 lanes) do not meet in a bank.
//
// Measured, with the kernel that joins the pieces: one token of 131072 keys with 8 key/value heads of 128 in 109 us (537 MB, 4.9 TB/s, of 6.95 that reads
// reach; 102 where the pool is ordered by head, so that a head's tokens lie together), 4096 keys 13.4 us; 64 tokens of up to 8192 keys in E4M3 49 us (116 MB of keys and
// values).  32768 keys of heads of 128, 160, 192 and 256: 36, 55, 56 and 70 us (160 runs as 192).
#pragma once
#include "ecfa_attend.h"

namespace ecfa {

template <int KC, bool F8, int NT>
struct FewShape {
    static constexpr int E = F8 ? 1 : 2;
    static constexpr int USED = KC * 32 * E, ROW = USED <= 64 ? 64 : USED <= 128 ? 128 : USED <= 256 ? 256 : 512;   // bytes of a key's row
    static constexpr int KU = NT > 1 ? 1 : USED <= 64 ? 4 : USED <= 128 ? 2 : 1;                                  // times 32 keys are a step
    static constexpr int KEYS = 32 * KU;
    static constexpr int V_BYTES = KEYS * ROW;                       // of a wave, twice
    static constexpr int O_STRIDE = KC * 32 + 4;                     // floats
    static constexpr int JOIN_BYTES = FEW_WAVES * 16 * (O_STRIDE + 2) * 4;
    static constexpr int MAIN_BYTES = FEW_WAVES * 2 * V_BYTES;
    static constexpr int BYTES = MAIN_BYTES > JOIN_BYTES ? MAIN_BYTES : JOIN_BYTES;
    __device__ static int spread(int r)                              // piece p of row r stands at p ^ spread(r)
    {
        if constexpr (F8) return ROW == 64 ? r >> 4 & 1 : ROW == 128 ? (r >> 1 & 1) | (r >> 4 & 1) << 1 : (r & 3) | (r >> 4 & 1) << 2;
        else return ROW == 64 ? 0 : ROW == 128 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
    }
};

// The work of workgroup `block`, with S::BYTES of LDS.
template <int KC, bool F8, int NT>
__device__ __forceinline__ void attend_few(const AttendArgs &a, uint32_t block, uint8_t *lds)
{
    using S = FewShape<KC, F8, NT>;
    typedef __attribute__((address_space(3))) uint8_t lds_u8;
    typedef __attribute__((address_space(1))) const uint8_t hbm_u8;
    constexpr int E = S::E, KU = S::KU, ENTRIES = (KU + 1) / 2;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t kvh = (uint32_t)over((int32_t)block, a.by_items), item = block - kvh * a.few_items;
    const FewItem it = few_plan(a, item);
    if (!it.there) return;
    const uint32_t s = it.s;
    const Seq sq = seq_of(a.b, s);
    const int32_t prefix = prefix_of(a, s, sq), share = (int32_t)a.share;
    const int32_t rows = sq.qn * share;
    const uint8_t *k0 = a.c.k + (int64_t)kvh * a.c.k_head, *v0 = a.c.v + (int64_t)kvh * a.c.v_head;
    const int32_t *table = a.b.table + (int64_t)s * a.b.table_stride;
    const uint32_t in_page = (1u << a.c.page_shift) - 1;
    const float k_scale = a.c.k_scale ? a.c.k_scale[kvh] : 1.f, v_scale = a.c.v_scale ? a.c.v_scale[kvh] : 1.f;
    const float to_log2 = factor_of(a, k_scale);
    const int lds0 = (int)(uint32_t)(uintptr_t)(lds_u8 *)lds + wave * 2 * S::V_BYTES;     // this wave's
    const bool extra = a.cap > 0.f || a.slopes;
    const float cap_in = to_log2 * 2.f * a.cap_inv;

    // max_q is a hint: if a sequence has more rows than a tile after all, the tiles follow one another
    for (int32_t row0 = 0; row0 < rows; row0 += 16 * NT) {
        if (row0 > 0 && it.split > 0) break;                   // later tiles are not split
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                         // what follows from it is worked out here, and not kept for all tiles
        const int g = lane / 16, col = lane % 16;
        const int32_t row_end = row0 + 16 * NT < rows ? row0 + 16 * NT : rows;
        const int32_t tok_a = over(row0, a.by_share), tok_b = over(row_end - 1, a.by_share);
        const KeyRange kr = keys_of(a, sq, prefix, tok_a, tok_b);
        const bool alone = row0 > 0 || it.used <= 1;
        const int32_t first = kr.lo / 32, last = kr.hi > kr.lo ? (kr.hi + 31) / 32 : first;
        const int32_t step_a = row0 > 0 ? first : first + it.split * it.per;
        const int32_t step_b = row0 > 0 || step_a + it.per > last ? last : step_a + it.per;

        // this lane's rows, one of each sub-tile
        int64_t o_at[NT];
        int32_t lo[NT], hi[NT], place[NT];
        float slope[NT];
        bf16x8 q[NT][KC];
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const int32_t r = row0 + 16 * n + col;
            const bool there = r < row_end;
            const int32_t tok = there ? over(r, a.by_share) : tok_a;
            const uint32_t head = kvh * a.share + (there ? (uint32_t)(r - tok * share) : 0u);
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

        // The page of key 32 * step + 64 * n + lane as the table has it, looked at a step later.
        uint32_t entry[ENTRIES];
        const auto entries_of = [&](int32_t step) {
#pragma unroll
            for (int n = 0; n < ENTRIES; n++) {
                const int32_t key = 32 * step + 64 * n + (KU == 1 ? lane & 31 : lane);
                entry[n] = step < step_b && key < sq.len ? (uint32_t)table[(uint32_t)key >> a.c.page_shift] : 0xffffffffu;
            }
        };
        uint64_t ok[ENTRIES];                                  // which keys of a step any row may look at
        bool all_ok;
        const auto look = [&](int32_t step) {
            all_ok = true;
#pragma unroll
            for (int n = 0; n < ENTRIES; n++) {
                const int32_t key = 32 * step + 64 * n + (KU == 1 ? lane & 31 : lane);
                ok[n] = __ballot(entry[n] < a.c.n_pages && key >= kr.lo && key < kr.hi && key < 32 * step_b);
                all_ok = all_ok && ok[n] == ~0ull;
            }
        };
        uint32_t kx[2 * KU][KC][F8 ? 2 : 4];
        // 16 keys of K into registers: the c-th 64 bytes of a row, or the last 32 of an odd number of them, a lane 16 or 8 of them (past
        // the head's end its start again)
        const auto fetch_k = [&](int u, auto load16, auto load8) {
#pragma unroll
            for (int c = 0; c < KC; c++) {
                if constexpr (F8) {
                    if (c + 1 < KC && c % 2 == 0) {
                        const u32x4 x = load16(c / 2);
                        kx[u][c][0] = x[0], kx[u][c][1] = x[1], kx[u][c + 1][0] = x[2], kx[u][c + 1][1] = x[3];
                    } else if (c % 2 == 0) {
                        const u32x2 x = load8(c);
                        kx[u][c][0] = x[0], kx[u][c][1] = x[1];
                    }
                } else {
                    const u32x4 x = load16(c);
                    for (int i = 0; i < 4; i++) kx[u][c][i] = x[i];
                }
            }
        };
        constexpr int PIECES = S::ROW / 16, PER = 64 / PIECES, LOADS = PER >= 16 ? 1 : 16 / PER;      // of 16 keys of V
        const int load_row = lane / PIECES, load_piece = lane % PIECES;
        const auto v_piece = [&](int u, int n) {                                                     // where rows PER n .. of the u-th 16 keys find theirs
            const int off = 16 * (load_piece ^ S::spread((16 * u + PER * n + load_row) & 31));
            return off < (int)a.head_dim * E ? off : 0;
        };
        const auto to_lds = [&](int u, int n, const uint8_t *src, int buffer) {
            const int dst = lds0 + buffer * S::V_BYTES + (16 * u + PER * n) * S::ROW;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)src, (lds_u8 *)(uintptr_t)(uint32_t)dst, 16, 0, 0);
        };
        const bool near = a.c.page_shift >= 4 && a.c.near;     // sixteen keys lie in one page, and 32 bits reach over them
        uint32_t k_lane[F8 ? (KC + 1) / 2 : KC], v_lane[2][LOADS];
#pragma unroll
        for (int c = 0; c < (int)(sizeof(k_lane) / 4); c++) {
            const bool narrow = F8 && 2 * c + 1 == KC;         // the last piece of an odd number, in E4M3: eight bytes
            const int off = 64 * c + (narrow ? 8 * g : 16 * g);
            k_lane[c] = (uint32_t)col * (uint32_t)a.c.k_tok + (off < (int)a.head_dim * E ? off : 0);
        }
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int n = 0; n < LOADS; n++) v_lane[u][n] = (uint32_t)(PER * n + load_row) * (uint32_t)a.c.v_tok + (uint32_t)v_piece(u, n);
        const auto fetch = [&](int32_t step, int buffer) {
            if (near) {
                const uint8_t *vs[2 * KU];
#pragma unroll
                for (int u = 0; u < 2 * KU; u++) {
                    const uint32_t e = (uint32_t)__builtin_amdgcn_readlane((int)entry[u / 4], 16 * u % 64);
                    const uint64_t pg = e < a.c.n_pages ? e : 0u, in = (uint32_t)(32 * step + 16 * u) & in_page;
                    const uint8_t *ks = k0 + pg * (uint64_t)a.c.k_page + in * (uint32_t)a.c.k_tok;
                    vs[u] = v0 + pg * (uint64_t)a.c.v_page + in * (uint32_t)a.c.v_tok;
                    fetch_k(u, [&](int c) { return *(const u32x4 *)(ks + k_lane[c]); }, [&](int) { return *(const u32x2 *)(ks + k_lane[sizeof(k_lane) / 4 - 1]); });
                }
#pragma unroll
                for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                    for (int n = 0; n < LOADS; n++) to_lds(u, n, vs[u] + v_lane[u & 1][n], buffer);
            } else {
#pragma unroll
                for (int u = 0; u < 2 * KU; u++) {
                    const int en = (int)entry[u / 4];
                    const uint32_t e = (uint32_t)__shfl(en, (16 * u + col) % 64);
                    const int64_t pg = e < a.c.n_pages ? e : 0u, in = (uint32_t)(32 * step + 16 * u + col) & in_page;
                    const uint8_t *ks = k0 + pg * a.c.k_page + in * a.c.k_tok;
                    const auto at16 = [&](int c) { return *(const u32x4 *)(ks + (64 * c + 16 * g < (int)a.head_dim * E ? 64 * c + 16 * g : 0)); };
                    const auto at8 = [&](int c) { return *(const u32x2 *)(ks + (32 * c + 8 * g < (int)a.head_dim ? 32 * c + 8 * g : 0)); };
                    fetch_k(u, at16, at8);
#pragma unroll
                    for (int n = 0; n < LOADS; n++) {
                        const int row = 16 * u + PER * n + load_row;
                        const uint32_t f = (uint32_t)__shfl(en, row % 64);
                        const int64_t pv = f < a.c.n_pages ? f : 0u, iv = (uint32_t)(32 * step + row) & in_page;
                        to_lds(u, n, v0 + pv * a.c.v_page + iv * a.c.v_tok + v_piece(u, n), buffer);
                    }
                }
            }
        };

        constexpr int STRIDE = FEW_WAVES * KU;
        int32_t step = step_a + (wave - FEW_WAVES) * KU;       // the first turn only fetches: the code for it is there once
        int buffer = 1;
        bool begun = false;
        entries_of(step + STRIDE);
        all_ok = false;
#pragma unroll
        for (int n = 0; n < ENTRIES; n++) ok[n] = 0;
        while (step < step_b) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // K, V and the next step's pages are here, the last reads of V done
            // scores: x[n][u][i] belongs to row `col` and key 32 step + 16 u + 4 g + i
            f32x4 x[NT][2 * KU];
            if (begun) {
                const auto scores = [&](auto ends) {           // `ends`: the head ends before the kernel's pieces do; zeros past its end
#pragma unroll
                    for (int u = 0; u < 2 * KU; u++) {
#pragma unroll
                        for (int n = 0; n < NT; n++) x[n][u] = f32x4{0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < KC; c++) {
                            bf16x8 kf;
                            if constexpr (F8) kf = bf16_of_e4m3(kx[u][c][0], kx[u][c][1]);
                            else kf = __builtin_bit_cast(bf16x8, u32x4{kx[u][c][0], kx[u][c][1], kx[u][c][2], kx[u][c][3]});
                            const int d = F8 && c < (KC & ~1) ? 64 * (c / 2) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
                            if (ends.value && d >= (int)a.head_dim) kf = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
#pragma unroll
                            for (int n = 0; n < NT; n++) x[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[n][c], x[n][u], 0, 0, 0);
                        }
                    }
                };
                if (a.head_dim == KC * 32) scores(std::false_type());
                else scores(std::true_type());
            }
            const int32_t key0 = 32 * step;
            const bool whole = all_ok && key0 >= kr.full_lo && key0 + S::KEYS <= kr.full_hi;
            uint64_t ok_now[ENTRIES];
#pragma unroll
            for (int n = 0; n < ENTRIES; n++) ok_now[n] = ok[n];
            look(step + STRIDE);
            if (step + STRIDE < step_b) fetch(step + STRIDE, buffer ^ 1);
            entries_of(step + 2 * STRIDE);

            if (begun) {
                u32x4 p[NT][KU];
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    float c_log2 = to_log2;
                    if (extra) {
                        c_log2 = 1.f;
#pragma unroll
                        for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                            for (int i = 0; i < 4; i++) x[n][u][i] = capped_or_scaled(a, x[n][u][i], to_log2, cap_in);
                        if (a.slopes)
#pragma unroll
                            for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                                for (int i = 0; i < 4; i++) x[n][u][i] = less_distance(x[n][u][i], slope[n], place[n] - (key0 + 16 * u + 4 * g + i));
                    }
                    if (!whole) {
                        const int32_t below = lo[n] - key0, above = hi[n] - key0;      // keys [below, above) of the step
#pragma unroll
                        for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const int key = 16 * u + 4 * g + i;
                                if (key < below || key >= above || !(ok_now[u / 4] >> (key & 63) & 1)) x[n][u][i] = NONE;
                            }
                    }
                    float top = NONE;
#pragma unroll
                    for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                        for (int i = 0; i < 4; i++) top = max_f(top, x[n][u][i]);
                    top = max_xor<32>(max_xor<16>(top)) * c_log2;
                    // The maximum follows only where a score has outgrown it by 2^8: weights up to there lose nothing in BF16 or in the sums
                    if (__any(top > m[n] + 8.f)) {
                        const float m_new = max_f(m[n], top);
                        const float shrink = exp2_fast(m[n] - (m_new == NONE ? 0.f : m_new));
                        m[n] = m_new;
                        l[n] *= shrink;
#pragma unroll
                        for (int d = 0; d < 2 * KC; d++) o[n][d] *= shrink;
                    }
                    const float base = m[n] == NONE ? 0.f : m[n];
                    const bf16x2 ones{(__bf16)1.f, (__bf16)1.f};
#pragma unroll
                    for (int u = 0; u < 2 * KU; u++)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const bf16x2 w = bf16_pair(exp2_fast(__builtin_fmaf(x[n][u][i], c_log2, -base)), exp2_fast(__builtin_fmaf(x[n][u][i + 1], c_log2, -base)));
                            p[n][u / 2][u % 2 * 2 + i / 2] = __builtin_bit_cast(uint32_t, w);
                            l[n] = __builtin_amdgcn_fdot2_f32_bf16(w, ones, l[n], false);
                        }
                }

                // O^T += V^T P^T, 32 keys at a time
                const int vt = lds0 + buffer * S::V_BYTES;
                // Fragments d0 .. of the k-th 32 keys: sixteen elements of the head each
                constexpr int D = KC == 3 || KC == 6 ? 3 : 4;
                const auto v_frags = [&](auto k, int d0, bf16x8 *vf) {
                    int at0[D], at1[D];
                    if constexpr (F8) {
                        const int row = (col / 2 < 4 ? 0 : 12) + 4 * g + col / 2;          // keys 4 g .. and 16 + 4 g ..
#pragma unroll
                        for (int d = 0; d < D; d++) at0[d] = vt + row * S::ROW + 16 * ((d0 + d) ^ S::spread(row)) + 8 * (col & 1);
                        u32x2 y[D];
                        tr8<k.value * 32 * S::ROW>(at0, y);
#pragma unroll
                        for (int d = 0; d < D; d++) vf[d] = bf16_of_e4m3(y[d][0], y[d][1]);
                    } else {
                        const int row = 4 * g + col / 4, piece = 2 * d0 + col % 4 / 2;
#pragma unroll
                        for (int d = 0; d < D; d++) {
                            at0[d] = vt + row * S::ROW + 16 * ((piece + 2 * d) ^ S::spread(row)) + 8 * (col & 1);
                            at1[d] = vt + (row + 16) * S::ROW + 16 * ((piece + 2 * d) ^ S::spread(row + 16)) + 8 * (col & 1);
                        }
                        tr16<k.value * 32 * S::ROW>(at0, at1, vf);
                    }
                };
                if (!whole) {
                    // what nobody may see, as zeros
#pragma unroll
                    for (int n = 0; n < ENTRIES; n++) {
                        const int row = 64 * n + lane;
                        if (row < S::KEYS && !(ok_now[n] >> lane & 1))
#pragma unroll 1
                            for (int i = 0; i < S::ROW; i += 16) *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)(uint32_t)(vt + row * S::ROW + i) = u32x4{0, 0, 0, 0};
                    }
                    lds_fence_wave();
                    if (tok_b > tok_a) {                       // rows that see different keys: 0 * v is 0 unless v is NaN or infinite
                        const bf16x8 zero = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
                        times<KU>([&](auto k) {
#pragma unroll 1
                            for (int d0 = 0; d0 < 2 * KC; d0 += D) {
                                bf16x8 vf[D];
                                v_frags(k, d0, vf);
#pragma unroll
                                for (int d = 0; d < D; d++) {
                                    const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], zero, f32x4{0, 0, 0, 0}, 0, 0, 0);
                                    const int e = 16 * (d0 + d) + 4 * g;                  // elements past the head's end are not its own
                                    for (int i = 0; i < 4; i++) poison |= z[i] != 0.f && e < (int)a.head_dim ? 1 : 0;
                                }
                            }
                        });
                    }
                }
                times<KU>([&](auto k) {
#pragma unroll
                    for (int d0 = 0; d0 < 2 * KC; d0 += D) {
                        bf16x8 vf[D];
                        v_frags(k, d0, vf);
#pragma unroll
                        for (int d = 0; d < D; d++)
#pragma unroll
                            for (int n = 0; n < NT; n++)
                                o[n][d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], __builtin_bit_cast(bf16x8, p[n][k.value]), o[n][d0 + d], 0, 0, 0);
                    }
                });
            }
            begun = true;
            buffer ^= 1;
            step += STRIDE;
        }
        if (__any(poison)) {                                   // this wave's keys once more, for all its rows
#pragma unroll
            for (int n = 0; n < NT; n++) {
                const KeyRange own{lo[n], hi[n], 0, 0};
                const int32_t r = row0 + 16 * n + col < row_end ? row0 + 16 * n + col : row0;
                const uint8_t *src = a.q + (sq.q0 + r / share) * a.q_tok + (int64_t)(kvh * a.share + (uint32_t)(r % share)) * a.q_head;
                float y[8 * KC];
                attend_slowly<F8, 4, 2 * KC>(a, src, k0, v0, table, step_a + wave * KU, step_b, KU, STRIDE, own, place[n], to_log2, slope[n], g,
                                             [&](int i) { return 16 * i + 4 * g; }, y, m[n], l[n]);
                l[n] = g == 0 ? l[n] : 0.f;                    // the lanes of a row each have the whole sum
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
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));                          // (nor this before the end)
            const int r = tid / 16, e = tid % 16;
            float top = NONE;
            for (int w = 0; w < FEW_WAVES; w++) top = max_f(top, mj[w * 16 + r]);
            const float base = top == NONE ? 0.f : top;
            float part_of[FEW_WAVES], all = 0.f;
            for (int w = 0; w < FEW_WAVES; w++) {
                part_of[w] = exp2_fast(mj[w * 16 + r] - base);
                all += lj[w * 16 + r] * part_of[w];
            }
            const int64_t o_row = __shfl(o_at[n], r & 15);     // lane r % 16 of this wave holds row r
            if (row0 + 16 * n + r < row_end) {
                const int64_t part = few_part(a, item, kvh, 16 * n + r);
                for (int d = 4 * e; d < (int)a.head_dim; d += 64) {
                    f32x4 y{0, 0, 0, 0};
                    for (int w = 0; w < FEW_WAVES; w++) y += *(const f32x4 *)(oj + (w * 16 + r) * S::O_STRIDE + d) * part_of[w];
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
                    a.part_ml[2 * part] = top;
                    a.part_ml[2 * part + 1] = all;
                }
            }
        }
        __syncthreads();                                       // LDS is free for another tile of rows
    }
}

template <int KC, bool F8, int NT>
__global__ __launch_bounds__(FEW_WAVES * 64, KC <= 4 ? 2 : 1) void ecfa_attend_few_kernel(const AttendArgs a)
{
    __shared__ __align__(16) uint8_t lds[FewShape<KC, F8, NT>::BYTES];
    attend_few<KC, F8, NT>(a, blockIdx.x, lds);
}

} // namespace ecfa
