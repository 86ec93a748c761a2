// Products of many rows, and of experts with the rows that were sent to them: Y = X W^T of E4M3 with block scales (ecfm.h).
#include "ecfm_device.h"

namespace ecfm {
namespace {

constexpr uint32_t FEW_WAVES = 8;
constexpr uint64_t MAX_TILES = (1u << 23) - 8;      // of a launch: its threads are counted in 32 bits, 512 a tile

// Few rows: what counts is that W streams from HBM.  A workgroup has 16 NT rows of W and 16 MT rows of X; its eight waves take every
// eighth block of 128 columns, straight from memory into the matrix cores' operands (a row of W is read by nobody else), and add
// up through LDS, in the order of the waves.  Columns are split within a workgroup, so that nothing has to be joined elsewhere.  16 x 14336 x 4096: 12.2 us,
// 4.9 TB/s of W, with the start of the waves and the sum at the end; W alone would take 8.5.
template <int NT, int MT, int U>
__global__ __launch_bounds__(64 * FEW_WAVES) void ecfm_few_kernel(const ProductArgs a)
{
    __shared__ f32x4 part[FEW_WAVES][NT * MT][64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t n0 = blockIdx.x % a.n_tiles * (16 * NT);
    Rows r;
    if (!Tiles<16 * MT>(a).find(a, blockIdx.x / a.n_tiles, &r)) return;
    const uint8_t *wp[NT], *xp[MT];
    const float *ws[NT], *xs[MT];
    for (int i = 0; i < NT; i++) {
        const uint32_t n = n0 + 16 * i + c;
        wp[i] = a.w + (int64_t)r.e * a.w_expert + (int64_t)(n < a.n ? n : a.n - 1) * a.w_row;
        const uint32_t nb = (n0 + 16 * i < a.n ? n0 + 16 * i : a.n - 1) / 128;
        ws[i] = a.w_scale ? a.w_scale + ((uint64_t)r.e * a.n_blocks + nb) * a.k_blocks : nullptr;
    }
    bool there[MT];
    for (int j = 0; j < MT; j++) {
        const uint32_t p = r.m0 + 16 * j + c < r.m1 ? r.m0 + 16 * j + c : r.m1 - 1;
        uint32_t x = a.rows ? (uint32_t)a.rows[p] : p;
        there[j] = x < a.x_rows;
        x = there[j] ? x : 0;
        xp[j] = a.x + (int64_t)x * a.x_row;
        xs[j] = a.x_scale + (uint64_t)x * a.x_per;
    }
    f32x4 sum[NT][MT] = {};
    for (uint32_t first = wave; first < a.k_blocks; first += U * FEW_WAVES) {
        Piece w[U][NT], x[U][MT];
        float sw[U][NT], sx[U][MT];
        // blocks behind the last one: the last one again, with scales of 0, both, since infinity times 0 is none (its own product is part of the sum, so a
        // NaN is in it anyway)
        for (int u = 0; u < U; u++) {
            const uint32_t b = first + u * FEW_WAVES, at = b < a.k_blocks ? b : a.k_blocks - 1;
            // in the last block some of the 128 columns may be missing: those of X count as zeros, in those of W's place stands the row's beginning
            const uint32_t near = at * 128 + 16 * g < a.k ? at * 128 + 16 * g : 0, far = at * 128 + 64 + 16 * g < a.k ? at * 128 + 64 + 16 * g : 0;
            for (int i = 0; i < NT; i++) {
                w[u][i].h[0] = *(const u32x4 *)(wp[i] + near);
                w[u][i].h[1] = *(const u32x4 *)(wp[i] + far);
                sw[u][i] = b < a.k_blocks ? (ws[i] ? ws[i][at] : 1.f) : 0.f;
            }
            for (int j = 0; j < MT; j++) {
                x[u][j].h[0] = *(const u32x4 *)(xp[j] + near);
                x[u][j].h[1] = *(const u32x4 *)(xp[j] + far);
                if (at * 128 + 16 * g >= a.k) x[u][j].h[0] = u32x4{0, 0, 0, 0};
                if (at * 128 + 64 + 16 * g >= a.k) x[u][j].h[1] = u32x4{0, 0, 0, 0};
                sx[u][j] = b >= a.k_blocks ? 0.f : a.x_per ? xs[j][a.x_per > 1 ? at : 0] : 1.f;
            }
        }
        for (int u = 0; u < U; u++)
            for (int i = 0; i < NT; i++)
                for (int j = 0; j < MT; j++) {
                    const f32x4 d = product(w[u][i], x[u][j]);
                    const float s = sw[u][i] * sx[u][j];
                    for (int q = 0; q < 4; q++) sum[i][j][q] = fmaf(d[q], s, sum[i][j][q]);
                }
    }
    for (int i = 0; i < NT; i++)
        for (int j = 0; j < MT; j++) part[wave][i * MT + j][lane] = sum[i][j];
    __syncthreads();
    for (uint32_t o = wave; o < NT * MT; o += FEW_WAVES) {
        const uint32_t i = o / MT, j = o % MT, m = r.m0 + 16 * j + c;
        if (m >= r.m1) continue;
        f32x4 v = part[0][o][lane];
        for (uint32_t p = 1; p < FEW_WAVES; p++) v += part[p][o][lane];
        uint32_t x = a.rows ? (uint32_t)a.rows[m] : m;
        const bool ok = x < a.x_rows;
        store_y(a, m, n0 + 16 * i + 4 * g, ok ? v : f32x4{0, 0, 0, 0});
    }
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) const float lds_f32;
typedef __attribute__((address_space(1))) const uint8_t hbm_u8;

__device__ const float one = 1.f;
__device__ const u32x4 zeros[1] = {};

// Many rows: what counts is that the matrix cores are fed.  A workgroup of eight waves has tiles of BN rows of W by BM of X, one after the other; block after
// block of 128 columns goes through a ring of STAGES buffers in LDS, loaded there without registers while an earlier one is multiplied, across
// the tiles' borders too.  A row's 16-byte pieces are stored by exclusive or with its number modulo 8, so that the sixteen rows of an operand
// are read from unlike banks.  Scales come by eight blocks of a row: block by block they would be as many requests to memory as the operands are
// (8192 x 14336 x 4096: 531 us, 466 so).
// 256 x 256: 2.36 PFLOP/s at 8192 x 14336 x 4096, matrix cores 59 % of the time busy at 1.85 GHz, where the power holds the card (fewer cycles did
// not take less time).  128 x 256, 4096 tokens: 6.7 TB/s beyond the dies' caches, W once for each 128 rows of an expert.  64 x 256, 48 tokens: 6.07 TB/s.
template <uint32_t BM, uint32_t BN, uint32_t WAVES_N, uint32_t STAGES>
__global__ __launch_bounds__(512, 2) void ecfm_many_kernel(const ProductArgs a)
{
    constexpr uint32_t TN = BN / WAVES_N, TM = BM / (8 / WAVES_N), NI = TN / 16, MJ = TM / 16;
    constexpr uint32_t BUFFER = (BN + BM) * 128, X_AT = BN * 128, WL = BN / 64, XL = BM / 64;
    constexpr uint32_t SCALES_AT = STAGES * BUFFER, SCALES = (BM + BN / 128) * 32;
    static_assert((NI - 1) * MJ >= WL + XL && NI % 2 == 0 && STAGES >= 2 && STAGES <= 7 && 128 % TN == 0 && 256 * TN <= BUFFER, "");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * (BUFFER + SCALES)];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t wn = wave % WAVES_N, wm = wave / WAVES_N;

    // Workgroups go to the eight dies in turn.  A die gets a run of tiles that lie together, eight along n by some along m, so that its cache serves
    // rows of W and X to several of them; its workgroups take them in turn.  Of the same expert up to HIGH along m are neighbours: those that read the same W
    // are taken at the same time, and mostly by the same workgroups again (4096 tokens of 256 experts 1790 -> 1750 us, against eight along n first; with
    // tiles of 128 along n 2021 -> 2237, so these go along n first).
    constexpr uint32_t HIGH = BN == 256 ? 4 : 1;
    const Tiles<BM> tiles(a);
    const uint32_t all = tiles.all * a.n_tiles, die = blockIdx.x % 8, share = all / 8 + (die < all % 8), each = gridDim.x / 8;
    const uint32_t run = die * (all / 8) + (die < all % 8 ? die : all % 8);
    const auto locate = [&](uint32_t i, Rows *r, uint32_t *n0) {
        if (i >= share) return false;
        const uint32_t group = (run + i) / (8 * tiles.all), first = group * 8, wide = a.n_tiles - first < 8 ? a.n_tiles - first : 8;
        const uint32_t in = run + i - group * 8 * tiles.all, t = in / wide;
        uint32_t t0, tn;
        if (!tiles.find(a, t, r, &t0, &tn)) return false;
        const uint32_t base = t - (t - t0) % HIGH, high = t0 + tn - base < HIGH ? t0 + tn - base : HIGH, w = in - base * wide, n = w / high, end = r->end;
        *n0 = (first + n) * BN;
        r->m0 = r->m0 + (base + (w - n * high)) * BM - t * BM;
        r->m1 = end - r->m0 < BM ? end : r->m0 + BM;
        return true;
    };
    // Rows of X that this lane loads: lane / 8 + 8 * ... (outside of X: the first); whether those that it multiplies, lane % 16 + 16 * j, are rows of X
    const auto rows_of_tile = [&](const Rows &r, uint32_t *x_row) {
        uint32_t lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                         // what follows from it is worked out here, and not kept for all tiles
        const uint32_t c = lane & 15;
#pragma unroll
        for (uint32_t i = 0; i < XL; i++) {
            const uint32_t m = r.m0 + (wave * XL + i) * 8 + (lane >> 3), p = m < r.m1 ? m : r.m1 - 1, x = a.rows ? (uint32_t)a.rows[p] : p;
            x_row[i] = x < a.x_rows ? x : 0;
        }
        uint32_t there = 0;
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) {
            const uint32_t m = r.m0 + wm * TM + 16 * j + c, p = m < r.m1 ? m : r.m1 - 1, x = a.rows ? (uint32_t)a.rows[p] : p;
            there |= (uint32_t)(x < a.x_rows) << j;
        }
        return there;
    };

    uint32_t turn = blockIdx.x / 8, n0;
    Rows r;
    if (!locate(turn, &r, &n0)) return;

    // What is loaded: block fb of the tile at f_w, piece (lane % 8) ^ (lane / 8) of the rows lane / 8 + 8 * ...: rows of X by their numbers, of W by their
    // distance from the tile's first
    const uint32_t piece = 16 * ((lane & 7) ^ (lane >> 3)), x_stride = (uint32_t)a.x_row, w_stride = (uint32_t)a.w_row;
    const uint8_t *f_w = nullptr;
    uint32_t w_off[WL], x_row[XL], f_e = 0, f_nb = 0, fb = 0, f_slot = SCALES_AT;
    bool f_more = true;                                        // this block has not been loaded yet
    const auto aim = [&](const Rows &t, uint32_t t_n0) {
        uint32_t lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                         // (here too)
        f_e = t.e;
        f_nb = t_n0 / 128;
        f_w = a.w + (int64_t)t.e * a.w_expert + (uint64_t)t_n0 * w_stride;
#pragma unroll
        for (uint32_t i = 0; i < WL; i++) {
            const uint32_t n = (wave * WL + i) * 8 + (lane >> 3), most = a.n - 1 - t_n0;
            w_off[i] = (n < most ? n : most) * w_stride;
        }
    };
    // Scales of blocks fb .. fb + 7, once in eight blocks, into the next slot of their ring.  Where there are none: a one, again and again
    const bool x_scaled = a.x_per != 0, w_scaled = a.w_scale != nullptr;
    const auto fetch_scales = [&] {
        uint32_t lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const uint32_t at = fb + (lane & 7) < a.k_blocks ? fb + (lane & 7) : a.k_blocks - 1;
        uint8_t *dst = lds + f_slot;
        f_slot = f_slot == SCALES_AT + (STAGES - 1) * SCALES ? SCALES_AT : f_slot + SCALES;
#pragma unroll
        for (uint32_t i = 0; i < XL; i++) {
            const float *from = x_scaled ? a.x_scale + ((uint64_t)x_row[i] * a.x_per + (a.x_per > 1 ? at : 0)) : &one;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)from, (lds_u8 *)(dst + (wave * XL + i) * 256), 4, 0, 0);
        }
        if (wave == 0 && lane < BN / 16) {
            const uint32_t n = f_nb + (lane >> 3);
            const float *from = w_scaled ? a.w_scale + (((uint64_t)f_e * a.n_blocks + (n < a.n_blocks ? n : a.n_blocks - 1)) * a.k_blocks + at) : &one;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)from, (lds_u8 *)(dst + BM * 32), 4, 0, 0);
        }
    };
    // The i-th of this wave's loads of block fb.  In a tile's last block some of the 128 columns may be missing: zeros in X, in their place in W the block's
    // first ones
    const auto fetch = [&](uint32_t buffer, uint32_t i) {
        const bool in = fb * 128 + piece < a.k;
        if (i < WL) {
            const uint8_t *from = f_w + (uint64_t)fb * 128 + (w_off[i] + (in ? piece : 0));
            __builtin_amdgcn_global_load_lds((hbm_u8 *)from, (lds_u8 *)(lds + buffer + (wave * WL + i) * 1024), 16, 0, 0);
        } else {
            const uint8_t *from = a.x + (uint64_t)fb * 128 + piece + (uint64_t)x_row[i - WL] * x_stride;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)(in ? from : (const uint8_t *)zeros), (lds_u8 *)(lds + buffer + X_AT + (wave * XL + i - WL) * 1024), 16, 0, 0);
        }
    };
    // To the next block, and behind the last one to the next tile's first; where there is no more, the last one again, where nobody reads it
    const auto advance = [&](bool more, const Rows &next, uint32_t next_n0, const uint32_t *next_row) {
        if (++fb < a.k_blocks) return;
        f_more = f_more && more;
        fb = f_more ? 0 : a.k_blocks - 1;
        if (f_more) {
#pragma unroll
            for (uint32_t i = 0; i < XL; i++) x_row[i] = next_row[i];
            aim(next, next_n0);
        }
    };
    // The block after the one that is multiplied is here for all, and nobody reads that one any more.  Later ones may be on their way, WL + XL loads a wave
    // each: loads into LDS are no loads to a barrier's own wait.
    const auto arrived = [&] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * (WL + XL)) : "memory"); };

    // what is multiplied
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8 *)lds, at0 = c * 128 + ((g ^ (c & 7)) << 4);
    const uint32_t w_at = lds0 + wn * TN * 128 + at0, x_at = lds0 + X_AT + wm * TM * 128 + at0;
    const uint32_t xs_at = lds0 + (wm * TM + c) * 32, ws_at = lds0 + BM * 32 + wn * TN / 128 * 32;
    f32x4 sum[NI][MJ] = {};
    // The sum takes a product's block where the products of the next row of tiles are under way: d and s_d are of the row before, across blocks too
    f32x4 d[MJ] = {};
    float s[MJ] = {}, s_d[MJ], s_x[MJ], s_w;
    Piece x[MJ], w[2];
    uint32_t rb = 0, r_slot = SCALES_AT + (STAGES - 1) * SCALES;
    const auto read = [&](uint32_t at, uint32_t tile) {
        Piece p;
        p.h[0] = *(lds_u32x4 *)(uintptr_t)(at + tile * 2048);
        p.h[1] = *(lds_u32x4 *)(uintptr_t)((at ^ 64) + tile * 2048);
        return p;
    };
    const auto to_scales = [&] {                               // of block rb of the tile that is read
        if (rb % 8 == 0) r_slot = r_slot == SCALES_AT + (STAGES - 1) * SCALES ? SCALES_AT : r_slot + SCALES;
        const uint32_t of_block = r_slot + rb % 8 * 4;
        rb = rb + 1 == a.k_blocks ? 0 : rb + 1;
        return of_block;
    };
    const auto read_scales = [&](uint32_t of_block) {
        s_w = *(lds_f32 *)(uintptr_t)(ws_at + of_block);
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) s_x[j] = *(lds_f32 *)(uintptr_t)(xs_at + j * 512 + of_block);
    };
    const auto read_first = [&](uint32_t buffer) {             // what a block's first products take
        w[0] = read(w_at + buffer, 0);
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) x[j] = read(x_at + buffer, j);
        read_scales(to_scales());
    };

    uint32_t ok = rows_of_tile(r, x_row), here = 0;
    aim(r, n0);
#pragma unroll
    for (uint32_t q = 0; q + 1 < STAGES; q++) {
        if (q) advance(false, r, n0, x_row);
        if (fb % 8 == 0 && f_more) fetch_scales();
#pragma unroll
        for (uint32_t i = 0; i < WL + XL; i++) fetch(q * BUFFER, i);
    }
    arrived();
    read_first(0);
    while (true) {
        Rows next = r;
        uint32_t next_n0 = n0, next_row[XL], next_ok = 0;
        turn += each;
        const bool more = locate(turn, &next, &next_n0);
        if (more) next_ok = rows_of_tile(next, next_row);
        const bool live = BM == 256 || r.m0 + wm * TM < r.m1;  // this wave has rows; if not, it only loads (4096 tokens of experts 1853 -> 1760 us)
        if (!live) {
            for (uint32_t b = 0; b < a.k_blocks; b++) {
                advance(more, next, next_n0, next_row);
                if (fb % 8 == 0 && f_more) fetch_scales();
                const uint32_t free = here ? here - BUFFER : (STAGES - 1) * BUFFER;
#pragma unroll
                for (uint32_t i = 0; i < WL + XL; i++) fetch(free, i);
                arrived();
                here = here + BUFFER == STAGES * BUFFER ? 0 : here + BUFFER;
                if (b + 1 < a.k_blocks) to_scales();
            }
            read_first(here);
        } else {
            for (uint32_t b = 0; b < a.k_blocks; b++) {
                const uint32_t free = here ? here - BUFFER : (STAGES - 1) * BUFFER, there = here + BUFFER == STAGES * BUFFER ? 0 : here + BUFFER;
                advance(more, next, next_n0, next_row);
                if (fb % 8 == 0 && f_more) fetch_scales();
                const uint32_t of_block = to_scales();
#pragma unroll
                for (uint32_t j = 0; j < MJ; j++) s_d[j] = s[j], s[j] = s_w * s_x[j];
                // A row of tiles at a time.  Reads are issued behind a product, never in front of one that has to wait for earlier ones: the wait would be
                // for them too.  Loads are issued a few at a time: all at once would hold the products up until the last of them is taken.  Where the
                // last row's products are left of the block, the barrier: the first reads of the next block then go beside them.
#pragma unroll
                for (uint32_t i = 0; i < NI; i++) {
                    f32x4 now[MJ];
                    if (i == NI - 1) arrived();
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (uint32_t j = 0; j < MJ; j++) {
                        now[j] = product(w[i & 1], x[j]);
                        __builtin_amdgcn_sched_barrier(0);
                        if (i + 1 < NI) {
                            if (j == 0) w[(i + 1) & 1] = read(w_at + here, i + 1);
                            if (i * MJ + j < WL + XL) fetch(free, i * MJ + j);
                        } else {
                            if (j == 0) w[0] = read(w_at + there, 0);
                            x[j] = read(x_at + there, j);
                            if (j == MJ - 1) read_scales(of_block);
                        }
                        f32x4 &to = i ? sum[i - 1][j] : sum[NI - 1][j];
                        const float by = i ? s[j] : s_d[j];
#pragma unroll
                        for (int q = 0; q < 4; q++) to[q] = fmaf(d[j][q], by, to[q]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < MJ; j++) d[j] = now[j];
                }
                here = there;
            }
#pragma unroll
            for (uint32_t j = 0; j < MJ; j++)
#pragma unroll
                for (int q = 0; q < 4; q++) sum[NI - 1][j][q] = fmaf(d[j][q], s[j], sum[NI - 1][j][q]);
            // Y by way of LDS, where the last block was: a piece of 16 rows and TN columns after the other, so that rows are stored 16 bytes a lane and in whole
            // lines.  Straight from the registers a store would have 32 bytes of each of 16 rows (8192 x 14336 x 4096: 432 us, 403 so).
            uint8_t *const out = lds + (here ? here - BUFFER : (STAGES - 1) * BUFFER) + wave * 16 * TN * 2;
            uint32_t lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));                     // what follows from it is worked out here, and not kept for all tiles
            const uint32_t g = lane >> 4, c = lane & 15;
#pragma unroll
            for (uint32_t j = 0; j < MJ; j++) {
                const uint32_t m = r.m0 + wm * TM + 16 * j;
                const bool there = ok >> j & 1;
                if (!a.lines) {
                    if (m + c < r.m1)
#pragma unroll
                        for (uint32_t i = 0; i < NI; i++) store_y(a, m + c, n0 + wn * TN + 16 * i + 4 * g, there ? sum[i][j] : f32x4{0, 0, 0, 0});
                    continue;
                }
#pragma unroll
                for (uint32_t i = 0; i < NI; i++) {
                    const f32x4 v = there ? sum[i][j] : f32x4{0, 0, 0, 0};
                    *(bf16x4 *)(out + c * TN * 2 + (((2 * i + g / 2) ^ (c & (TN / 8 - 1))) << 4) + (g & 1) * 8) = __builtin_convertvector(v, bf16x4);
                }
#pragma unroll
                for (uint32_t q = 0; q < TN / 32; q++) {
                    const uint32_t at = q * 64 + lane, to = at / (TN / 8), n = n0 + wn * TN + at % (TN / 8) * 8;
                    const u32x4 v = *(const u32x4 *)(out + to * TN * 2 + (((at % (TN / 8)) ^ (to & (TN / 8 - 1))) << 4));
                    if (m + to < r.m1 && n < a.n) *(u32x4 *)((__bf16 *)a.y + (int64_t)(m + to) * a.y_row + n) = v;
                }
            }
        }
        if (!more) break;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // before the buffer that Y went through is loaded again
        r = next;
        n0 = next_n0;
        ok = next_ok;
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) {
            s[j] = 0;
            d[j] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (uint32_t i = 0; i < NI; i++) sum[i][j] = f32x4{0, 0, 0, 0};
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // what was loaded behind the last block is here too
}

// The most tiles along m that there can be, and of bm x bn.
uint32_t tiles_of(const ProductArgs &a, uint32_t bm) { return (a.m + bm - 1) / bm + (a.starts ? (a.experts < a.m ? a.experts : a.m) : 0); }
uint64_t tiles_of(const ProductArgs &a, uint32_t bm, uint32_t bn) { return (uint64_t)tiles_of(a, bm) * ((a.n + bn - 1) / bn); }

// Launches a workgroup for each of them, or `most` that take them in turn.
template <class K>
int launch_tiles(K kernel, ProductArgs a, uint32_t threads, uint32_t bm, uint32_t bn, uint32_t most, hipStream_t s)
{
    a.n_tiles = (a.n + bn - 1) / bn;
    a.m_tiles = tiles_of(a, bm);
    const uint64_t tiles = tiles_of(a, bm, bn);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(((tiles < most ? tiles : most) + 7) / 8 * 8)), dim3(threads), 0, s, a);
    return hipGetLastError() == hipSuccess ? ECF8_OK : ECF8_E_HIP;
}

int check(const ecfm_weights *w, const ecfm_x *x, const ecfm_y *y, ProductArgs *a)
{
    if (w->rows == 0 || w->rows > (1u << 24) || w->cols == 0 || w->cols % 16 || w->cols > (1u << 24) || w->experts == 0 || w->experts > 4096) return ECF8_E_ARG;
    if (x->rows > (1u << 28) || y->rows > (1u << 28) || (y->dtype != ECFA_F32 && y->dtype != ECFA_BF16)) return ECF8_E_ARG;
    a->k_blocks = (w->cols + 127) / 128;
    a->n_blocks = (w->rows + 127) / 128;
    if (x->scale_cols && x->scale_cols != 1 && x->scale_cols != a->k_blocks) return ECF8_E_ARG;
    if (!w->d || (y->rows && (!x->d || !y->d || x->rows == 0)) || (x->scale_cols && x->rows && !x->d_scale) || (!x->scale_cols && x->d_scale)) return ECF8_E_ARG;
    const int64_t e = y->dtype == ECFA_F32 ? 4 : 2;
    a->w_row = w->rows > 1 ? w->row_stride : 0;
    a->w_expert = w->experts > 1 ? w->expert_stride : 0;
    a->x_row = x->rows > 1 ? x->row_stride : 0;
    a->y_row = y->rows > 1 ? y->row_stride : 0;
    if (a->w_row < 0 || a->w_row > (1 << 24) || a->x_row < 0 || a->x_row > 0xffffffffll) return ECF8_E_ARG;
    if (((uintptr_t)w->d & 15) || (a->w_row & 15) || (a->w_expert & 15) || ((uintptr_t)x->d & 15) || (a->x_row & 15) || ((uintptr_t)w->d_scale & 3)
        || ((uintptr_t)x->d_scale & 3) || ((uintptr_t)y->d & (e - 1))) return ECF8_E_ALIGN;
    a->w = w->d;
    a->x = x->d;
    a->w_scale = w->d_scale;
    a->x_scale = x->d_scale;
    a->y = y->d;
    a->n = w->rows;
    a->k = w->cols;
    a->m = y->rows;
    a->x_rows = x->rows;
    a->x_per = x->scale_cols;
    a->experts = w->experts;
    a->f32 = y->dtype == ECFA_F32;
    a->wide = a->y_row % 4 == 0 && (uintptr_t)y->d % (4 * e) == 0;
    a->lines = !a->f32 && a->y_row % 8 == 0 && a->n % 8 == 0 && (uintptr_t)y->d % 16 == 0;
    return ECF8_OK;
}

// What a round of workgroups, one to a compute unit, takes: the same for each tile and that for each block of 128 columns, in us, as measured with the card
// full (cols 2048 to 14336).  The kernel is the one whose rounds come out shortest.  What these leave out: the bytes of W, which bound experts with few rows (the
// estimates there are 31 us for 44, 517 for 417, 1531 for 1750; of one token the second best is chosen by 3 %); the stores of Y, which are
// four elements at a time and less where n is not a multiple of eight or Y fp32 (4200 x 4400 x 272 23 us, fp32 33, 4200 x 4401 x 272 61 and 68); and
// that a workgroup goes through all of K, however few tiles there are (the rows of 14336 columns below).
// In us, that kernel and its neighbours, inputs past the caches:
//   16 x 14336 x 4096                  16 x 64 15.1, 16 x 32 17.9, 64 x 128 19.1
//   64 x 4096 x 4096                   32 x 32 12.2, 16 x 64 13.1, 64 x 128 18.6
//   777 x 1001 x 2064                  32 x 64 12.0, 32 x 32 13.7, 64 x 128 14.2
//   200 x 4096 x 4096                  64 x 128 18.3, 128 x 128 21.2, 32 x 64 28.5
//   64 x 4096 x 14336                  34, 128 rows 47, 256 rows 55, 512 rows 58 (bytes: 8.7, 8.9, 9.9, 20 with the products)
//   2048 x 4096 x 4096                 128 x 256 38, 128 x 128 46, 256 x 256 62
//   8192 x 14336 x 4096                256 x 256 411, 128 x 256 479, 128 x 128 601
//   1 token of 8 experts, 4096 x 7168  64 x 128 44.2, 16 x 64 42.8, 64 x 256 53.5
//   48 tokens, 256 of 7168 x 2048      64 x 256 417, 16 x 64 439, 128 x 128 419
//   4096 tokens, 256 of 4096 x 7168    128 x 256 1750, 128 x 128 1975, 256 x 256 2179
struct Shape {
    uint32_t bm, bn;
    float tile, block;
    bool together;                             // several workgroups fit a compute unit: parts of rounds count as parts
    int (*launch)(const ProductArgs &, hipStream_t);
};

template <int NT, int MT, int U>
int few(const ProductArgs &a, hipStream_t s)
{
    return launch_tiles(ecfm_few_kernel<NT, MT, U>, a, 64 * FEW_WAVES, 16 * MT, 16 * NT, MAX_TILES, s);
}

template <uint32_t BM, uint32_t BN, uint32_t WAVES_N, uint32_t STAGES>
int many(const ProductArgs &a, hipStream_t s)
{
    // (a tile that ends before the ring is full once: one to a workgroup)
    return launch_tiles(ecfm_many_kernel<BM, BN, WAVES_N, STAGES>, a, 512, BM, BN, a.k_blocks + 1 < STAGES ? MAX_TILES : 256, s);
}

const Shape SHAPES[] = {
    {16, 16, 2.f, 0.10f, true, few<1, 1, 2>},          {16, 32, 2.f, 0.17f, true, few<2, 1, 2>},
    {16, 64, 2.f, 0.26f, true, few<4, 1, 1>},          {32, 32, 2.f, 0.23f, true, few<2, 2, 1>},
    {32, 64, 2.f, 0.35f, true, few<4, 2, 1>},          {64, 128, 6.f, 0.45f, false, many<64, 128, 2, 6>},
    {64, 256, 6.f, 0.78f, false, many<64, 256, 4, 3>}, {128, 128, 4.f, 0.66f, false, many<128, 128, 2, 4>},
    {128, 256, 5.f, 1.05f, false, many<128, 256, 4, 3>}, {256, 256, 6.f, 1.80f, false, many<256, 256, 2, 2>},
};

int launch(const ProductArgs &a, hipStream_t s)
{
    const Shape *best = nullptr;
    double least = 0;
    for (const Shape &v : SHAPES) {
        if (tiles_of(a, v.bm, v.bn) > MAX_TILES) continue;
        // tiles along m: of experts every last one is half empty, and as far as is known here each has rows
        double tiles = (a.m + v.bm - 1) / v.bm;
        if (a.starts) {
            const double hit = a.experts < a.m ? a.experts : a.m, full = (double)a.m / v.bm + 0.5 * hit;
            tiles = full > hit ? full : hit;
        }
        tiles *= (a.n + v.bn - 1) / v.bn;
        double rounds = tiles <= 256 ? 1 : tiles / 256;
        if (!v.together && (!a.starts || rounds < 4)) rounds = (double)(uint64_t)(rounds + 0.999);
        const double us = rounds * (v.tile + a.k_blocks * v.block);
        if (!best || us < least) {
            best = &v;
            least = us;
        }
    }
    return best ? best->launch(a, s) : ECF8_E_ARG;
}

} // namespace
} // namespace ecfm

using namespace ecfm;

extern "C" {

int ecfm_gemm(const ecfm_weights *weights, const ecfm_x *x, const ecfm_y *y, void *stream)
{
    ProductArgs a{};
    if (!weights || !x || !y || weights->experts != 1 || x->rows != y->rows) return ECF8_E_ARG;
    const int rc = check(weights, x, y, &a);
    if (rc || y->rows == 0) return rc;
    return launch(a, (hipStream_t)stream);
}

int ecfm_gemm_experts(const ecfm_weights *weights, const int32_t *d_starts, const ecfm_x *x, const int32_t *d_rows, const ecfm_y *y, void *stream)
{
    ProductArgs a{};
    if (!weights || !x || !y || (!d_rows && x->rows != y->rows)) return ECF8_E_ARG;
    const int rc = check(weights, x, y, &a);
    if (rc) return rc;
    if (((uintptr_t)d_starts & 3) || ((uintptr_t)d_rows & 3)) return ECF8_E_ALIGN;
    if (y->rows == 0) return ECF8_OK;
    if (!d_starts) return ECF8_E_ARG;
    a.starts = d_starts;
    a.rows = d_rows;
    return launch(a, (hipStream_t)stream);
}

} // extern "C"
