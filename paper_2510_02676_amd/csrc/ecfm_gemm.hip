// Products of many rows, and of experts with the rows that were sent to them: Y = X W^T of E4M3 with block scales (ecfm.h).
#include "ecfm_device.h"

namespace ecfm {
namespace {

constexpr uint32_t FEW_WAVES = 8;
constexpr uint64_t MAX_TILES = (1u << 23) - 8;      // of a launch: its threads are counted in 32 bits, 512 a tile

// Few rows: what counts is that W streams from HBM.  A workgroup has 16 NT rows of W and 16 MT rows of X; its eight waves take every
// eighth block of 128 columns, straight from memory into the matrix cores' operands (a row of W is read by nobody else), and add
// up through LDS, in the order of the waves.
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
        // blocks behind the last one: the last one again, times nothing (its own product is part of the sum, so a NaN is in it anyway)
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
                sx[u][j] = a.x_per > 1 ? xs[j][at] : 1.f;
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
        if (a.x_per == 1 && ok) v *= a.x_scale[x];
        store_y(a, m, n0 + 16 * i + 4 * g, ok ? v : f32x4{0, 0, 0, 0});
    }
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) const float lds_f32;
typedef __attribute__((address_space(1))) const uint8_t hbm_u8;

__device__ const float one = 1.f;
__device__ const u32x4 zeros[1] = {};

// Many rows: what counts is that the matrix cores are fed.  A workgroup of eight waves has 256 rows of W and BM of X, block after block of 128 columns
// in one of two buffers in LDS, loaded there without registers while the other one is multiplied.  A row's 16-byte pieces are stored by
// exclusive or with its number modulo 8, so that the sixteen rows of an operand are read from unlike banks.  Scales come by eight blocks of a row:
// block by block they would be as many requests to memory as the operands are.
template <uint32_t BM, uint32_t BN, uint32_t WAVES_N, uint32_t STAGES>
__global__ __launch_bounds__(512, 2) void ecfm_many_kernel(const ProductArgs a)
{
    constexpr uint32_t TN = BN / WAVES_N, TM = BM / (8 / WAVES_N), NI = TN / 16, MJ = TM / 16;
    constexpr uint32_t BUFFER = (BN + BM) * 128, X_AT = BN * 128, WL = BN / 64, XL = BM / 64;
    constexpr uint32_t SCALES_AT = STAGES * BUFFER, SCALES = (BM + BN / 128) * 32;
    static_assert((NI - 1) * MJ >= WL + XL && STAGES >= 2 && STAGES <= 7 && 128 % TN == 0, "");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[SCALES_AT + 2 * SCALES];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    Rows r;
    uint32_t n0;
    {
        const Tiles<BM> tiles(a);
        // Workgroups go to the eight dies in turn.  A die gets a run of tiles that lie together, eight along n by some along m, so that its cache serves
        // rows of W and X to several of them
        const uint32_t all = tiles.all * a.n_tiles, share = all / 8, more = all % 8, die = blockIdx.x % 8, i = blockIdx.x / 8;
        if (i >= share + (die < more)) return;
        const uint32_t id = die * share + (die < more ? die : more) + i;
        const uint32_t group = id / (8 * tiles.all), first = group * 8, wide = a.n_tiles - first < 8 ? a.n_tiles - first : 8, in = id - group * 8 * tiles.all;
        n0 = (first + in % wide) * BN;
        if (!tiles.find(a, in / wide, &r)) return;
    }
    const uint32_t wn = wave % WAVES_N, wm = wave / WAVES_N;

    // what this lane loads: piece (lane % 8) ^ (lane / 8) of the rows lane / 8 + 8 * ..., and their scale of block lane % 8 of eight
    const uint32_t piece = 16 * ((lane & 7) ^ (lane >> 3));
    const uint8_t *wp[WL], *xp[XL];
    uint32_t x_row[XL];
    for (uint32_t i = 0; i < WL; i++) {
        const uint32_t n = n0 + (wave * WL + i) * 8 + (lane >> 3);
        wp[i] = a.w + (int64_t)r.e * a.w_expert + (int64_t)(n < a.n ? n : a.n - 1) * a.w_row + piece;
    }
    for (uint32_t i = 0; i < XL; i++) {
        const uint32_t m = r.m0 + (wave * XL + i) * 8 + (lane >> 3), p = m < r.m1 ? m : r.m1 - 1, x = a.rows ? (uint32_t)a.rows[p] : p;
        x_row[i] = x < a.x_rows ? x : 0;
        xp[i] = a.x + (int64_t)x_row[i] * a.x_row + piece;
    }
    // The i-th of this wave's loads, of the block that the addresses are at
    const auto fetch = [&](uint32_t buffer, uint32_t i) {
        uint8_t *dst = lds + buffer + (i < WL ? (wave * WL + i) * 1024 : X_AT + (wave * XL + i - WL) * 1024);
        __builtin_amdgcn_global_load_lds((hbm_u8 *)(i < WL ? wp[i] : xp[i - WL]), (lds_u8 *)dst, 16, 0, 0);
    };
    // Addresses to block b.  In the last one some of the 128 columns may be missing: zeros.  Behind it they stay where they are.
    const auto advance = [&](uint32_t b) {
        const uint32_t step = b > 0 && b < a.k_blocks ? 128 : 0;
#pragma unroll
        for (uint32_t i = 0; i < WL; i++) wp[i] += step;
#pragma unroll
        for (uint32_t i = 0; i < XL; i++) xp[i] += step;
        if (b * 128 + 128 > a.k && b * 128 + piece >= a.k) {
#pragma unroll
            for (uint32_t i = 0; i < WL; i++) wp[i] = (const uint8_t *)zeros;
#pragma unroll
            for (uint32_t i = 0; i < XL; i++) xp[i] = (const uint8_t *)zeros;
        }
    };
    // The block after the one that is multiplied is here for all, and nobody reads that one any more.  Later ones may be on their way, WL + XL loads a wave
    // each: loads into LDS are no loads to a barrier's own wait.
    const auto arrived = [&] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * (WL + XL)) : "memory"); };
    // Scales of blocks b .. b + 7 (b a multiple of 8).  Where there are none: a one, again and again
    const bool x_scaled = a.x_per > 1, w_scaled = a.w_scale != nullptr;
    const auto fetch_scales = [&](uint32_t b) {
        const uint32_t at = b + (lane & 7) < a.k_blocks ? b + (lane & 7) : a.k_blocks - 1;
        uint8_t *dst = lds + SCALES_AT + (b & 8 ? SCALES : 0);
#pragma unroll
        for (uint32_t i = 0; i < XL; i++) {
            const float *from = x_scaled ? a.x_scale + ((uint64_t)x_row[i] * a.x_per + at) : &one;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)from, (lds_u8 *)(dst + (wave * XL + i) * 256), 4, 0, 0);
        }
        if (wave == 0 && lane < BN / 16) {
            const uint32_t n = n0 / 128 + (lane >> 3);
            const float *from = w_scaled ? a.w_scale + (((uint64_t)r.e * a.n_blocks + (n < a.n_blocks ? n : a.n_blocks - 1)) * a.k_blocks + at) : &one;
            __builtin_amdgcn_global_load_lds((hbm_u8 *)from, (lds_u8 *)(dst + BM * 32), 4, 0, 0);
        }
    };

    // what this lane multiplies
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8 *)lds, at0 = c * 128 + ((g ^ (c & 7)) << 4);
    const uint32_t xs_at = lds0 + SCALES_AT + (wm * TM + c) * 32, ws_at = lds0 + SCALES_AT + BM * 32 + wn * TN / 128 * 32;
    f32x4 sum[NI][MJ] = {};
    // The sum takes a product's block where the products of the next row of tiles are under way: d and s_d are of the row before, across blocks too
    f32x4 d[MJ] = {};
    float s[MJ] = {}, s_d[MJ], s_x[MJ], s_w;
    Piece x[MJ], w[2];
    const auto read = [&](uint32_t at, uint32_t tile) {
        Piece p;
        p.h[0] = *(lds_u32x4 *)(uintptr_t)(at + tile * 2048);
        p.h[1] = *(lds_u32x4 *)(uintptr_t)((at ^ 64) + tile * 2048);
        return p;
    };
    const auto read_scales = [&](uint32_t b) {
        const uint32_t of_block = (b & 8 ? SCALES : 0) + b % 8 * 4;
        s_w = *(lds_f32 *)(uintptr_t)(ws_at + of_block);
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) s_x[j] = *(lds_f32 *)(uintptr_t)(xs_at + j * 512 + of_block);
    };
    const uint32_t w_at = lds0 + wn * TN * 128 + at0, x_at = lds0 + X_AT + wm * TM * 128 + at0;

    fetch_scales(0);
#pragma unroll
    for (uint32_t b = 0; b + 1 < STAGES; b++) {
        advance(b);
#pragma unroll
        for (uint32_t i = 0; i < WL + XL; i++) fetch(b * BUFFER, i);
    }
    arrived();
    w[0] = read(w_at, 0);
#pragma unroll
    for (uint32_t j = 0; j < MJ; j++) x[j] = read(x_at, j);
    read_scales(0);
    uint32_t here = 0;
    for (uint32_t b = 0; b < a.k_blocks; b++) {
        const uint32_t free = here ? here - BUFFER : (STAGES - 1) * BUFFER, there = here + BUFFER == STAGES * BUFFER ? 0 : here + BUFFER;
        if (b % 8 == 0 && b + 8 < a.k_blocks) fetch_scales(b + 8);
        advance(b + STAGES - 1);
#pragma unroll
        for (uint32_t j = 0; j < MJ; j++) s_d[j] = s[j], s[j] = s_w * s_x[j];
        // A row of tiles at a time.  Reads are issued behind a product, never in front of one that has to wait for earlier ones: the wait would be for
        // them too.  Loads of the next block are issued a few at a time: all at once would hold the products up until the last of them is taken.  Where
        // the last row's products are left of the block, the barrier: the first reads of the next block then go beside them.
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
                    if (j == MJ - 1) read_scales(b + 1);
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
    if (STAGES > 2) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");    // what was loaded behind the last block is here too
#pragma unroll
    for (uint32_t j = 0; j < MJ; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) sum[NI - 1][j][q] = fmaf(d[j][q], s[j], sum[NI - 1][j][q]);
    // Y by way of LDS, a piece of 16 rows and TN columns after the other, so that rows are stored 16 bytes a lane and in whole lines: straight from the
    // registers a store would have 32 bytes of each of 16 rows.  (Nobody reads the buffers any more but for what nobody uses.)
    uint8_t *const out = lds + wave * 16 * TN * 2;
#pragma unroll
    for (uint32_t j = 0; j < MJ; j++) {
        const uint32_t m = r.m0 + wm * TM + 16 * j, mine = m + c < r.m1 ? m + c : r.m1 - 1, row = a.rows ? (uint32_t)a.rows[mine] : mine;
        const bool there = row < a.x_rows;
        const float last = a.x_per == 1 && there ? a.x_scale[row] : 1.f;
        if (!a.lines) {
            if (m + c < r.m1)
#pragma unroll
                for (uint32_t i = 0; i < NI; i++) store_y(a, m + c, n0 + wn * TN + 16 * i + 4 * g, there ? sum[i][j] * last : f32x4{0, 0, 0, 0});
            continue;
        }
#pragma unroll
        for (uint32_t i = 0; i < NI; i++) {
            const f32x4 v = there ? sum[i][j] * last : f32x4{0, 0, 0, 0};
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

// Launches a workgroup for each tile of bm x bn that there can be.
template <class K>
int launch_tiles(K kernel, ProductArgs a, uint32_t threads, uint32_t bm, uint32_t bn, hipStream_t s)
{
    a.n_tiles = (a.n + bn - 1) / bn;
    const uint64_t tiles = (uint64_t)(a.m + bm - 1) / bm + (a.starts ? (a.experts < a.m ? a.experts : a.m) : 0);
    if (tiles * a.n_tiles > MAX_TILES) return ECF8_E_ARG;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles * a.n_tiles + 7) / 8 * 8)), dim3(threads), 0, s, a);
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
// full (cols 4096 to 14336).  The kernel is the one whose rounds come out shortest.
struct Shape {
    uint32_t bm, bn;
    float tile, block;
    int (*launch)(const ProductArgs &, hipStream_t);
};

template <int NT, int MT, int U>
int few(const ProductArgs &a, hipStream_t s)
{
    return launch_tiles(ecfm_few_kernel<NT, MT, U>, a, 64 * FEW_WAVES, 16 * MT, 16 * NT, s);
}

template <uint32_t BM, uint32_t BN, uint32_t WAVES_N, uint32_t STAGES>
int many(const ProductArgs &a, hipStream_t s)
{
    return launch_tiles(ecfm_many_kernel<BM, BN, WAVES_N, STAGES>, a, 512, BM, BN, s);
}

const Shape SHAPES[] = {
    {16, 16, 2.f, 0.10f, few<1, 1, 2>},        {16, 32, 2.f, 0.17f, few<2, 1, 2>},         {16, 64, 2.f, 0.26f, few<4, 1, 1>},
    {32, 32, 2.f, 0.23f, few<2, 2, 1>},        {32, 64, 2.f, 0.35f, few<4, 2, 1>},         {64, 128, 3.5f, 0.45f, many<64, 128, 2, 6>},
    {64, 256, 4.f, 0.70f, many<64, 256, 4, 3>}, {128, 128, 4.f, 0.66f, many<128, 128, 2, 4>}, {128, 256, 5.f, 1.05f, many<128, 256, 4, 3>},
    {256, 256, 6.f, 1.80f, many<256, 256, 2, 2>},
};

int launch(const ProductArgs &a, hipStream_t s)
{
    const Shape *best = nullptr;
    double least = 0;
    for (const Shape &v : SHAPES) {
        // tiles along m: of experts every last one is half empty, and as far as is known here each has rows
        double tiles = (a.m + v.bm - 1) / v.bm;
        if (a.starts) {
            const double hit = a.experts < a.m ? a.experts : a.m, full = (double)a.m / v.bm + 0.5 * hit;
            tiles = full > hit ? full : hit;
        }
        tiles *= (a.n + v.bn - 1) / v.bn;
        const double rounds = tiles <= 256 ? 1 : a.starts ? tiles / 256 : (double)(((uint64_t)tiles + 255) / 256);
        const double us = rounds * (v.tile + a.k_blocks * v.block);
        if (!best || us < least) {
            best = &v;
            least = us;
        }
    }
    return best->launch(a, s);
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
