// What the kernels of the products of many rows share: their arguments, which rows of which expert a workgroup has, one product of
// 16 x 128 by 128 x 16 on the FP8 matrix cores.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "ecfm.h"

namespace ecfm {

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct ProductArgs {
    const uint8_t *w, *x;
    const float *w_scale, *x_scale;
    const int32_t *starts, *rows;                  // NULL: one expert with every row; row p of X
    void *y;
    int64_t w_row, w_expert, x_row, y_row;         // strides: bytes, of Y elements
    uint32_t n, k, k_blocks, n_blocks;             // rows and columns of W, its 128 x 128 blocks
    uint32_t m, x_rows, experts, x_per;            // rows of Y and X; x_per: scales a row of X
    uint32_t n_tiles, m_tiles;                     // tiles along n; along m at most
    uint32_t f32, wide, lines;                     // Y in fp32; four elements of Y may be stored at once; BF16, and eight (n a multiple of eight)
};

struct Rows {                                      // m0 .. m1 of Y, expert e, whose rows end at `end`
    uint32_t e, m0, m1, end;
};

__device__ inline uint32_t cut(int32_t v, uint32_t m) { return v < 0 ? 0 : (uint32_t)v > m ? m : (uint32_t)v; }

// The rows of expert e: begin, and how many.  Starts that fall give none.
__device__ inline uint32_t rows_of(const ProductArgs &a, uint32_t e, uint32_t *n)
{
    const uint32_t b = cut(a.starts[e], a.m), c = cut(a.starts[e + 1], a.m);
    *n = c > b ? c - b : 0;
    return b;
}

// The tiles of BM rows, experts one after the other, each beginning with a tile of its own.  All lanes of a wave together: a lane counts the
// tiles of ceil(experts / 64) experts, a scan over the lanes adds them up; then find() looks for a tile's owner.
template <uint32_t BM>
struct Tiles {
    uint32_t mine, upto, all;

    __device__ explicit Tiles(const ProductArgs &a)
    {
        if (!a.starts) {
            all = a.m_tiles;
            return;
        }
        const uint32_t lane = threadIdx.x & 63, per = (a.experts + 63) / 64;
        mine = 0;
        for (uint32_t i = 0; i < per; i++) {
            const uint32_t e = lane * per + i;
            uint32_t n = 0;
            if (e < a.experts) rows_of(a, e, &n);
            mine += (n + BM - 1) / BM;
        }
        upto = mine;
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t v = __shfl_up(upto, d);
            upto += lane >= d ? v : 0;
        }
        all = __builtin_amdgcn_readlane(upto, 63);
        all = all < a.m_tiles ? all : a.m_tiles;               // (starts that fall could claim more)
    }

    // false: there is no tile t; else its expert's first tile and how many these are
    __device__ bool find(const ProductArgs &a, uint32_t t, Rows *r, uint32_t *t0 = nullptr, uint32_t *tn = nullptr) const
    {
        if (t >= all) return false;
        if (!a.starts) {
            r->e = 0;
            r->m0 = t * BM;
            r->m1 = a.m - r->m0 < BM ? a.m : r->m0 + BM;
            r->end = a.m;
            if (t0) *t0 = 0;
            if (tn) *tn = all;
            return true;
        }
        const uint64_t hit = __ballot(upto > t);
        if (!hit) return false;
        const uint32_t per = (a.experts + 63) / 64, l = (uint32_t)__ffsll((unsigned long long)hit) - 1;
        uint32_t before = __builtin_amdgcn_readlane(upto - mine, l);
        for (uint32_t e = l * per; e < a.experts && e < (l + 1) * per; e++) {
            uint32_t n;
            const uint32_t b = rows_of(a, e, &n), tiles = (n + BM - 1) / BM;
            if (t - before < tiles) {
                r->e = e;
                r->m0 = b + (t - before) * BM;
                r->m1 = b + n - r->m0 < BM ? b + n : r->m0 + BM;
                r->end = b + n;
                if (t0) *t0 = before;
                if (tn) *tn = tiles;
                return true;
            }
            before += tiles;
        }
        return false;
    }
};

// A lane's 32 of the 128 columns of a row: 16 at 16 g and 16 at 64 + 16 g (g = lane / 16).  Which 32 does not matter as long as both operands
// take the same; this way a load of a wave covers 64 columns of 16 rows.
union Piece {
    i32x8 v;
    u32x4 h[2];
};

// d[i] of lane l: row 4 (l / 16) + i of the first operand by row l % 16 of the second, over 128 columns.  The one place where a sum has fewer bits than
// fp32: of eight neighbouring products the matrix core drops what lies more than 13 bits below the largest, and joins the eights with 24.  That is 2^-16 of an
// ordinary result's norm, 2^-8 of the rounding to BF16 behind it; exact sums would need the F16 matrix cores, at half the rate and with E4M3 spread out to F16.
__device__ inline f32x4 product(const Piece &a, const Piece &b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

// Four neighbours along n of row m of Y.
__device__ inline void store_y(const ProductArgs &a, uint32_t m, uint32_t n, const f32x4 &v)
{
    if (n >= a.n) return;
    const int64_t at = (int64_t)m * a.y_row + n;
    if (a.wide && n + 4 <= a.n) {
        if (a.f32) *(f32x4 *)((float *)a.y + at) = v;
        else *(bf16x4 *)((__bf16 *)a.y + at) = __builtin_convertvector(v, bf16x4);
        return;
    }
    for (uint32_t i = 0; i < 4; i++)
        if (n + i < a.n) {
            if (a.f32) ((float *)a.y)[at + i] = v[i];
            else ((__bf16 *)a.y)[at + i] = (__bf16)v[i];
        }
}

} // namespace ecfm
