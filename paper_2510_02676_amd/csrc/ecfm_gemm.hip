// Products of many rows, and of experts with the rows that were sent to them: Y = X W^T of E4M3 with block scales (ecfm.h).
#include "ecfm_device.h"

namespace ecfm {
namespace {

constexpr uint32_t FEW_WAVES = 8;

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
    if (!find_rows<16 * MT>(a, a.first_tile + blockIdx.x / a.n_tiles, &r)) return;
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

// Launches the tiles of `rows` rows of Y, 16 MT (or whatever the kernel takes) at a time.
template <class K>
int launch_tiles(K kernel, ProductArgs a, uint32_t threads, uint32_t bm, uint32_t bn, hipStream_t s)
{
    a.n_tiles = (a.n + bn - 1) / bn;
    const uint64_t tiles = (uint64_t)(a.m + bm - 1) / bm + (a.starts ? (a.experts < a.m ? a.experts : a.m) : 0);
    const uint64_t most = 0x7fffffffu / threads / a.n_tiles ? 0x7fffffffu / threads / a.n_tiles : 1;   // of a launch: its threads are counted in 32 bits
    for (uint64_t t = 0; t < tiles; t += most) {
        a.first_tile = (uint32_t)t;
        const uint64_t n = tiles - t < most ? tiles - t : most;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(n * a.n_tiles)), dim3(threads), 0, s, a);
        if (hipGetLastError() != hipSuccess) return ECF8_E_HIP;
    }
    return ECF8_OK;
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
    return ECF8_OK;
}

int launch(const ProductArgs &a, hipStream_t s)
{
    return launch_tiles(ecfm_few_kernel<1, 1, 2>, a, 64 * FEW_WAVES, 16, 16, s);
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
