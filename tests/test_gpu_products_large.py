"""The products on their larger tiles, several to a workgroup: sizes at which every shape of tile is chosen, odd ones, with what lies beside the operands, rows of
nobody, types and strides.  The reference is 64-bit products on the device, an expert at a time, from the definition."""
import math

import numpy as np
import pytest
import torch

import products_reference as ref
from attention_reference import E4M3
from paper_2510_02676_amd import ecfm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = 0x7f


def values(x):
    return torch.from_numpy(E4M3).to(DEV)[x.long()]


def spread(scale, rows, cols):
    return scale.double()[torch.arange(rows, device=DEV) // 128][:, torch.arange(cols, device=DEV) // 128]


def bytes_of(gen, shape, size=60.0):
    x = torch.randn(shape, generator=gen, device=DEV).mul_(size).clamp_(-448, 448)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def laid(x, gap):
    """Rows of x (..., k) k + gap bytes apart, NaN between and behind them."""
    wide = torch.full((*x.shape[:-1], x.shape[-1] + gap), NAN, dtype=torch.uint8, device=DEV)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def check(y, x, xs, w, ws, starts, rows):
    """y (m, n) against experts' products, in place of nobody's rows 777."""
    n, k = w.shape[-2:]
    half = torch.finfo(y.dtype).eps / 2
    there = torch.zeros(y.shape[0], dtype=torch.bool, device=DEV)
    for e in range(w.shape[0]):
        a, b = starts[e], starts[e + 1]
        if a == b:
            continue
        there[a:b] = True
        r = torch.arange(a, b, device=DEV) if rows is None else rows[a:b].long()
        ok = (r >= 0) & (r < x.shape[0])
        r = r.clamp(0, x.shape[0] - 1)
        xv, wv = values(x[r]), values(w[e])
        if xs is not None:
            s = xs[r].double()
            xv = xv * (s[:, None] if s.dim() == 1 else s[:, torch.arange(k, device=DEV) // 128])
        if ws is not None:
            wv = wv * spread(ws[e], n, k)
        xv = torch.where(ok[:, None], xv, torch.zeros_like(xv))
        want, size = xv @ wv.T.contiguous(), xv.abs() @ wv.abs().T.contiguous()
        off = (7 * 2.0 ** -13 + 16 * 2.0 ** -24 + (ref.blocks(k) + 12) * 2.0 ** -24) * size      # (products_reference.product_bound)
        worst = ((y[a:b].double() - want).abs() / (off + half * (want.abs() + off) + 1e-38)).max().item()
        assert worst <= 1, (e, a, b, worst)
    assert (y[~there] == 777).all()


DENSE = [(200, 4000, 2064), (130, 4100, 7184), (1000, 2100, 1040), (1500, 3001, 144), (600, 9000, 16), (4300, 4090, 1040), (4200, 4401, 272), (4200, 4400, 128),
         (5000, 4500, 1152)]


@pytest.mark.parametrize("m,n,k", DENSE)
@pytest.mark.parametrize("scales,dtype,y_gap", [("group", torch.bfloat16, 0), ("row", torch.bfloat16, 1), (None, torch.float32, 0), ("group", torch.float32, 3)])
def test_products(m, n, k, scales, dtype, y_gap):
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    x, w = bytes_of(gen, (m, k)), bytes_of(gen, (1, n, k))
    xs = None if scales is None else torch.rand((m,) if scales == "row" else (m, ref.blocks(k)), generator=gen, device=DEV) + 0.1
    ws = torch.rand((1, ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1 if scales else None
    y = torch.full((m + 1, n + y_gap), 777.0, dtype=dtype, device=DEV)
    weights = ecfm.Weights(laid(w, 16)[0], None if ws is None else ws[0])
    ecfm.ecfm_gemm(weights, laid(x, 32), xs, y=y[:-1, :n])
    check(y[:-1, :n], x, xs, w, ws, [0, m], None)
    assert (y[-1] == 777).all() and (y[:, n:] == 777).all()
    again = ecfm.ecfm_gemm(weights, laid(x, 32), xs, dtype=dtype)
    assert torch.equal(again, y[:-1, :n])


# rows, experts, and how unlike the experts' numbers of rows are
EXPERTS = [(450, 300, 1000, 1040, 1.0), (600, 40, 3000, 2064, 0.3), (900, 150, 2000, 1040, 2.0), (9000, 64, 1000, 144, 0.7), (3000, 200, 1500, 144, 1.5), (20000, 40, 700, 272, 0.7),
           (4000, 60, 260, 272, 3.0), (9000, 300, 100, 528, 1.0), (30000, 50, 300, 16, 0.2), (8, 8, 4000, 7168, 0.0), (5000, 600, 1000, 16, 1.0), (6000, 20, 1000, 656, 6.0)]


@pytest.mark.parametrize("m,experts,n,k,unlike", EXPERTS)
@pytest.mark.parametrize("scales,gather", [("group", True), ("row", False)])
def test_experts(m, experts, n, k, unlike, scales, gather):
    gen = torch.Generator(device=DEV).manual_seed(m + experts)
    rng = np.random.default_rng(m)
    share = np.exp(rng.normal(0, unlike, experts))
    counts = rng.multinomial(m - 7, share / share.sum())
    starts = [3] + (3 + np.cumsum(counts)).tolist()                        # three rows before the first, four behind the last
    tokens = m // 2 if gather else m
    x, w = bytes_of(gen, (tokens, k)), bytes_of(gen, (experts, n, k))
    xs = torch.rand((tokens,) if scales == "row" else (tokens, ref.blocks(k)), generator=gen, device=DEV) + 0.1
    ws = torch.rand((experts, ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1
    rows = None
    if gather:
        rows = torch.randint(0, tokens, (m,), generator=gen, device=DEV).to(torch.int32)
        rows[5::97] = -1
        rows[11::89] = tokens
    y = torch.full((m, n), 777.0, dtype=torch.bfloat16, device=DEV)
    s = torch.tensor(starts, dtype=torch.int32, device=DEV)
    ecfm.ecfm_gemm_experts(ecfm.Weights(laid(w, 16), ws), s, laid(x, 16), xs, rows=rows, y=y)
    check(y, x, xs, w, ws, starts, rows)


@pytest.mark.parametrize("m,n,k", [(200, 4000, 2064), (1000, 2100, 1040), (1500, 3000, 144), (4200, 4400, 272)])
def test_nan_and_infinities_stay_where_they_are(m, n, k):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, w = bytes_of(gen, (m, k)), bytes_of(gen, (n, k))
    xs, ws = torch.rand((m, ref.blocks(k)), generator=gen, device=DEV) + 0.1, torch.rand((ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1
    plain = ecfm.ecfm_gemm(ecfm.Weights(w, ws), x, xs)
    hit_rows, hit_cols = [0, m // 2, m - 1], [3, n - 1]
    x[0, 0], x[m // 2, k - 1], xs[m - 1, ref.blocks(k) - 1] = NAN, 0xff, math.inf
    w[3, k - 1], w[n - 1, 0] = NAN, NAN
    got = ecfm.ecfm_gemm(ecfm.Weights(w, ws), x, xs)
    rest = torch.ones((m, n), dtype=torch.bool, device=DEV)
    rest[hit_rows], rest[:, hit_cols] = False, False
    assert torch.equal(got[rest], plain[rest])
    assert got[[0, m // 2]].isnan().all() and got[:, hit_cols].isnan().all() and not got[m - 1].isfinite().any()


@pytest.mark.parametrize("m,experts,n,k", [(9000, 64, 1000, 144), (900, 150, 2000, 1040)])
def test_a_captured_call_with_many_tiles(m, experts, n, k):
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, w = bytes_of(gen, (m, k)), bytes_of(gen, (experts, n, k))
    xs, ws = torch.rand((m, ref.blocks(k)), generator=gen, device=DEV) + 0.1, torch.rand((experts, ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1
    weights, starts = ecfm.Weights(w, ws), torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    y = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    ecfm.ecfm_gemm_experts(weights, starts, x, xs, y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ecfm.ecfm_gemm_experts(weights, starts, x, xs, y=y)
    rng = np.random.default_rng(3)
    for unlike in (0.0, 1.0, 4.0):
        share = np.exp(rng.normal(0, unlike, experts))
        s = [0] + np.cumsum(rng.multinomial(m, share / share.sum())).tolist()
        starts.copy_(torch.tensor(s, dtype=torch.int32))
        y.fill_(777)
        graph.replay()
        torch.cuda.synchronize()
        check(y, x, xs, w, ws, s, None)
        assert torch.equal(y, ecfm.ecfm_gemm_experts(weights, starts, x, xs))


def test_starts_that_fall_with_many_tiles():
    m, experts, n, k = 5000, 64, 700, 144
    gen = torch.Generator(device=DEV).manual_seed(4)
    x, w = bytes_of(gen, (m, k)), bytes_of(gen, (experts, n, k))
    y = torch.full((m + 2, n), 777.0, dtype=torch.bfloat16, device=DEV)
    for starts in ([0, m] * 32 + [0], [m, 0] * 32 + [m], list(range(m, m - 65, -1)), [2 ** 31 - 1, -2 ** 31] * 32 + [7]):
        ecfm.ecfm_gemm_experts(ecfm.Weights(w), torch.tensor(starts, dtype=torch.int32, device=DEV), x, y=y[1:-1])
        torch.cuda.synchronize()
        assert (y[0] == 777).all() and (y[-1] == 777).all()


def test_rows_of_x_far_apart_on_large_tiles():
    """Rows 2^23 bytes apart, so that the last ones lie beyond 2^32."""
    m, n, k, far = 700, 3000, 272, 1 << 23
    gen = torch.Generator(device=DEV).manual_seed(5)
    x, w = bytes_of(gen, (m, k)), bytes_of(gen, (1, n, k))
    wide = torch.as_strided(torch.empty(far * m, dtype=torch.uint8, device=DEV), (m, k), (far, 1))
    wide.copy_(x)
    xs = torch.rand((m, ref.blocks(k)), generator=gen, device=DEV) + 0.1
    y = ecfm.ecfm_gemm(ecfm.Weights(w[0]), wide, xs)
    check(y, x, xs, w, None, [0, m], None)
    del wide
    torch.cuda.empty_cache()
