"""ecfm_gate and ecfm_combine against the definitions in 64 bits: both types, odd sizes, strides, numbers of any size, places that lead nowhere."""
import math

import numpy as np
import pytest
import torch

import products_reference as ref
from attention_reference import E4M3
from paper_2510_02676_amd import ecfm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def wide(x, gap):
    out = torch.full((x.shape[0], x.shape[1] + gap), math.nan, dtype=x.dtype)
    out[:, :x.shape[1]] = x
    return out.to(DEV)[:, :x.shape[1]]


def check_gate(g, u, group, gap=0):
    rows, cols = g.shape
    q, scale = ecfm.ecfm_gate(wide(g, gap), wide(u, 2 * gap), group)
    assert q.dtype == torch.float8_e4m3fn and scale.shape == ((rows, cols // 128) if group else (rows,))
    h = ref.gate(g.double().numpy(), u.double().numpy())
    parts = h.reshape(rows, -1, 128) if group else h
    most = np.maximum(np.abs(parts).max(axis=-1), 2.0 ** -100)
    s = scale.cpu().double().numpy()
    # fp32: exp to 2 of its last places, the product g t, the sum 1 + t, the quotient, the product with u, 448 into the largest: 8 half steps; what is
    # below the smallest normal number of fp32 is off by its step
    near = 8 * 2.0 ** -24
    assert (np.abs(s - most / 448) <= near * most / 448 + 2.0 ** -149).all()
    got = E4M3[q.cpu().view(torch.uint8).numpy()].reshape(parts.shape) * s[..., None]
    # half a step of E4M3: 2^-4 of the value, or 2^-10 (half its smallest number) times the scale
    tol = np.maximum(2.0 ** -4 * np.abs(parts), 2.0 ** -10 * s[..., None]) * (1 + 2.0 ** -10) + 3 * near * np.abs(parts) + 2.0 ** -140
    assert (np.abs(got - parts) <= tol).all(), np.abs(got - parts).max()


@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (3, 48), (5, 2048), (17, 1040), (2, 8192), (3, 8208), (2, 40960), (300, 256), (1000, 128)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("gap", [0, 8])
def test_gate(rows, cols, dtype, gap):
    gen = torch.Generator().manual_seed(cols)
    g, u = (torch.randn((rows, cols), generator=gen).mul(torch.exp(2 * torch.randn((rows, 1), generator=gen))).to(dtype) for _ in range(2))
    check_gate(g, u, 0, gap)
    if cols % 128 == 0:
        check_gate(g, u, 128, gap)


@pytest.mark.parametrize("group", [0, 128])
def test_gate_of_numbers_of_any_size(group):
    rows = [(0.0, 1.0), (-0.0, 3.0), (1e-30, 1e-30), (-20.0, 2.0), (-60.0, 1e20), (-80.0, 1e30), (50.0, 1e30), (1e30, 1e-30), (3e38, 0.5), (1.0, 0.0), (-3e38, 1.0)]
    gen = torch.Generator().manual_seed(0)
    noise = torch.rand((2, len(rows), 256), generator=gen) * 0.1 + 0.95
    g = torch.tensor([r[0] for r in rows])[:, None] * noise[0]
    u = torch.tensor([r[1] for r in rows])[:, None] * noise[1]
    check_gate(g, u, group)


def test_gate_with_infinities():
    g, u = torch.ones((5, 256)), torch.ones((5, 256))
    g[0, 3], u[1, 200], g[2, 5], g[3, 7], u[4, 130] = math.inf, -math.inf, -math.inf, math.nan, math.nan
    q, s = ecfm.ecfm_gate(g.to(DEV), u.to(DEV))
    assert s[0].item() == math.inf and s[1].item() == math.inf and s[2].isfinite() and s[3].isnan() and s[4].isnan()
    assert E4M3[int(q[2, 5].view(torch.uint8))] == 0 and not q[2].float().isnan().any()
    _, s = ecfm.ecfm_gate(g.to(DEV), u.to(DEV), 128)
    assert s.isfinite().tolist() == [[False, True], [True, False], [True, True], [False, True], [True, False]]


def test_gate_of_no_rows_and_in_given_memory():
    x = torch.randn((0, 128), device=DEV)
    assert ecfm.ecfm_gate(x, x, 128)[1].shape == (0, 1)
    x = torch.randn((4, 128), device=DEV)
    q, s = torch.zeros((4, 128), dtype=torch.uint8, device=DEV), torch.zeros(4, device=DEV)
    a = ecfm.ecfm_gate(x, x, 0, q, s)
    b = ecfm.ecfm_gate(x, x)
    assert a[0] is q and a[1] is s and torch.equal(b[0].view(torch.uint8), q) and torch.equal(b[1], s)


def check_combine(tokens, top, cols, rows, dtype, add=None, out=None, gap=0, seed=0, holes=True):
    gen = torch.Generator().manual_seed(seed)
    y = torch.randn((rows, cols), generator=gen).to(dtype)
    place = torch.randint(-2 if holes else 0, rows + 2 if holes else max(rows, 1), (tokens, top), generator=gen).to(torch.int32)
    w = torch.randn((tokens, top), generator=gen)
    a = None if add is None else torch.randn((tokens, cols), generator=gen).to(add)
    got = ecfm.ecfm_combine(wide(y, gap), place.to(DEV), w.to(DEV), add=None if a is None else wide(a, gap), dtype=out)
    assert got.dtype == out
    want = np.zeros((tokens, cols)) if a is None else a.double().numpy().copy()
    size = np.abs(want)
    for j in range(top):
        p = place[:, j].long().numpy()
        ok = (p >= 0) & (p < rows)
        if rows:
            term = w[:, j].double().numpy()[:, None] * y.double().numpy()[np.where(ok, p, 0)] * ok[:, None]
            want, size = want + term, size + np.abs(term)
    half = 2.0 ** -8 if out == BF else 2.0 ** -24
    err = np.abs(got.cpu().double().numpy() - want)
    assert (err <= (top + 1) * 2.0 ** -24 * size + half * (np.abs(want) + (top + 1) * 2.0 ** -24 * size) + 1e-40).all()


@pytest.mark.parametrize("tokens,top,cols,rows", [(1, 1, 8, 1), (1, 8, 7168, 8), (3, 2, 40, 6), (50, 6, 1000, 300), (300, 32, 64, 9600), (7, 5, 16, 0)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("add", [None, BF, F32])
@pytest.mark.parametrize("out", [BF, F32])
def test_combine(tokens, top, cols, rows, dtype, add, out):
    check_combine(tokens, top, cols, rows, dtype, add, out)
    check_combine(tokens, top, cols, rows, dtype, add, out, gap=8, seed=1, holes=rows == 0)


def test_combine_onto_what_is_there_and_no_tokens():
    y, place, w = torch.randn((6, 128), device=DEV), torch.tensor([[0, 5], [3, -1]], dtype=torch.int32, device=DEV), torch.tensor([[0.5, 2.0], [3.0, math.nan]], device=DEV)
    x = torch.randn((2, 128), device=DEV).to(BF)
    want = ecfm.ecfm_combine(y, place, w, add=x)
    assert want[1].isfinite().all()                                        # the weight of a place that leads nowhere does not count
    got = x.clone()
    assert ecfm.ecfm_combine(y, place, w, add=got, out=got) is got and torch.equal(got, want)
    assert ecfm.ecfm_combine(y, place[:0], w[:0]).shape == (0, 128)


def test_combine_of_rows_beyond_32_bits():
    cols = 1 << 14
    rows = (1 << 32) // (2 * cols) + 3
    y = torch.empty((rows, cols), dtype=BF, device=DEV)
    y[0], y[rows - 1] = 1.0, 2.0
    place = torch.tensor([[rows - 1, 0]], dtype=torch.int32, device=DEV)
    assert (ecfm.ecfm_combine(y, place, torch.tensor([[1.0, 0.5]], device=DEV)) == 2.5).all()
