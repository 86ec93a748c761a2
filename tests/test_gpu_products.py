"""ecfm_gemm and ecfm_gemm_experts against the definitions in 64 bits: odd and ragged sizes, scales of all kinds, strides, NaN in and beside the operands, experts
without rows, starts and row numbers of any value, rows that belong to nobody left as they were, streams, graphs."""
import numpy as np
import pytest
import torch

import products_reference as ref
from paper_2510_02676_amd import ecf8, ecfm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = 0x7f
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float32)}          # half a step, relative to the value


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def e4m3(g, shape, size=60.0):
    return torch.randn(shape, generator=g).mul(size).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def laid(x, gap):
    """A copy of x (..., k) on the device whose rows lie k + gap bytes apart, NaN between and behind them."""
    if not gap:
        return x.to(DEV)
    wide = torch.full((*x.shape[:-1], x.shape[-1] + gap), NAN, dtype=torch.uint8)
    wide[..., :x.shape[-1]] = x
    return wide.to(DEV)[..., :x.shape[-1]]


def inputs(m, n, k, scales, w_scaled=True, seed=0, experts=None):
    g = torch.Generator().manual_seed(seed)
    lead = () if experts is None else (experts,)
    w, x = e4m3(g, (*lead, n, k)), e4m3(g, (m, k))
    ws = torch.rand((*lead, ref.blocks(n), ref.blocks(k)), generator=g) * 0.01 + 1e-3 if w_scaled else None
    xs = None if scales is None else torch.rand((m,) if scales == "row" else (m, ref.blocks(k)), generator=g) + 0.1
    return x, xs, w, ws


def dev(t):
    return None if t is None else t.to(DEV)


def arr(t):
    return None if t is None else t.numpy()


def check(got, want, size, k):
    tol = ref.product_bound(want, size, k, HALF[got.dtype])
    got = got.cpu().double().numpy()
    assert np.isfinite(got).all()
    worst = np.abs(got - want) / tol
    assert worst.max(initial=0.0) <= 1, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


SIZES = [(1, 1, 16), (1, 16, 128), (2, 17, 144), (3, 7168, 48), (8, 64, 4096), (16, 16, 256), (16, 48, 2064), (17, 33, 272), (31, 144, 1008), (33, 1000, 512),
         (64, 130, 1040), (65, 129, 128), (97, 300, 144), (128, 128, 384), (129, 257, 384), (200, 64, 7168), (255, 255, 256), (256, 256, 512), (257, 513, 272),
         (300, 520, 640), (513, 640, 256), (700, 1001, 1040), (1025, 300, 400)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("scales", [None, "row", "group"])
def test_products(m, n, k, scales):
    x, xs, w, ws = inputs(m, n, k, scales, w_scaled=scales != "row" or m % 2 == 1)
    y = torch.full((m + 2, n), 777.0, dtype=torch.bfloat16, device=DEV)
    weights = ecfm.Weights(dev(w), dev(ws))
    assert ecfm.ecfm_gemm(weights, dev(x), dev(xs), y=y[1:-1]).data_ptr() == y[1:-1].data_ptr()
    check(y[1:-1], *ref.product(arr(x), arr(xs), arr(w), arr(ws)), k)
    assert (y[0] == 777).all() and (y[-1] == 777).all()
    assert torch.equal(ecfm.ecfm_gemm(weights, dev(x).view(torch.float8_e4m3fn), dev(xs)), y[1:-1])       # the same again, in memory of the call


@pytest.mark.parametrize("m,n,k", [(1, 5, 16), (5, 200, 272), (40, 36, 528), (130, 100, 144), (300, 300, 272)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("y_gap", [0, 1, 4])
def test_strides_and_types(m, n, k, dtype, y_gap):
    x, xs, w, ws = inputs(m, n, k, "group", seed=1)
    y = torch.full((m, n + y_gap), 777.0, dtype=dtype, device=DEV)
    ecfm.ecfm_gemm(ecfm.Weights(laid(w, 32), dev(ws)), laid(x, 16), dev(xs), y=y[:, :n])
    check(y[:, :n], *ref.product(arr(x), arr(xs), arr(w), arr(ws)), k)
    assert (y[:, n:] == 777).all()
    fresh = ecfm.ecfm_gemm(ecfm.Weights(laid(w, 32), dev(ws)), laid(x, 16), dev(xs), dtype=dtype)
    assert fresh.dtype == dtype and torch.equal(fresh, y[:, :n])


@pytest.mark.parametrize("m,n,k", [(7, 50, 272), (70, 50, 144), (300, 290, 272)])
def test_rows_backwards_and_the_same_row_many_times(m, n, k):
    x, xs, w, ws = inputs(m, n, k, "row", seed=2)
    want, size = ref.product(arr(x), arr(xs), arr(w), arr(ws))
    flat = dev(w)
    once = torch.as_strided(dev(x), (m, k), (0, 1))                        # every row is the first one
    got = ecfm.ecfm_gemm(ecfm.Weights(flat, dev(ws)), once, dev(xs))
    row, row_size = ref.product(arr(x[:1].expand(m, k).contiguous()), arr(xs), arr(w), arr(ws))
    check(got, row, row_size, k)
    c = ecfm.Weights(flat, dev(ws))
    d_x, d_xs, y = dev(x), dev(xs), torch.empty((m, n), dtype=torch.float32, device=DEV)
    back = ecfm._Y(y[-1].data_ptr(), -n, m, ecfm._DTYPE[y.dtype])          # rows of Y from the last to the first: a negative stride, through the C ABI
    s = torch.cuda.current_stream().cuda_stream
    assert ecfm._lib.ecfm_gemm(c.c, ecfm._X(d_x.data_ptr(), d_xs.data_ptr(), k, m, 1), back, s) == ecf8.OK
    check(y.flip(0), want, size, k)


@pytest.mark.parametrize("m,n,k", [(9, 40, 272), (80, 140, 272), (300, 290, 272)])
def test_nan_stays_in_its_row_and_column(m, n, k):
    x, xs, w, ws = inputs(m, n, k, "group", seed=3)
    want, size = ref.product(arr(x), arr(xs), arr(w), arr(ws))
    x[m // 2, k - 1], w[n - 3, 5], x[0, 0] = NAN, 0xff, NAN
    got = ecfm.ecfm_gemm(ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs), dtype=torch.float32).cpu()
    hit = torch.zeros((m, n), dtype=torch.bool)
    hit[m // 2], hit[0], hit[:, n - 3] = True, True, True
    assert got[hit].isnan().all()
    got[hit], want[hit.numpy()] = 0, 0
    check(got, want, size, k)


def test_scales_of_any_size_and_sign():
    x, xs, w, ws = inputs(20, 300, 400, "group", seed=4)
    xs[3], xs[4], ws[1, 2], ws[2] = 1e30, 0.0, -3.0, 1e-30
    got = ecfm.ecfm_gemm(ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs), dtype=torch.float32)
    check(got, *ref.product(arr(x), arr(xs), arr(w), arr(ws)), 400)
    xs[7, 1] = float("inf")                                                # a quantiser's scale of a group with an infinity
    got = ecfm.ecfm_gemm(ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs)).cpu()
    assert not got[7].isfinite().any() and got[:7].isfinite().all() and got[8:].isfinite().all()


@pytest.mark.parametrize("m,n,k", [(9, 40, 272), (40, 100, 1152), (70, 140, 128), (300, 290, 400)])
def test_infinite_scales(m, n, k):
    """A block whose scale is infinite gives an infinity of its sum's sign, whichever block of the row it is."""
    x, xs, w, ws = inputs(m, n, k, "group", seed=10)
    for b in range(ref.blocks(k)):
        xs[b % m, b] = float("inf")
        ws[0, b] *= -1 if b % 2 else 1
    xs[m - 1, -1] = float("-inf")
    got = ecfm.ecfm_gemm(ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs), dtype=torch.float32).cpu().numpy()
    for r, b in [(b % m, b) for b in range(ref.blocks(k))] + [(m - 1, ref.blocks(k) - 1)]:
        if np.isinf(arr(xs)[r]).sum() > 1:
            continue
        part = ref.E4M3[arr(x)[r, 128 * b:128 * b + 128]] @ ref.E4M3[arr(w)[:, 128 * b:128 * b + 128]].T
        clear = np.abs(part) > 2.0 ** -9 * np.abs(ref.E4M3[arr(x)[r, 128 * b:128 * b + 128]]).sum() * 448
        want = np.sign(part) * np.sign(arr(ws)[np.arange(n) // 128, b]) * np.float64(arr(xs)[r, b])
        assert clear.any() and (got[r][clear] == want[clear]).all()


@pytest.mark.parametrize("m", [3, 70, 200])
def test_operands_further_apart_than_32_bits(m):
    n, k, far = 40, 144, (1 << 31) // m // 16 * 16 + 16 * 1000             # rows of X; the last one lies beyond 2^31, in Y beyond 2^32 bytes
    x, xs, w, ws = inputs(m, n, k, "row", seed=5)
    room = torch.empty(far * m, dtype=torch.uint8, device=DEV)
    wide = torch.as_strided(room, (m, k), (far, 1))
    wide.copy_(dev(x))
    out = torch.as_strided(torch.empty(far * m, dtype=torch.bfloat16, device=DEV), (m, n), (far, 1))
    ecfm.ecfm_gemm(ecfm.Weights(dev(w), dev(ws)), wide, dev(xs), y=out)
    check(out, *ref.product(arr(x), arr(xs), arr(w), arr(ws)), k)
    del room, out
    torch.cuda.empty_cache()


def experts_want(x, xs, w, ws, starts, rows, m, n):
    """(Y, size, rows that are written)."""
    want, size, there = np.zeros((m, n)), np.zeros((m, n)), np.zeros(m, dtype=bool)
    for e in range(w.shape[0]):
        a, b = (min(max(v, 0), m) for v in starts[e:e + 2])
        for p in range(a, b):
            there[p] = True
        if b <= a:
            continue
        r = np.arange(a, b) if rows is None else np.asarray(rows[a:b])
        ok = (r >= 0) & (r < x.shape[0])
        r = np.where(ok, r, 0)
        y, s = ref.product(arr(x)[r], None if xs is None else arr(xs)[r], arr(w[e]), None if ws is None else arr(ws[e]))
        want[a:b], size[a:b] = y * ok[:, None], s * ok[:, None]
    return want, size, there


def run_experts(counts, n, k, scales="group", gather=False, first=0, behind=0, dtype=torch.bfloat16, seed=0, w_gap=0, tokens=0):
    starts = [first] + (first + np.cumsum(counts)).tolist()
    m = starts[-1] + behind
    g = torch.Generator().manual_seed(seed + 100)
    tokens = (tokens or max(1, m // 3)) if gather else m
    rows = torch.randint(0, tokens, (m,), generator=g).tolist() if gather else None
    x, xs, w, ws = inputs(tokens, n, k, scales, seed=seed, experts=len(counts))
    y = torch.full((m, n), 777.0, dtype=dtype, device=DEV)
    ecfm.ecfm_gemm_experts(ecfm.Weights(laid(w, w_gap), dev(ws)), i32(starts), dev(x), dev(xs), rows=None if rows is None else i32(rows), y=y)
    want, size, there = experts_want(x, xs, w, ws, starts, rows, m, n)
    check(y[torch.from_numpy(there)], want[there], size[there], k)
    assert (y.cpu()[~torch.from_numpy(there)] == 777).all()


COUNTS = [[1], [0, 3], [16, 0, 17, 1], [0, 0, 0, 5], [1] * 70, [40, 0, 130, 7, 64, 65], [300, 1, 0, 255], [0] * 200 + [2] + [0] * 99, [257, 600], [130] * 5]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "%dx%d" % (len(c), sum(c)))
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("n,k,scales", [(17, 144, "group"), (260, 272, "row"), (128, 16, None)])
def test_experts(counts, gather, n, k, scales):
    run_experts(counts, n, k, scales, gather, seed=len(counts))


@pytest.mark.parametrize("counts", [[3, 0, 9], [200, 30]], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_nobody(counts, dtype):
    run_experts(counts, 70, 272, gather=True, first=2, behind=40, dtype=dtype, w_gap=16)
    run_experts([0] * len(counts), 70, 272, first=5, behind=3, dtype=dtype)


def test_many_experts():
    counts = np.random.default_rng(0).integers(0, 4, 1025).tolist()
    run_experts(counts, 20, 48, "row", gather=True)
    run_experts([0] * 4095 + [70], 20, 48)


@pytest.mark.parametrize("size", [20, 300])
def test_starts_and_rows_of_any_value(size):
    n, k, m, experts = 70, 144, size, 6
    x, xs, w, ws = inputs(9, n, k, "group", seed=6, experts=experts)
    for starts in ([-5, 3, 3, size // 2, size // 2, size + 7, 2 ** 31 - 1], [0, 0, 0, 0, 0, 0, 0], [-2 ** 31, -1, 0, 1, 2, size, size]):
        rows = [(-1, 0, 8, 9, 2 ** 31 - 1, -2 ** 31, 4)[i % 7] for i in range(m)]
        y = torch.full((m + 2, n), 777.0, device=DEV)
        ecfm.ecfm_gemm_experts(ecfm.Weights(dev(w), dev(ws)), i32(starts), dev(x), dev(xs), rows=i32(rows), y=y[1:-1])
        want, size_, there = experts_want(x, xs, w, ws, starts, rows, m, n)
        check(y[1:-1][torch.from_numpy(there)], want[there], size_[there], k)
        assert (y[1:-1].cpu()[~torch.from_numpy(there)] == 777).all() and (y[0] == 777).all() and (y[-1] == 777).all()
    # starts that fall: which rows are written is not said, but none outside
    y = torch.full((m + 2, n), 777.0, device=DEV)
    ecfm.ecfm_gemm_experts(ecfm.Weights(dev(w), dev(ws)), i32([0, m, 0, m, 3, m, 0]), dev(x), dev(xs), rows=i32([0] * m), y=y[1:-1])
    assert (y[0] == 777).all() and (y[-1] == 777).all()


def test_no_rows():
    x, xs, w, ws = inputs(0, 30, 144, "group", experts=2)
    assert ecfm.ecfm_gemm_experts(ecfm.Weights(dev(w), dev(ws)), i32([0, 0, 0]), dev(x), dev(xs)).shape == (0, 30)
    assert ecfm.ecfm_gemm(ecfm.Weights(dev(w)[0], dev(ws)[0]), dev(x), dev(xs)).shape == (0, 30)


def test_experts_further_apart_than_32_bits():
    n, k, far = 33, 144, (1 << 32) + 4096
    x, xs, w, ws = inputs(50, n, k, "row", seed=7, experts=2)
    room = torch.empty(far + n * k, dtype=torch.uint8, device=DEV)
    wide = torch.as_strided(room, (2, n, k), (far, k, 1))
    wide.copy_(dev(w))
    y = ecfm.ecfm_gemm_experts(ecfm.Weights(wide, dev(ws)), i32([0, 21, 50]), dev(x), dev(xs))
    want, size, _ = experts_want(x, xs, w, ws, [0, 21, 50], None, 50, n)
    check(y, want, size, k)
    del room, wide
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m", [24, 400])
def test_a_captured_call_follows_what_is_rewritten(m):
    n, k, experts = 130, 272, 5
    x, xs, w, ws = inputs(m, n, k, "group", seed=8, experts=experts)
    weights, d_x, d_xs = ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs)
    starts, rows, y = i32([0] * 6), i32([0] * m), torch.zeros((m, n), device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ecfm.ecfm_gemm_experts(weights, starts, d_x, d_xs, rows=rows, y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ecfm.ecfm_gemm_experts(weights, starts, d_x, d_xs, rows=rows, y=y)
    gen = np.random.default_rng(1)
    for _ in range(4):
        s = np.concatenate(([0], np.sort(gen.integers(0, m + 1, experts - 1)), [m])).tolist()
        r = gen.integers(0, m, m).tolist()
        starts.copy_(i32(s))
        rows.copy_(i32(r))
        y.fill_(777)
        graph.replay()
        torch.cuda.synchronize()
        want, size, _ = experts_want(x, xs, w, ws, s, r, m, n)
        check(y, want, size, k)
        assert torch.equal(y, ecfm.ecfm_gemm_experts(weights, starts, d_x, d_xs, rows=rows, dtype=torch.float32))


@pytest.mark.parametrize("m", [5, 300])
def test_on_another_stream(m):
    x, xs, w, ws = inputs(m, 200, 400, "group", seed=9)
    weights, d_x, d_xs = ecfm.Weights(dev(w), dev(ws)), dev(x), dev(xs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = ecfm.ecfm_gemm(weights, d_x, d_xs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check(y, *ref.product(arr(x), arr(xs), arr(w), arr(ws)), 400)
