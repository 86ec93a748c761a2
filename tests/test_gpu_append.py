"""ecfa_append and ecfa_quant against the definitions in 64 bits: both layouts of pairs, parts of a head, positions to 10^6 and beyond, all
types, places in holes and before the start, everything else in the pool untouched; rows that hold zeros, infinities, NaN and
numbers of any size."""
import itertools
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
from paper_2510_02676_amd import ecf8, ecfa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def freqs(rot, base=10000.0):
    return [int(base ** (-2.0 * j / rot) / (2 * math.pi) * 2.0 ** 64) for j in range(rot // 2)]


def check_append(kv, qn, heads=4, kv_heads=2, dim=64, rot=None, interleaved=False, src=torch.float32, cache="bf16", page=16, order="token", pos=None, scale=1.0,
                 base=10000.0, holes=(), seed=0, single=False, with_q=True, with_kv=True, width=None, size=1.0):
    g = torch.Generator().manual_seed(seed)
    rot = dim if rot is None else rot
    need = [-(-max(0, n) // page) for n in kv]
    width = max(max(need), 1) if width is None else width
    pages = sum(need) + 2
    ids = torch.randperm(pages, generator=g).tolist()
    table = [[-1] * width for _ in kv]
    for s, n in enumerate(need):
        for j in range(min(n, width)):
            table[s][j] = ids.pop()
    for s, j, what in holes:
        table[s][j] = what
    start = [0] + list(itertools.accumulate(qn))
    n = start[-1]
    shape = (pages, kv_heads, page, dim) if order == "head" else (pages, page, kv_heads, dim)
    old = torch.randint(0, 256, (*shape[:-1], shape[-1] * (1 if cache == "e4m3" else 2)), dtype=torch.uint8, generator=g)
    pools = [old.to(DEV), old.flip(0).contiguous().to(DEV)]
    before = [p.clone() for p in pools]
    views = [p if cache == "e4m3" else p.view(torch.bfloat16) for p in pools]
    if order == "head":
        views = [v.transpose(1, 2) for v in views]
    scales = [None, None] if cache != "e4m3" else [torch.rand(kv_heads, generator=g) * 0.02 + 0.005 for _ in range(2)]
    q, k, v = (torch.randn((n, h, dim), generator=g).mul(size).to(src) for h in (heads, kv_heads, kv_heads))
    f = freqs(rot, base) if rot else []
    rope = None
    if rot:
        rope = ecfa.Rope(torch.tensor(f, dtype=torch.int64, device=DEV), interleaved=interleaved, scale=scale, pos=None if pos is None else i32(pos))
    c = ecfa.Cache(views[0], views[1], *(None if x is None else x.to(DEV) for x in scales))
    b = ecfa.Batch(i32(table).view(len(kv), width), i32(kv), None if single else i32(start), n_tokens=n)
    q_out = torch.full((n + 2, heads, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
    got = ecfa.ecfa_append(c, b, *((k.to(DEV), v.to(DEV)) if with_kv else (None, None)), *((q.to(DEV), q_out[1:-1]) if with_q else (None, None)), rope=rope)
    torch.cuda.synchronize()
    toks = ref.tokens(start, kv, table, page, pages)
    # places of tokens that come before the cache's start: negative, counted down from 0
    places = [max(0, kv[s]) - qn[s] + i for s in range(len(kv)) for i in range(qn[s])]
    where = places if pos is None else pos
    turn = lambda x: ref.turned(x.double().numpy(), where, f, rot, interleaved, scale) if rot else x.double().numpy()  # noqa: E731
    assert torch.isnan(q_out[0]).all() and torch.isnan(q_out[-1]).all()
    if with_q:
        assert got.data_ptr() == q_out[1:-1].data_ptr()
        want = turn(q)
        assert ref.near_bf16(got.cpu().double().numpy(), want, 2 * np.abs(q.double().numpy()).max(-1, keepdims=True) * abs(scale)).all()
    written = torch.zeros((pages, page), dtype=torch.bool)
    for view, new, sc in ((views[0], turn(k), scales[0]), (views[1], v.double().numpy(), scales[1])):
        held = ref.values(view)
        for t, (s, _, slots) in enumerate(toks):
            p = places[t]
            if not with_kv or p < 0 or p >= len(slots) or slots[p] is None:
                continue
            written[slots[p]] = True
            most = 2 * np.abs(new[t]).max(-1, keepdims=True) + 2 * np.abs(k[t].double().numpy()).max(-1, keepdims=True)
            if cache == "e4m3":
                by = sc.double().numpy()[:, None]
                assert ref.near_e4m3(held[slots[p]], new[t] / by, most / by).all()
            else:
                assert ref.near_bf16(held[slots[p]], new[t], most).all()
    for view, pool, was in zip(views, pools, before):
        was = was if cache == "e4m3" else was.view(torch.bfloat16)
        was = was.transpose(1, 2) if order == "head" else was
        same = (view.contiguous().view(torch.uint8) == was.contiguous().view(torch.uint8)).all(-1).all(-1).cpu()
        assert same[~written].all()
    return written


@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 160, 176, 192, 240, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_sizes_and_parts(dim, interleaved):
    for rot in sorted({dim, 16, dim // 32 * 16 or 16}):
        check_append([20, 7], [5, 1], dim=dim, rot=rot, interleaved=interleaved, seed=dim + rot, cache="e4m3" if dim % 32 else "bf16")


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_and_orders(src, cache, order, interleaved):
    check_append([33, 1, 70, 5], [33, 1, 7, 0], src=src, cache=cache, order=order, interleaved=interleaved, dim=128, rot=96)
    check_append([33, 1, 70], [1, 1, 1], src=src, cache=cache, order=order, interleaved=interleaved, single=True)
    check_append([33, 1, 70], [1, 1, 1], src=src, cache=cache, rot=0)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (40, 40), (64, 8), (71, 1), (130, 13)])
def test_heads(heads, kv_heads):
    check_append([9, 30], [2, 3], heads=heads, kv_heads=kv_heads, dim=48, seed=heads)


@pytest.mark.parametrize("page", [1, 2, 8, 64, 512])
def test_pages(page):
    check_append([130, 1, 65], [67, 1, 65], page=page)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_more_than_the_caches_hold(src, cache, interleaved):
    """Over 32 MB of results, which are written another way."""
    check_append([280, 9, 3], [270, 2, 1], heads=128, kv_heads=128, dim=256, rot=224, src=src, cache=cache, interleaved=interleaved)


def test_positions_far_out():
    pos = [0, 1, 4095, 131071, 10 ** 6, 10 ** 6 + 1, 2 ** 31 - 1, -1, -7, 12345678]
    for interleaved in (False, True):
        check_append([40], [10], dim=128, base=500000.0, pos=pos, interleaved=interleaved)


def test_scale_of_the_rotation():
    check_append([40], [10], scale=1.2079, dim=128)


def test_only_q_and_only_kv():
    assert not check_append([40, 3], [10, 2], with_kv=False).any()
    assert check_append([40, 3], [10, 2], with_q=False).sum() == 12


def test_places_that_are_not_there():
    # before the start of the cache, in a hole, behind the table's end
    assert check_append([4, 0, -2], [9, 1, 2]).sum() == 4
    assert check_append([40], [40], holes=[(0, 1, -1)]).sum() == 24
    assert check_append([40], [40], holes=[(0, 0, 10 ** 6), (0, 2, 2 ** 31 - 1)]).sum() == 16
    assert check_append([100], [60], width=4).sum() == 24


def test_e4m3_is_limited_and_nan_stays():
    for size in (1e4, 1e30):
        check_append([20], [20], cache="e4m3", size=size, rot=0)
    k = torch.full((1, 1, 16), float("nan"), device=DEV)
    v = torch.tensor([math.inf, -math.inf, 448, 449, 464, 465, 1e38, -500, 0.0, -0.0, 2.0 ** -10, 2.0 ** -9, 2.0 ** -9 * 1.5, 2.0 ** -11, -3e38, 1.0625], device=DEV)
    pool = torch.zeros((2, 1, 16, 1, 16), dtype=torch.uint8, device=DEV)
    ecfa.ecfa_append(ecfa.Cache(pool[0], pool[1]), ecfa.Batch(i32([[0]]), i32([1])), k, v.view(1, 1, 16))
    got = ref.E4M3[pool.cpu().numpy()][:, 0, 0, 0]
    assert np.isnan(got[0]).all()
    assert got[1].tolist() == [448, -448, 448, 448, 448, 448, 448, -448, 0, 0, 0, 2.0 ** -9, 2.0 ** -8, 0, -448, 1.0]
    assert pool[1, 0, 0, 0, 9] == 0x80


def test_q_in_place_and_strided_rows():
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((7, 3, 6, 80), generator=g).bfloat16().to(DEV)          # q, k, v of a fused projection, heads apart
    want = ref.turned(wide[:, 0, :4, 16:].cpu().double().numpy(), list(range(13, 20)), freqs(64), 64, False)
    pool = torch.zeros((2, 2, 16, 4, 64), dtype=torch.bfloat16, device=DEV)
    q, k, v = wide[:, 0, :4, 16:], wide[:, 1, :4, 16:], wide[:, 2, 1:5, 16:]
    b = ecfa.Batch(i32([[1, 0]]), i32([20]), i32([0, 7]), n_tokens=7)
    kept = wide.clone()
    ecfa.ecfa_append(ecfa.Cache(pool[0], pool[1]), b, k, v, q, q, ecfa.Rope(torch.tensor(freqs(64), device=DEV)))
    torch.cuda.synchronize()
    assert ref.near_bf16(q.cpu().double().numpy(), want, 10.0).all()
    assert torch.equal(wide[:, 1:], kept[:, 1:]) and torch.equal(wide[:, 0, 4:], kept[:, 0, 4:]) and torch.equal(wide[:, 0, :4, :16], kept[:, 0, :4, :16])
    assert torch.equal(pool[1].view(32, 4, 64)[[29, 30, 31, 0, 1, 2, 3]], v)


def test_many_sequences():
    for n in (63, 64, 65, 200, 4097):
        qn = [(i * 7) % 4 for i in range(n)]
        check_append([q + i % 5 for i, q in enumerate(qn)], qn, heads=1, kv_heads=1, dim=16, page=8)


@pytest.mark.parametrize("kind", ["plain", "linear", "base", "ramp"])
def test_frequencies(kind):
    rot, base, factor, orig = 64, 10000.0, 4.0, 2048.0
    got, scale = ecfa.rope_freq(rot, base, {"plain": 0, "linear": 1, "base": 2, "ramp": 3}[kind], factor, orig, 32.0, 1.0, device="cpu")
    got = got.double().numpy() / 2.0 ** 64 * 2 * math.pi
    j = np.arange(rot // 2)
    want = base ** (-2.0 * j / rot)
    if kind == "linear":
        want = want / factor
    if kind == "base":
        want = (base * factor ** (rot / (rot - 2))) ** (-2.0 * j / rot)
        assert want[0] == 1 and abs(want[-1] / (base ** (-2.0 * j[-1] / rot) / factor) - 1) < 1e-12
    if kind == "ramp":
        turns = orig * want / (2 * math.pi)
        assert np.allclose(got[turns > 40], want[turns > 40]) and np.allclose(got[turns < 0.9], want[turns < 0.9] / factor)
        assert (np.diff(got) < 0).all() and ((got <= want * (1 + 1e-9)) & (got >= want / factor * (1 - 1e-9))).all()
        assert abs(scale - (1 + 0.1 * math.log(factor))) < 1e-6
    else:
        assert np.allclose(got, want, rtol=1e-12) and scale == 1.0


def check_quant(x, group):
    q, scale = ecfa.ecfa_quant(x, group)
    torch.cuda.synchronize()
    q, scale, x = ref.E4M3[q.view(torch.uint8).cpu().numpy()], scale.cpu().double().numpy(), x.cpu().double().numpy()
    rows, cols = x.shape
    parts = x.reshape(rows, -1, 128) if group else x[:, None, :]
    most = np.maximum(np.abs(parts).max(-1), 2.0 ** -100)
    scale = scale.reshape(most.shape)
    assert (np.abs(scale - most / 448) <= 2.0 ** -23 * most / 448).all()
    held = parts * (448 / most)[..., None]
    q = q.reshape(parts.shape)
    assert (np.abs(q - held) <= np.maximum(2.0 ** -4 * np.abs(held), 2.0 ** -10) * (1 + 1e-6)).all()
    assert (np.abs(q).max(-1)[most > 2.0 ** -100] == 448).all()


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 1024), (3, 1040), (5, 128), (2, 4096), (7, 8192), (3, 8208), (2, 32768), (1, 65536 + 16), (1, 1 << 20), (1000, 48), (4099, 256)])
def test_rows_to_e4m3(rows, cols, src):
    g = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn((rows, cols), generator=g) * torch.exp(3 * torch.randn((rows, 1), generator=g))).to(src).to(DEV)
    check_quant(x, 0)
    if cols % 128 == 0:
        check_quant(x, 128)


def test_rows_to_e4m3_strides_and_sizes():
    x = torch.randn((9, 640), device=DEV)
    check_quant(x[:, 64:576], 0)
    check_quant(x[::2, :512], 128)
    check_quant(torch.randn((1, 384), device=DEV).expand(5, 384), 128)
    for size in (2.0 ** -126, 2.0 ** -110, 1e-20, 1e30, 1e38):
        y = torch.rand((3, 256), device=DEV) * 2 - 1
        y[:, ::128] = 1
        if size >= 2.0 ** -99:
            check_quant(y * size, 0)
            check_quant(y * size, 128)
    # below 2^-100 the largest number counts as 2^-100: a row of zeros has a scale all the same
    for tiny in (0.0, 2.0 ** -126, 2.0 ** -110, 2.0 ** -101):
        q, s = ecfa.ecfa_quant(torch.full((2, 128), tiny, device=DEV))
        assert (s.cpu().double() - 2.0 ** -100 / 448).abs().max() <= 2.0 ** -123 / 448
        held = 448 * tiny * 2.0 ** 100
        assert (np.abs(ref.E4M3[q.view(torch.uint8).cpu().numpy()] - held) <= max(2.0 ** -4 * held, 2.0 ** -10)).all()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_a_row_that_is_not_finite_says_so(group, what):
    x = torch.randn((3, 256), device=DEV)
    x[1, 200] = what
    q, s = ecfa.ecfa_quant(x, group)
    s = s.cpu()
    bad = s[1] if group == 0 else s[1, 1]
    assert torch.isnan(bad) if what != what else bad == math.inf
    fine = torch.ones_like(s, dtype=torch.bool)
    fine[(1, 1) if group else 1] = False
    assert torch.isfinite(s[fine]).all()
    check_quant(x[[0, 2]].contiguous(), group)


def test_rows_of_nothing():
    q, s = ecfa.ecfa_quant(torch.empty((0, 256), device=DEV))
    assert q.shape == (0, 256) and s.shape == (0,)


def test_refusals_on_the_device_side_of_the_binding():
    x = torch.randn((4, 256), device=DEV)
    for bad in (dict(group=64), dict(q=torch.empty((4, 128), dtype=torch.uint8, device=DEV)), dict(scale=torch.empty((3,), device=DEV))):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.ecfa_quant(x, **bad)
    for bad in (x.half(), x.t(), x[:, 1:], x[:, :200]):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.ecfa_quant(bad)


def e4m3_bytes(y):
    """fp32 numbers as E4M3 bytes, limited to 448, to the nearest, ties to the even byte."""
    value = ref.E4M3[:127]
    y = y.astype(np.float64)
    size = np.minimum(np.abs(y), 448.0)
    between = (value[1:] + value[:-1]) / 2
    below = np.searchsorted(between, size, side="left")          # between[below - 1] < size <= between[below]
    tie = (below < 126) & (size == between[np.minimum(below, 125)])
    return np.where(tie & (below % 2 == 1), below + 1, below).astype(np.uint8) | np.where(np.signbit(y), 128, 0).astype(np.uint8)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
def test_e4m3_is_of_the_quotient_by_the_scale(src):
    """Numbers whose quotient by the scale is a tie of E4M3, and their neighbours, by scales that are no powers of two; and scales that have no
    reciprocal in fp32, denormals among them: the bytes are those of the fp32 quotient."""
    value = ref.E4M3[:127]
    ties = np.concatenate([(value[1:] + value[:-1]) / 2, [0.0, 448.0, 464.0]])
    scales = np.array([0.0123, 0.3, 7.7, 1.0 / 3.0, 2.0 ** -128, 2.0 ** -129 * 1.25, 1e-42, 1e-30, 2.0 ** -90 * 1.1, 2.0 ** -90 * 0.9, 8e26, 2.0 ** 90 * 1.7], dtype=np.float32)
    near = []
    for by in scales:
        x = (ties * float(by)).astype(np.float32)
        if src == torch.bfloat16:
            x = torch.from_numpy(x).bfloat16().float().numpy()
        else:
            bits = np.minimum(x.view(np.int32)[:, None] + np.arange(-4, 5, dtype=np.int32), 0x7f000000)
            x = np.maximum(bits, 0).view(np.float32).ravel()
        near.append(np.concatenate([x, -x]))
    near = np.stack(near)                                        # (heads, numbers)
    near = np.pad(near, ((0, 0), (0, -near.shape[1] % 128))).reshape(len(scales), -1, 128).transpose(1, 0, 2).copy()
    n = near.shape[0]
    want = e4m3_bytes(np.divide(near, scales[:, None], dtype=np.float32))
    if src == torch.float32:                                     # (what a reciprocal would give is something else)
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            other = near * (np.float32(1) / scales)[:, None]
        assert (e4m3_bytes(np.nan_to_num(other)) != want).sum() > 100
    x = torch.from_numpy(near).to(src).to(DEV)
    pool = torch.zeros((2, -(-n // 16), 16, len(scales), 128), dtype=torch.uint8, device=DEV)
    by = torch.from_numpy(scales).to(DEV)
    b = ecfa.Batch(torch.arange(pool.shape[1], dtype=torch.int32, device=DEV)[None], i32([n]), i32([0, n]), n_tokens=n)
    ecfa.ecfa_append(ecfa.Cache(pool[0], pool[1], by, by), b, x, -x)
    got = pool.view(2, -1, len(scales), 128)[:, :n].cpu().numpy()
    assert np.array_equal(got[0], want) and np.array_equal(got[1], want ^ 128)


def test_refusals_of_tensors_on_the_host_and_of_wrong_shapes(monkeypatch):
    """Every tensor of a call in turn left on the host, or of a shape or type that does not fit: refused before the library hears of it."""
    def reached(*a):
        raise AssertionError("reached the library")

    for name in ("_append", "_attend", "_quant"):
        monkeypatch.setattr(ecfa, name, reached)
    t = lambda *s, d=torch.bfloat16, on=DEV: torch.zeros(s, dtype=d, device=on)  # noqa: E731
    n32 = lambda *s, on=DEV: t(*s, d=torch.int32, on=on)  # noqa: E731
    f32 = lambda *s, on=DEV: t(*s, d=torch.float32, on=on)  # noqa: E731
    pool, table, host = t(2, 2, 16, 2, 64), n32(2, 4), torch.device("cpu")
    rope = lambda on=DEV, pos=None: ecfa.Rope(t(32, d=torch.int64, on=on), pos=pos)  # noqa: E731
    c, b, k, q = ecfa.Cache(pool[0], pool[1]), ecfa.Batch(table, n32(2)), t(2, 2, 64), t(2, 4, 64)
    away = ecfa.Batch(table.cpu(), n32(2, on=host))
    attend = lambda **m: ecfa.ecfa_attend(c, b, **{**dict(q=q, out=q, workspace=t(1 << 20, d=torch.uint8)), **m})  # noqa: E731
    append = lambda **m: ecfa.ecfa_append(c, b, **{**dict(k=k, v=k, q=q, q_out=q), **m})  # noqa: E731
    bad = [lambda: ecfa.Cache(pool[0], pool[1].cpu()), lambda: ecfa.Cache(pool[0], pool[1], f32(2, on=host)), lambda: ecfa.Cache(pool[0], pool[1], None, f32(2, on=host)),
           lambda: ecfa.Batch(table, n32(2, on=host)), lambda: ecfa.Batch(table.cpu(), n32(2)), lambda: ecfa.Batch(table, n32(2), n32(3, on=host), 2), lambda: rope(pos=n32(2, on=host)),
           lambda: ecfa.ecfa_attend(c, away, q), lambda: ecfa.ecfa_append(c, away, k, k), lambda: ecfa.ecfa_attend(ecfa.Cache(pool[0].cpu(), pool[1].cpu()), b, q),
           lambda: append(rope=rope(host)), lambda: append(rope=rope(pos=n32(3)))]
    bad += [lambda m=m: attend(**m) for m in (dict(q=q.cpu()), dict(out=q.cpu()), dict(workspace=t(1 << 20, d=torch.uint8, on=host)), dict(slopes=f32(4, on=host)),
                                              dict(prefix=n32(2, on=host)), dict(workspace=t(16, d=torch.uint8).expand(1 << 16, 16)), dict(slopes=f32(3)), dict(prefix=n32(3)),
                                              dict(out=t(2, 2, 64)), dict(q=t(3, 4, 64)), dict(q=t(2, 4, 32)), dict(q=t(2, 256)), dict(q=t(2, 4, 64, d=torch.float16)),
                                              dict(q=t(2, 64, 4).transpose(1, 2)))]
    bad += [lambda m=m: append(**m) for m in (dict(k=k.cpu()), dict(v=k.cpu()), dict(q=q.cpu()), dict(q_out=q.cpu()), dict(k=t(2, 4, 64)), dict(q_out=t(2, 2, 64)), dict(q=None))]
    x, x8, sc = t(4, 256), t(4, 256, d=torch.uint8), f32(4)
    bad += [lambda: ecfa.ecfa_quant(x.cpu()), lambda: ecfa.ecfa_quant(x, q=x8.cpu()), lambda: ecfa.ecfa_quant(x, scale=sc.cpu()), lambda: ecfa.ecfa_quant(x, 128, x8, sc)]
    for i, call in enumerate(bad):
        with pytest.raises(ecf8.Ecf8Error) as e:
            call()
        assert e.value.code == ecf8.E_ARG, i


def test_bf16_is_of_the_quotient_by_the_scale():
    """A cache of BF16 with scales: the fp32 quotient, rounded once."""
    g = torch.Generator().manual_seed(4)
    scales = torch.tensor([0.0123, 0.3, 7.7, 1.0 / 3.0, 2.0 ** -100, 2.0 ** 100, 1e-30, 1e20])
    x = torch.randn((300, 8, 64), generator=g) * scales[:, None].clamp(2.0 ** -90, 2.0 ** 90)
    x[0, :, :4] = torch.tensor([0.0, -0.0, math.inf, -math.inf])
    pool = torch.zeros((2, 19, 16, 8, 64), dtype=torch.bfloat16, device=DEV)
    by = scales.to(DEV)
    b = ecfa.Batch(torch.arange(19, dtype=torch.int32, device=DEV)[None], i32([300]), i32([0, 300]), n_tokens=300)
    ecfa.ecfa_append(ecfa.Cache(pool[0], pool[1], by, by), b, x.to(DEV), -x.to(DEV))
    want = (x / scales[:, None]).bfloat16().view(torch.int16)
    got = pool.view(2, -1, 8, 64)[:, :300].cpu().view(torch.int16)
    assert torch.equal(got[0], want) and torch.equal(got[1], want ^ -32768)
