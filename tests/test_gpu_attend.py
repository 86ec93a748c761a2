"""ecfa_attend against the definition in 64 bits: lengths from nothing to past a step and past a split, heads shared and not, head sizes
that fill no register, pages that end inside a step, both cache types and both orders, masks that leave rows without a key, what is
stored in places that nobody sees, hints that are wrong, other streams, graphs, and pools that 32 bits cannot address."""
import itertools

import numpy as np
import pytest
import torch

import attention_reference as ref
from paper_2510_02676_amd import ecf8, ecfa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Setting:
    """A pool, a table in no order and a batch; `kv` and `qn` a length each per sequence."""

    def __init__(self, kv, qn, heads=8, kv_heads=2, dim=128, page=16, cache="bf16", order="token", seed=0, holes=(), width=None, single=False, scales=True,
                 hints=True):
        g = torch.Generator().manual_seed(seed)
        self.page, self.kv, self.qn, self.heads = page, kv, qn, heads
        need = [-(-max(0, n) // page) for n in kv]
        width = max(max(need), 1) if width is None else width
        pages = sum(need) + 2
        ids = torch.randperm(pages, generator=g).tolist()
        self.table = [[-1] * width for _ in kv]
        for s, n in enumerate(need):
            for j in range(min(n, width)):
                self.table[s][j] = ids.pop()
        for s, j, what in holes:
            self.table[s][j] = what
        self.q_start = [0] + list(itertools.accumulate(qn))
        k, v = (torch.randn((pages, page, kv_heads, dim), generator=g) for _ in range(2))
        self.k_scale = self.v_scale = None
        if cache == "e4m3":
            if scales:
                self.k_scale, self.v_scale = (torch.rand(kv_heads, generator=g) * 0.02 + 0.005 for _ in range(2))
                k, v = k / self.k_scale[:, None], v / self.v_scale[:, None]
            k, v = (x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
        else:
            k, v = k.bfloat16(), v.bfloat16()
        if order == "head":
            k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
        self.k, self.v, self.pages = k, v, pages
        self.q = (torch.randn((self.q_start[-1], heads, dim), generator=g) * 2).bfloat16()
        self.single, self.hints = single, hints

    def batch(self, **more):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        hints = dict(max_q=max(self.qn), max_kv=max(max(self.kv), 1)) if self.hints else {}
        return ecfa.Batch(i32(self.table), i32(self.kv), None if self.single else i32(self.q_start), n_tokens=self.q_start[-1], **{**hints, **more})

    def device_cache(self):
        up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        k, v = (torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=DEV).copy_(x) for x in (self.k, self.v))
        return ecfa.Cache(k, v, up(self.k_scale), up(self.v_scale))

    def run(self, **opts):
        q = self.q.to(DEV)
        out = torch.full((q.shape[0] + 2, *q.shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV)
        ecfa.ecfa_attend(self.device_cache(), self.batch(), q, out=out[1:-1], **opts)
        torch.cuda.synchronize()
        assert torch.isnan(out[0]).all() and torch.isnan(out[-1]).all()
        return out[1:-1].cpu().double().numpy()

    def want(self, scale=None, causal=True, window=0, softcap=0.0, slopes=None, prefix=None):
        toks = ref.tokens(self.q_start, self.kv, self.table, self.page, self.pages)
        return ref.attend(self.q, ref.values(self.k, self.k_scale), ref.values(self.v, self.v_scale), toks, self.q.shape[2] ** -0.5 if scale is None else scale,
                          causal, window, softcap, None if slopes is None else slopes.cpu().numpy(), None if prefix is None else prefix.tolist())


def check(setting, **opts):
    got = setting.run(**opts)
    want, size = setting.want(**opts)
    bad = ~(np.abs(got - want) <= ref.attend_bound(want, size))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(got - want).max()))
    return got, want


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 160, 192, 256])
def test_head_sizes(dim, cache):
    check(Setting([37, 5], [3, 2], dim=dim, cache=cache, seed=dim))
    check(Setting([70, 5], [30, 5], heads=4, kv_heads=1, dim=dim, cache=cache, seed=dim))


@pytest.mark.parametrize("kv", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700, 1500])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_single_tokens(kv, cache):
    check(Setting([kv, max(0, kv - 1), 3], [1, 1, 1], cache=cache, single=True, seed=kv))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 40, 63, 65, 129, 200])
@pytest.mark.parametrize("more", [0, 1, 77])
def test_chunks(n, more):
    check(Setting([n + more, 40, 0], [n, 1, 0], cache="e4m3" if n % 2 else "bf16", seed=n))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (5, 5), (15, 5), (16, 1), (17, 1), (32, 2), (33, 1), (71, 1), (12, 12), (128, 1)])
@pytest.mark.parametrize("qn", [1, 6, 45])
def test_heads_shared_and_not(heads, kv_heads, qn):
    check(Setting([60, 9], [qn, 2], heads=heads, kv_heads=kv_heads, dim=64, seed=heads))


@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 128, 256])
@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_pages(page, order, cache):
    check(Setting([1, 150, 33], [1, 21, 2], page=page, order=order, cache=cache, heads=4, seed=page))
    check(Setting([1, 150, 300], [1, 1, 1], page=page, order=order, cache=cache, single=True, seed=page))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("qn,kv", [([1, 1, 1], [90, 1, 200]), ([40, 1, 13], [90, 7, 200]), ([130, 3, 66], [140, 3, 300])])
def test_masks_and_scores(qn, kv, cache):
    make = lambda: Setting(kv, qn, cache=cache, seed=sum(kv))  # noqa: E731
    slopes = 2.0 ** -torch.arange(1, 9, dtype=torch.float32, device=DEV)
    prefix = torch.tensor([60, 0, 1000], dtype=torch.int32, device=DEV)
    check(make(), causal=False)
    for window in (1, 7, 32, 33, 64, 1000, 2 ** 32 - 1):
        check(make(), window=window)
        check(make(), window=window, causal=False)
    check(make(), softcap=2.0)
    check(make(), softcap=50.0, scale=0.3)
    check(make(), slopes=slopes)
    check(make(), slopes=slopes, causal=False, softcap=5.0)
    check(make(), prefix=prefix)
    check(make(), prefix=prefix, slopes=slopes, softcap=5.0)


def test_rows_without_a_key_are_zeros():
    # more new tokens than the cache holds: the first ones come before every key; and sequences of nothing
    s = Setting([5, 0, 2, -3], [9, 3, 1, 2])
    got, want = check(s)
    assert not got[:4].any() and not got[9:12].any() and not got[13:].any() and got[4:9].any()
    # all pages of a sequence are holes
    s = Setting([40, 40], [2, 2], holes=[(0, j, -1) for j in range(3)])
    got, _ = check(s)
    assert not got[:2].any() and got[2:].any()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_holes_and_pages_that_are_none(cache):
    s = Setting([200, 100], [30, 1], cache=cache, holes=[(0, 1, -1), (0, 4, 10 ** 6), (0, 12, -2 ** 31), (1, 0, 2 ** 31 - 1)])
    check(s)
    check(s, causal=False)
    # a table that is narrower than the sequence: what it does not name is not seen
    check(Setting([200, 100], [30, 1], cache=cache, width=5))


def poison(s, where, what):
    """Puts `what` into V and K of one key of a sequence."""
    seq, key = where
    p, at = s.table[seq][key // s.page], key % s.page
    for x in (s.k, s.v):
        if x.dtype == torch.uint8:
            x[p, at] = 0x7F
        else:
            x[p, at] = what


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("qn", [1, 3, 20, 70])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_does_not_matter(cache, qn, what):
    """NaN and infinities behind the end of a sequence, before a window, and in keys that only later tokens see; tokens that do see them
    get what the definition says."""
    s = Setting([85, 85], [qn, qn], cache=cache, seed=5)
    clean = s.run()
    for page in range(s.pages):                                 # everything that belongs to nobody
        for at in range(s.page):
            if not any(t[j // s.page] == page and j % s.page == at for t in s.table for j in range(85)):
                s.k[page, at] = 0x7F if cache == "e4m3" else what
                s.v[page, at] = 0xFF if cache == "e4m3" else what
    assert np.array_equal(s.run(), clean)
    check(s)
    # the newest key of sequence 0: only its last token sees it; the others' sums may be made in another order
    want, size = s.want()
    poison(s, (0, 84), what)
    got = s.run()
    assert np.array_equal(got[qn:], clean[qn:]) and np.isnan(got[qn - 1]).all()
    assert (np.abs(got - want) <= ref.attend_bound(want, size))[:qn - 1].all()
    # an old key of sequence 1, outside of everybody's window
    s = Setting([85, 85], [qn, qn], cache=cache, seed=5)
    clean = s.run(window=10)
    poison(s, (1, 85 - qn - 10), what)
    assert np.array_equal(s.run(window=10), clean)
    # in a value alone, where the weights are finite: an infinity reaches the tokens that see it, in its element
    if cache == "bf16":
        s = Setting([85, 85], [qn, qn], cache=cache, seed=5)
        key = 85 - (qn + 1) // 2
        s.v[s.table[0][key // s.page], key % s.page, 1, 9] = what
        want, size = s.want()
        got = s.run()
        hit = np.zeros(got.shape, dtype=bool)
        hit[qn - (85 - key):qn, 4:, 9] = True
        assert (np.abs(got - want) <= ref.attend_bound(want, size))[~hit].all()
        assert (np.isnan(got[hit]) if what != what else got[hit] == what).all()


def test_large_scores():
    """Weights of one key against all others, and scores far below the rest, in and out of the first step."""
    s = Setting([300, 40], [5, 1], heads=2, kv_heads=1, dim=64)
    s.q *= 40
    check(s)
    check(s, scale=1e-6)


def test_hints_do_not_change_what_is_computed():
    s = Setting([300, 40, 900], [45, 1, 2])
    want, size = s.want()
    cache, q = s.device_cache(), s.q.to(DEV)
    for max_q, max_kv in ((0, 0), (1, 1), (2, 64), (45, 900), (10 ** 6, 10 ** 6), (3, 10 ** 9)):
        b = s.batch(max_q=max_q, max_kv=max_kv)
        got = ecfa.ecfa_attend(cache, b, q)
        again = ecfa.ecfa_attend(cache, b, q)
        torch.cuda.synchronize()
        assert torch.equal(got, again)
        assert (np.abs(got.cpu().double().numpy() - want) <= ref.attend_bound(want, size)).all(), (max_q, max_kv)


def test_starts_that_are_wrong_stay_inside():
    """Starts beyond the rows, falling or negative ones: rows that belong to a sequence by them are written, no others."""
    s = Setting([60, 60], [4, 4])
    q, out = s.q.to(DEV), torch.full((10, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    for starts in ([0, 4, 1000], [-5, 4, 8], [6, 2, 8], [0, 2 ** 31 - 1, -2 ** 31], [8, 8, 8]):
        b = s.batch()
        b.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        ecfa.ecfa_attend(s.device_cache(), b, q, out=out[1:9])
        torch.cuda.synchronize()
        assert (out[0] == 7).all() and (out[9] == 7).all() and not torch.isnan(out).any()


def test_strides():
    """q and out as parts of wider rows, heads apart, and pools that are parts of larger ones."""
    s = Setting([75, 33], [9, 1], heads=4, kv_heads=2, dim=96)
    want, size = s.want()
    wide = torch.full((10, 3, 4, 112), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 1, :, 8:104] = s.q.to(DEV)
    q = wide[:, 1, :, 8:104]
    out = torch.zeros((4, 10, 104), dtype=torch.bfloat16, device=DEV).transpose(0, 1)[:, :, 8:]
    pool = torch.full((2, s.pages, 3, 16, 2, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    k, v = pool[0, :, 2, :, :, 16:112], pool[1, :, 0, :, :, 32:]
    k.copy_(s.k)
    v.copy_(s.v)
    ecfa.ecfa_attend(ecfa.Cache(k, v), s.batch(), q, out=out)
    torch.cuda.synchronize()
    assert (np.abs(out.cpu().double().numpy() - want) <= ref.attend_bound(want, size)).all()


def test_many_sequences():
    kv = [(i * 37) % 90 for i in range(150)]
    check(Setting(kv, [1] * 150, heads=2, kv_heads=1, dim=64, single=True))
    qn = [(i * 7) % 5 for i in range(150)]
    check(Setting([max(a, b) for a, b in zip(kv, qn)], qn, heads=2, kv_heads=1, dim=64))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_long_sequences(cache):
    """Past many splits; against 32-bit torch on the device in one piece, whose own error is far below the bound."""
    s = Setting([20011, 3], [1, 1], heads=8, kv_heads=2, cache=cache, single=True, page=64)
    s2 = Setting([6007, 3], [200, 1], heads=8, kv_heads=2, cache=cache, page=64)
    for x in (s, s2):
        got = x.run()
        k, v = (torch.from_numpy(ref.values(p, sc)).to(DEV) for p, sc in ((x.k, x.k_scale), (x.v, x.v_scale)))
        key = torch.arange(x.kv[0])
        slot = torch.tensor(x.table[0])[key // 64]
        k, v = k[slot, key % 64], v[slot, key % 64]              # (keys, kv_heads, dim), 64 bits
        for h in range(8):
            sc = x.q[:x.qn[0], h].to(DEV).double() @ k[:, h // 4].T * 128 ** -0.5
            place = torch.arange(x.kv[0] - x.qn[0], x.kv[0], device=DEV)
            sc.masked_fill_(key.to(DEV)[None, :] > place[:, None], -float("inf"))
            w = torch.softmax(sc, -1)
            want, size = (w @ v[:, h // 4]).cpu().numpy(), (w @ v[:, h // 4].abs()).cpu().numpy()
            assert (np.abs(got[:x.qn[0], h] - want) <= ref.attend_bound(want, size)).all()


def test_a_pool_beyond_32_bits():
    """Pages more than 2^32 bytes into the pool."""
    pages, page, heads, dim = 1 << 17, 32, 8, 128                # 8 GiB of keys and as much of values
    k = torch.empty((pages, page, heads, dim), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    s = Setting([90, 50], [1, 20], heads=16, kv_heads=8, dim=dim, page=page)
    far = {p: pages - 1 - 5000 * i for i, p in enumerate(sorted({p for t in s.table for p in t if p >= 0}))}
    for p, f in far.items():
        k[f].copy_(s.k[p])
        v[f].copy_(s.v[p])
    want, size = s.want()
    s.table = [[far.get(p, -1) for p in t] for t in s.table]
    got = ecfa.ecfa_attend(ecfa.Cache(k, v), s.batch(), s.q.to(DEV)).cpu().double().numpy()
    assert (np.abs(got - want) <= ref.attend_bound(want, size)).all()
    # and the same places written by append
    new = torch.randn((21, 8, dim), device=DEV)
    ecfa.ecfa_append(ecfa.Cache(k, v), s.batch(), new, -new)
    for t, (seq, place, slots) in enumerate(ref.tokens(s.q_start, s.kv, s.table, page, pages)):
        p, at = slots[place]
        assert torch.equal(k[p, at], new[t].bfloat16()) and torch.equal(v[p, at], -new[t].bfloat16())


def test_another_stream_and_a_shared_pool():
    s = Setting([400, 90], [1, 1], single=True)
    cache, b, q = s.device_cache(), s.batch(), s.q.to(DEV)
    want = ecfa.ecfa_attend(cache, b, q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(side):
            got = ecfa.ecfa_attend(cache, b, q)
        other = ecfa.ecfa_attend(cache, b, q, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(other, want)


def test_a_captured_step_follows_its_tensors():
    """Append, attend and quant in one graph; lengths, tables and inputs are rewritten between replays."""
    s = Setting([10, 300], [1, 1], single=True, width=40)
    used = {p for t in s.table for p in t}
    free = [p for p in range(s.pages) if p not in used]
    s.table[0][1] = free[0]                                      # room for the steps to come
    if s.table[1][19] < 0:
        s.table[1][19] = free[1]
    cache, b = s.device_cache(), s.batch()
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((2, h, 128), generator=g).to(DEV) for h in (8, 2, 2))
    rope = ecfa.Rope(ecfa.rope_freq(128)[0].to(DEV))
    work = ecfa.attend_workspace(cache, b, 8)
    turned, out = (torch.empty((2, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    e4, sc = torch.empty((2, 1024), dtype=torch.uint8, device=DEV), torch.empty((2,), device=DEV)

    def step(cache):
        ecfa.ecfa_append(cache, b, k, v, q, turned, rope)
        ecfa.ecfa_attend(cache, b, turned, out=out, workspace=work)
        ecfa.ecfa_quant(out.view(2, 1024), q=e4, scale=sc)

    step(cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g))
        b.kv_len.copy_(torch.tensor([10 + i, 300 + i], dtype=torch.int32))
        twin = ecfa.Cache(cache.k.clone(), cache.v.clone())
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (turned, out, e4, sc, cache.k, cache.v)]
        for x in (turned, out, e4, sc):
            x.zero_()
        step(twin)
        torch.cuda.synchronize()
        for a, c in zip(got, (turned, out, e4, sc, twin.k, twin.v)):
            assert torch.equal(a, c)


def test_a_workspace_that_is_too_small_or_missing():
    s = Setting([5000], [1], single=True)
    cache, b, q = s.device_cache(), s.batch(), s.q.to(DEV)
    out = torch.full_like(q, 5.0)
    work = ecfa.attend_workspace(cache, b, 8)
    with pytest.raises(ecf8.Ecf8Error) as e:
        ecfa.ecfa_attend(cache, b, q, out=out, workspace=work[:-4])
    assert e.value.code == ecf8.E_CAPACITY
    with pytest.raises(ecf8.Ecf8Error) as e:
        ecfa.ecfa_attend(cache, b, q, out=out, workspace=torch.empty(work.numel() + 16, dtype=torch.uint8, device=DEV)[8:])
    assert e.value.code == ecf8.E_ALIGN
    torch.cuda.synchronize()
    assert (out == 5).all()


@pytest.mark.parametrize("qn", [1, 4, 50])
def test_caps_and_slopes_of_any_size(qn):
    """Caps on both sides of where the limit's formula changes, scores far beyond them, slopes that leave a few keys."""
    for cap in (0.01, 1.0, 63.9, 64.0, 64.1, 1e4, 1e30):
        check(Setting([90, 30], [qn, 1], dim=64), softcap=cap)
        check(Setting([90, 30], [qn, 1], dim=64), softcap=cap, scale=7.0)
    slopes = torch.tensor([0.0, 1e-6, 0.5, 3.0, 40.0, 1e4, -0.01, 0.25], device=DEV)
    check(Setting([90, 30], [qn, 1], dim=64), slopes=slopes)
    check(Setting([90, 30], [qn, 1], dim=64), slopes=slopes, softcap=100.0, window=40)


@pytest.mark.parametrize("heads,kv_heads", [(20, 1), (40, 2), (4, 1), (66, 2)])
def test_chunks_and_single_tokens_together(heads, kv_heads):
    """Long and short sequences in one batch, cut into pieces and not; more than 32 heads to a key/value head have no short ones."""
    for kv, qn in (([700, 1100, 7, 0, 64], [90, 1, 1, 1, 3]), ([60, 5, 2000, 1], [33, 2, 1, 1])):
        check(Setting(kv, qn, heads=heads, kv_heads=kv_heads, dim=64, cache="e4m3" if heads == 4 else "bf16"))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_tokens_of_a_pool_far_apart(cache):
    """Tokens 2^25 bytes apart, the pages between one another's tokens: offsets within a page pass what 32 bits hold."""
    apart, heads, dim, page = 1 << (24 if cache == "bf16" else 25), 2, 64, 128
    s = Setting([75, 200, 33], [1, 20, 1], heads=4, kv_heads=heads, dim=dim, page=page, cache=cache)
    mem = torch.zeros(2 * (page - 1) * apart + 4 * s.pages * heads * dim, dtype=s.k.dtype, device=DEV)
    at = (heads * dim, 2 * apart, dim, 1)
    k, v = (torch.as_strided(mem, (s.pages, page, heads, dim), at, first) for first in (0, 2 * s.pages * heads * dim))
    k.copy_(s.k)
    v.copy_(s.v)
    want, size = s.want()
    b, q = s.batch(), s.q.to(DEV)
    c = ecfa.Cache(k, v, *(None if x is None else x.to(DEV) for x in (s.k_scale, s.v_scale)))
    got = ecfa.ecfa_attend(c, b, q).cpu().double().numpy()
    assert (np.abs(got - want) <= ref.attend_bound(want, size)).all()
    if cache == "bf16":                                          # and each token alone
        single = ecfa.Batch(b.page_table, b.kv_len)
        one = ecfa.ecfa_attend(c, single, q[[0, 20, 21]].contiguous()).cpu().double().numpy()
        assert (np.abs(one - want[[0, 20, 21]]) <= ref.attend_bound(want, size)[[0, 20, 21]]).all()


def test_more_sequences_than_are_cut_into_pieces():
    for n in (1024, 1025):
        kv = [(i * 37) % 150 for i in range(n - 1)] + [900]
        check(Setting(kv, [1] * n, heads=2, kv_heads=1, dim=32, single=True, page=32))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("qn", [1, 3, 40, 100])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_pieces_of_which_some_hold_nothing(cache, qn, what):
    """Long sequences cut in pieces: holes that take up a whole piece, windows that leave most of them out, NaN in places that are not seen."""
    s = Setting([2600, 1300], [qn, 1], heads=4, kv_heads=1, dim=64, cache=cache, holes=[(0, j, -1) for j in range(30, 100)], seed=qn)
    check(s)
    check(s, window=300)
    check(s, prefix=torch.tensor([2600, 5], dtype=torch.int32, device=DEV))
    clean, windowed = s.run(), s.run(window=300)
    poison(s, (0, 2600 - qn - 300), what)
    assert np.array_equal(s.run(window=300), windowed)
    poison(s, (0, 2599), what)                                   # seen by the last token alone
    got, (want, size) = s.run(window=300), s.want(window=300)
    assert np.isnan(got[qn - 1]).all() and np.array_equal(got[qn:], windowed[qn:])
    assert (np.abs(got - want) <= ref.attend_bound(want, size))[:qn - 1].all()
    assert np.array_equal(s.run()[qn:], clean[qn:])


def test_counts_that_a_launch_cannot_hold():
    one = torch.zeros((1, 1, 16), dtype=torch.bfloat16, device=DEV)
    pool = torch.zeros((2, 1, 16, 1, 16), dtype=torch.bfloat16, device=DEV)
    table, n = torch.zeros((1, 1), dtype=torch.int32, device=DEV), 1 << 21
    long = ecfa.Batch(table, torch.ones(1, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), n_tokens=n)
    q = one.expand(n, 1024, 16)
    with pytest.raises(ecf8.Ecf8Error) as e:                     # 2^31 rows to a key/value head
        ecfa.ecfa_attend(ecfa.Cache(pool[0], pool[1]), long, q, out=q)
    assert e.value.code == ecf8.E_ARG
    heads = torch.zeros((2, 1, 16, 64, 16), dtype=torch.bfloat16, device=DEV)
    many = ecfa.Batch(table.expand(n, 1), torch.ones(n, dtype=torch.int32, device=DEV))
    q = one.expand(n, 64, 16)
    with pytest.raises(ecf8.Ecf8Error) as e:                     # 2^27 workgroups
        ecfa.ecfa_attend(ecfa.Cache(heads[0], heads[1]), many, q, out=q)
    assert e.value.code == ecf8.E_ARG


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("kv,qn", [([3, 400], [200, 200]), ([3, 3000], [200, 200]), ([3, 420, 7, 300, 90], [130, 260, 1, 2, 70]), ([3, 2600, 1, 1900], [260, 50, 1, 40])])
def test_rows_before_the_first_sequence(cache, kv, qn):
    """Starts that begin above 0: the rows before them belong to nobody, whole tiles of them; keys cut in pieces and not, with single tokens and
    without."""
    s = Setting(kv, qn, cache=cache, seed=len(kv))
    want, size = s.want()
    whole = s.batch()
    b = ecfa.Batch(whole.page_table[1:], whole.kv_len[1:].contiguous(), whole.q_start[1:].contiguous(), n_tokens=s.q_start[-1], max_q=max(qn[1:]), max_kv=max(kv))
    q = s.q.to(DEV)
    out = torch.full((q.shape[0] + 2, *q.shape[1:]), 7.0, dtype=torch.bfloat16, device=DEV)
    ecfa.ecfa_attend(s.device_cache(), b, q, out=out[1:-1])
    torch.cuda.synchronize()
    got, first = out.cpu().double().numpy(), qn[0]
    assert (got[:first + 1] == 7).all() and (got[-1] == 7).all()
    assert (np.abs(got[1:-1] - want) <= ref.attend_bound(want, size))[first:].all()


@pytest.mark.parametrize("max_kv", [400, 3000])
def test_starts_that_are_wrong_stay_inside_with_many_rows(max_kv):
    s = Setting([max_kv, 300, 40], [200, 100, 100], heads=16, kv_heads=2)
    q, out = s.q.to(DEV), torch.full((402, 16, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    for starts in ([200, 400, 400, 400], [399, 400, 1000, 2000], [-5, 200, 300, 400], [300, 100, 400, 50], [0, 2 ** 30, -2 ** 30, 400], [2 ** 31 - 1, 0, 400, 400], [128, 64, 32, 0]):
        b = s.batch()
        b.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        ecfa.ecfa_attend(s.device_cache(), b, q, out=out[1:401])
        torch.cuda.synchronize()
        assert (out[0] == 7).all() and (out[401] == 7).all()


def test_memory_of_a_call_on_another_stream(monkeypatch):
    """What a call allocates for another stream is no block that the current stream has just let go, whose kernels may still be using it."""
    s = Setting([5000], [1], single=True)
    cache, b, q = s.device_cache(), s.batch(), s.q.to(DEV)
    k, v = (torch.zeros((1, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    side, given, attend = torch.cuda.Stream(), [], ecfa._attend
    monkeypatch.setattr(ecfa, "_attend", lambda *a: given.append(a[5]) or attend(*a))
    x = torch.randn((4, 1024), device=DEV)
    torch.cuda.synchronize()
    for call in (lambda stream: ecfa.ecfa_attend(cache, b, q, stream=stream), lambda stream: ecfa.ecfa_append(cache, b, k, v, q, stream=stream),
                 lambda stream: ecfa.ecfa_quant(x, stream=stream), lambda stream: ecfa.ecfa_quant(x, 128, stream=stream)):
        for _ in range(3):
            given.clear()
            mine = call(None)
            held = {y.data_ptr() for y in (mine if isinstance(mine, tuple) else (mine,))} | {p for p in given if p}
            given.clear()
            del mine
            other = call(side)
            got = {y.data_ptr() for y in (other if isinstance(other, tuple) else (other,))} | {p for p in given if p}
            assert not held & got
            torch.cuda.synchronize()


def test_calls_in_flight_on_two_streams():
    """Unlike inputs, no buffers given: each gets its own result, whichever runs first."""
    made = [(Setting([5000 + 64 * i], [1], single=True, seed=i), ) for i in range(4)]
    made = [(s.device_cache(), s.batch(), s.q.to(DEV)) for s, in made]
    want = [ecfa.ecfa_attend(*m) for m in made]
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    for _ in range(5):
        busy @ busy                                              # what is queued here comes later than what is queued there
        got = [ecfa.ecfa_attend(*m, stream=side if i % 2 else None) for i, m in enumerate(made * 3)]
        torch.cuda.synchronize()
        for i, y in enumerate(got):
            assert torch.equal(y, want[i % 4])


def test_strides_that_lead_nowhere():
    """One token, one head, one page, one token to a page: what the stride to the next would be does not matter."""
    s = Setting([70], [1], heads=1, kv_heads=1, dim=64, page=1, single=True)
    want, size = s.want()
    odd = lambda x, i, by: torch.as_strided(x, x.shape, [by if j == i else n for j, n in enumerate(x.stride())])  # noqa: E731
    q, out = s.q.to(DEV), torch.zeros((1, 1, 64), dtype=torch.bfloat16, device=DEV)
    cache = ecfa.Cache(odd(odd(s.k.to(DEV), 1, 7), 2, 3), odd(odd(s.v.to(DEV), 1, 5), 2, 9))
    got = ecfa.ecfa_attend(cache, s.batch(), odd(odd(q, 0, 5), 1, 3), out=odd(odd(out, 0, 1), 1, 11))
    assert (np.abs(got.cpu().double().numpy() - want) <= ref.attend_bound(want, size)).all()
    x = torch.randn((1, 256), device=DEV)
    for group in (0, 128):
        a, b = ecfa.ecfa_quant(x, group), ecfa.ecfa_quant(odd(x, 0, 3), group)
        assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("qn", [1, 4, 50])
@pytest.mark.parametrize("cap", [1e-45, 1e-40, 2.0 ** -127, 2.0 ** -99, 2.0 ** 99, 2.0 ** 101, 2.0 ** 127, 3.4e38])
def test_caps_at_the_ends_of_fp32(cap, qn):
    """Caps without a reciprocal in fp32 make all scores alike; caps that log2(e) times them overflows change none.  A score of 0 stays one."""
    s = Setting([90, 30], [qn, 1], dim=64)
    s.q[:, 3] = 0
    check(s, softcap=cap)
    s = Setting([90, 30], [qn, 1], dim=64, cache="e4m3")
    check(s, softcap=cap, scale=3.0)


@pytest.mark.parametrize("qn", [1, 4, 50])
def test_scales_at_the_ends_of_fp32(qn):
    """Scales so small that the scores vanish, masked keys beside them; the largest scale, with dot products of 0."""
    for scale in (1e-45, 1e-40):
        check(Setting([90, 30], [qn, 1], dim=64), scale=scale)
    s = Setting([90, 30], [qn, 1], dim=64)
    s.q[:] = 0
    check(s, scale=3.4e38)
    s = Setting([90, 30], [qn, 1], dim=64, cache="e4m3")
    s.k_scale = torch.tensor([1e-45, 2e-45])
    check(s)
    check(s, window=20, softcap=3.0)


def test_windows_that_32_bits_would_change():
    """-1 would be all keys, 2^32 + 5 five of them."""
    s = Setting([60], [1], single=True)
    cache, b, q = s.device_cache(), s.batch(), s.q.to(DEV)
    for window in (-1, 1 << 32, (1 << 32) + 5):
        with pytest.raises(ecf8.Ecf8Error) as e:
            ecfa.ecfa_attend(cache, b, q, window=window)
        assert e.value.code == ecf8.E_ARG


@pytest.mark.parametrize("kv,qn", [([90, 700], [1, 1]), ([90, 700], [50, 3])])
def test_a_bf16_cache_with_scales(kv, qn):
    """Scales that are powers of two: bit for bit what keys and values that much larger give."""
    s = Setting(kv, qn, seed=9)
    plain, q, k, v = s.device_cache(), s.q.to(DEV), torch.tensor([0.25, 2.0], device=DEV), torch.tensor([4.0, 0.5], device=DEV)
    larger = ecfa.Cache(plain.k * k[:, None].bfloat16(), plain.v * v[:, None].bfloat16())
    for more in (dict(), dict(softcap=20.0, window=60)):
        got = ecfa.ecfa_attend(ecfa.Cache(plain.k, plain.v, k, v), s.batch(), q, **more)
        assert torch.equal(got, ecfa.ecfa_attend(larger, s.batch(), q, **more))
