"""Every key is counted once.  With q = 0 all weights are equal; key j has a one in one element of one key/value head and zeros
elsewhere, so that an element of the result is the number of its keys that the token sees, over the number of all of them: a key
that is lost or taken twice at the border of a step, a wave, a piece or a tile moves it by one whole, whatever the length."""
import itertools
import math
import random

import pytest
import torch

from paper_2510_02676_amd import ecfa

gpu = pytest.mark.gpu
DEV = "cuda:0"


def seen_by(kv, qn, causal, window, prefix):
    """[lo, hi) of the keys that each new token of a sequence sees."""
    places = range(kv - qn, kv)
    return [(max(0, p + 1 - window) if window else 0, min(kv, max(p + 1, prefix)) if causal else kv) for p in places]


def counts(ranges, elements):
    """(tokens, elements): how many of the keys e, e + elements, ... lie in each range."""
    lo, hi = (torch.tensor(x)[:, None] for x in zip(*ranges))
    e = torch.arange(elements)[None]
    up = lambda x: torch.clamp((x - e + elements - 1) // elements, min=0)  # noqa: E731
    return up(hi) - up(lo)


def as_counted(got, ranges):
    """Results back to numbers of keys; `want` may be up to 100, of which BF16 leaves 2^-8 at most, 0.4, unsure."""
    return got * torch.tensor([max(0, hi - lo) for lo, hi in ranges], dtype=torch.float64)[:, None]


def agree(got, want):
    assert want.max() <= 100
    return bool(((got - want).abs() < 0.45).all())


def check(kv, qn, share=4, kv_heads=2, dim=128, page=16, cache="bf16", causal=True, window=0, prefix=None, order="token", hints=True, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + sum(kv))
    need = [-(-n // page) for n in kv]
    ids = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(kv), max(need)), -1, dtype=torch.int32, device=DEV)
    shape = (sum(need) + 2, page, kv_heads, dim) if order == "token" else (sum(need) + 2, kv_heads, page, dim)
    k = torch.randn(shape, generator=g, device=DEV).clamp_(-3, 3)
    one, zero, kind = (1.0, 0.0, torch.bfloat16) if cache == "bf16" else (0x38, 0, torch.uint8)
    k = k.bfloat16() if cache == "bf16" else k.to(torch.float8_e4m3fn).view(torch.uint8)
    v = torch.full(shape, zero, dtype=kind, device=DEV)
    if order == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    at, elements = 0, kv_heads * dim
    for s, n in enumerate(kv):
        table[s, :need[s]] = ids[at:at + need[s]]
        at += need[s]
        j = torch.arange(n, device=DEV)
        v[table[s].long()[j // page], j % page, j % elements // dim, j % dim] = one
    start = [0] + list(itertools.accumulate(qn))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    single = all(n == 1 for n in qn)
    b = ecfa.Batch(table, i32(kv), None if single else i32(start), n_tokens=start[-1], **(dict(max_q=max(qn), max_kv=max(kv)) if hints else {}))
    q = torch.zeros((start[-1], kv_heads * share, dim), dtype=torch.bfloat16, device=DEV)
    got = ecfa.ecfa_attend(ecfa.Cache(k, v), b, q, causal=causal, window=window, prefix=None if prefix is None else i32(prefix)).cpu().double()
    got = got.view(start[-1], kv_heads, share, dim).transpose(1, 2).reshape(start[-1], share, elements)
    for s, n in enumerate(kv):
        if qn[s] == 0:
            continue
        ranges = seen_by(n, qn[s], causal, window, prefix[s] if prefix else 0)
        want = counts(ranges, elements)
        for h in range(share):
            mine = as_counted(got[start[s]:start[s + 1], h], ranges)
            assert agree(mine, want), (s, h, [(t, e, float(mine[t, e]), int(want[t, e])) for t, e in torch.nonzero((mine - want).abs() >= 0.45)[:8].tolist()])


def test_one_key_lost_or_taken_twice_is_seen():
    """On the CPU, in the oracle: any single key of the longest and shortest sequences below, and a step of 32."""
    for kv, elements in ((65541, 1024), (20011, 256), (700, 128), (1, 128)):
        ranges = seen_by(kv, 1, True, 0, 0)
        want = counts(ranges, elements).double()
        assert int(want.sum()) == kv
        got = lambda x: as_counted((x / kv).bfloat16().double(), ranges)  # noqa: E731
        assert agree(got(want), want)
        for j in random.Random(kv).sample(range(kv), min(kv, 50)):
            for by in (-1, 1):
                other = want.clone()
                other[0, j % elements] += by
                assert not agree(got(other), want)
    ranges = seen_by(300, 200, True, 70, 0)
    assert counts(ranges, 128).sum(1).tolist() == [70] * 200
    assert counts(seen_by(50, 3, True, 0, 49), 64).sum(1).tolist() == [49, 49, 50] and counts(seen_by(50, 3, False, 0, 0), 64).sum(1).tolist() == [50] * 3


@gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
def test_single_tokens(dim, cache):
    """Steps of 32 to 128 keys to a wave, four waves, pieces of every length; lengths about their borders."""
    for kv in (31, 33, 127, 129, 511, 512, 513, 1024, 1025, 2047, 4097, 6007):
        check([kv], [1], dim=dim, cache=cache, kv_heads=4)
    check([20011], [1], dim=dim, cache=cache, kv_heads=8)
    check([20011], [1], dim=dim, cache=cache, kv_heads=8, share=1, window=9999, order="head")


@gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [2, 7, 64, 300, 1025])
def test_ragged_decode_steps(n, cache):
    """Pieces that the device deals out by the lengths of all sequences; more sequences than are cut."""
    rng = random.Random(n)
    most = 8192 if n < 300 else 700
    kv = [most] + [int(math.exp(rng.uniform(0, math.log(most)))) for _ in range(n - 1)]
    check(kv, [1] * n, cache=cache, page=64, kv_heads=2 if n > 64 else 4)
    check(kv, [1] * n, cache=cache, page=64, kv_heads=2 if n > 64 else 4, window=333, hints=False)


@gpu
def test_a_long_sequence_among_short_ones():
    for cache in ("bf16", "e4m3"):
        check([65541, 3, 1, 500], [1] * 4, kv_heads=8, cache=cache, page=64)
        check([3, 1, 500, 65541], [1] * 4, kv_heads=8, cache=cache, page=1, share=1)


@gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("qn", [2, 4, 5, 8])
def test_up_to_32_rows(qn, dim, cache):
    for kv in ([600], [3001], [5000, 40, 1200]):
        check(kv, [qn] * len(kv), dim=dim, cache=cache, kv_heads=4)
        check(kv, [qn] * len(kv), dim=dim, cache=cache, kv_heads=4, window=700)


@gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_chunks(dim, cache):
    """Tiles of 128 rows, alone and cut in pieces; masks whose borders cross them."""
    for kv, qn in (([200], [200]), ([1111], [33]), ([6007, 900, 3000], [200, 77, 130]), ([4000], [60])):
        check(kv, qn, dim=dim, cache=cache, kv_heads=2 if max(kv) < 5000 else 4, share=2)
        for window in (1, 31, 32, 33, 64, 1000):
            check(kv, qn, dim=dim, cache=cache, kv_heads=2 if max(kv) < 5000 else 4, share=2, window=window)
        check(kv, qn, dim=dim, cache=cache, kv_heads=4, share=2, causal=False)
        check(kv, qn, dim=dim, cache=cache, kv_heads=4, share=2, prefix=[950] * len(kv))


@gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("share", [3, 8, 20])
def test_chunks_and_single_tokens_in_one_batch(share, cache):
    for kv, qn in (([700, 5100, 7, 64], [90, 1, 1, 3]), ([60, 5, 4000, 1, 2500], [33, 2, 1, 1, 1]), ([3000, 3000, 3000], [1, 200, 0])):
        for window in (0, 500):
            check(kv, qn, cache=cache, share=share, dim=64, kv_heads=2, page=32, window=window)
            check(kv, qn, cache=cache, share=share, dim=128, kv_heads=2, page=8, window=window, hints=False)
