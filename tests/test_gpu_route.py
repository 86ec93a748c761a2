"""ecfm_route against sorting a token at a time in 64 bits: ties, scores of both kinds, a bias, groups, experts that are out, sizes around those of a
workgroup, a captured call."""
import math

import numpy as np
import pytest
import torch

import products_reference as ref
from paper_2510_02676_amd import ecfm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(logits, top, bias=None, routes=None, **options):
    """One call against the reference; weights are off by the rounding to fp32 and by 64-bit exponentials."""
    tokens, experts = logits.shape
    r = ecfm.ecfm_route(logits.to(DEV), top, bias=None if bias is None else bias.to(DEV), routes=routes, **options)
    ids, weights = ref.route(logits.double().numpy(), top, bias=None if bias is None else bias.tolist(), **options)
    assert r.ids.tolist() == ids
    starts, rows, place = ref.sort_pairs(ids, experts)
    assert r.starts.tolist() == starts and r.rows.tolist() == rows and r.place.tolist() == place
    got, want = r.weights.cpu().double().numpy(), np.array(weights).reshape(tokens, top)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 1e-13 * np.abs(want) + 1e-44).all()
    return r


def logits(tokens, experts, seed=0, dtype=torch.float32, size=1.5):
    return torch.randn((tokens, experts), generator=torch.Generator().manual_seed(seed)).mul(size).to(dtype)


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 63, 64, 65, 200])
@pytest.mark.parametrize("experts,top", [(1, 1), (2, 1), (2, 2), (7, 3), (64, 6), (65, 8), (128, 4), (256, 8), (300, 32), (1024, 10)])
def test_sizes(tokens, experts, top):
    check(logits(tokens, experts, tokens), top)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups,top_groups,experts,top", [(1, 1, 60, 4), (8, 4, 256, 8), (4, 1, 64, 6), (5, 5, 35, 12), (64, 3, 64, 2), (16, 7, 1024, 9), (3, 2, 771, 5)])
def test_options(sigmoid, normalise, with_bias, groups, top_groups, experts, top):
    bias = torch.randn(experts, generator=torch.Generator().manual_seed(3)) * 0.3 if with_bias else None
    check(logits(50, experts, 1), top, bias=bias, sigmoid=sigmoid, normalise=normalise, groups=groups, top_groups=top_groups, scale=2.5)


@pytest.mark.parametrize("groups", [1, 4])
def test_ties_go_to_the_lower_number(groups):
    x = torch.randint(0, 3, (70, 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    check(x, 6, groups=groups, top_groups=max(1, groups // 2))
    check(x, 6, groups=groups, top_groups=max(1, groups // 2), sigmoid=True)
    check(torch.zeros((5, 256)), 8, groups=groups)


def test_large_logits_in_order():
    x = torch.arange(200, dtype=torch.float32).flip(0).mul(3.0).expand(3, 200).contiguous() + 40       # sigmoids that are 1 in 64 bits too
    check(x, 5, sigmoid=True)
    check(-x, 5, sigmoid=True)
    check(-x * 10, 5, sigmoid=True)                                                                     # all scores 0: weights 0
    check(x * 1e36, 5)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_experts_that_are_out(sigmoid, groups):
    x = logits(40, 64, 5)
    gen = torch.Generator().manual_seed(6)
    x[torch.rand(x.shape, generator=gen) < 0.7] = -math.inf
    x[torch.rand(x.shape, generator=gen) < 0.05] = math.nan
    x[3] = -math.inf                                                       # nothing left
    x[4] = math.nan
    x[5], x[5, 17] = -math.inf, -2.0                                       # one left
    x[6, 20], x[6, 33] = math.inf, math.inf                                # two that are larger than all
    for top_groups in {1, groups}:
        r = check(x, 8, sigmoid=sigmoid, groups=groups, top_groups=top_groups, normalise=sigmoid)
    assert r.ids[3].tolist() == [-1] * 8 and r.weights[3].tolist() == [0] * 8 and r.place[4].tolist() == [-1] * 8 and r.ids[5, 0] == 17
    bias = torch.zeros(64)
    bias[:30], bias[31] = -math.inf, math.nan
    check(x, 8, sigmoid=sigmoid, bias=bias, groups=groups, top_groups=groups)
    check(torch.full((9, 64), -math.inf), 3)


@pytest.mark.parametrize("tokens,experts,top", [(4096, 256, 8), (16384, 40, 3), (16385, 256, 4), (20011, 64, 2), (70000, 5, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens(tokens, experts, top, dtype):
    x = logits(tokens, experts, 7, dtype)
    x[::97] = -math.inf
    r = ecfm.ecfm_route(x.to(DEV), top)
    v, i = x.double().sort(dim=1, descending=True, stable=True)
    ids = torch.where(v == -math.inf, -1, i)[:, :top]
    assert torch.equal(r.ids.cpu().long(), ids)
    flat = torch.where(ids < 0, experts, ids).reshape(-1)
    order = flat.sort(stable=True).indices
    n = int((flat < experts).sum())
    assert r.starts.tolist() == [0] + torch.bincount(flat, minlength=experts + 1)[:experts].cumsum(0).tolist()
    assert torch.equal(r.rows[:n].cpu().long(), order[:n] // top) and (r.rows[n:] == -1).all()
    place = torch.full((tokens * top,), -1)
    place[order[:n]] = torch.arange(n)
    assert torch.equal(r.place.cpu().long().view(-1), place)


def test_no_tokens():
    r = ecfm.ecfm_route(torch.empty((0, 30), device=DEV), 4)
    assert r.starts.tolist() == [0] * 31 and r.ids.shape == (0, 4)


def test_rows_apart():
    x = logits(70, 100, 8)
    wide = torch.full((70, 130), math.nan)
    wide[:, :100] = x
    r = ecfm.ecfm_route(wide.to(DEV)[:, :100], 5)
    ids, _ = ref.route(x.double().numpy(), 5)
    assert r.ids.tolist() == ids


def test_a_captured_call_and_the_same_routes_again():
    for tokens in (30, 300):
        x = torch.zeros((tokens, 64), device=DEV)
        routes = ecfm.Routes(tokens, 6, 64)
        ecfm.ecfm_route(x, 6, routes=routes)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ecfm.ecfm_route(x, 6, routes=routes)
        for seed in range(4):
            new = logits(tokens, 64, seed)
            x.copy_(new)
            graph.replay()
            torch.cuda.synchronize()
            ids, _ = ref.route(new.double().numpy(), 6)
            starts, rows, place = ref.sort_pairs(ids, 64)
            assert routes.ids.tolist() == ids and routes.starts.tolist() == starts and routes.rows.tolist() == rows and routes.place.tolist() == place
            check(new, 6, routes=routes)


@pytest.mark.parametrize("tokens,experts,top", [(32, 256, 8), (33, 256, 8), (17, 512, 4), (512, 96, 5), (513, 96, 5), (2049, 257, 3), (4097, 1000, 3), (9001, 1024, 2), (20011, 1000, 3), (40001, 64, 2),
                                                (65535, 9, 2), (65536, 9, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shares_of_the_workgroups(tokens, experts, top, dtype):
    test_many_tokens(tokens, experts, top, dtype)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups,top_groups,experts,top,tokens", [(8, 4, 256, 8, 601), (2, 1, 256, 8, 70), (32, 5, 256, 8, 70), (32, 2, 64, 4, 41), (12, 5, 96, 6, 70), (8, 3, 384, 8, 70),
                                                                  (33, 4, 66, 3, 45), (44, 7, 132, 4, 45), (4, 2, 1024, 8, 45), (10, 3, 1000, 8, 45), (64, 9, 512, 8, 45)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_groups_of_all_kinds(sigmoid, groups, top_groups, experts, top, tokens, dtype):
    check(logits(tokens, experts, 9, dtype), top, bias=torch.randn(experts, generator=torch.Generator().manual_seed(10)), sigmoid=sigmoid, groups=groups, top_groups=top_groups)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts", [64, 100, 256, 1024])
@pytest.mark.parametrize("options", [dict(), dict(sigmoid=True), dict(groups=4, top_groups=2)])
def test_the_ends_of_the_numbers(dtype, experts, options):
    """Zeros of both signs are the same, the largest numbers and infinity are ordered as the type has them, and what is out is never chosen."""
    ends = torch.tensor([0.0, -0.0, 1e-40, -1e-40, torch.finfo(dtype).max, -torch.finfo(dtype).max, math.inf, -math.inf, math.nan, 700.0, -700.0, -720.0, 1.0])
    x = ends[torch.randint(0, len(ends), (40, experts), generator=torch.Generator().manual_seed(11))].to(dtype)
    check(x, 32 if experts > 64 else 20, **options)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts", [64, 256, 512])
def test_a_first_number_off_the_alignment(dtype, experts):
    x, bias = logits(70, experts, 12, dtype), torch.randn(experts, generator=torch.Generator().manual_seed(13))
    room, other = torch.full((70 * experts + 1,), math.nan, dtype=dtype, device=DEV), torch.full((experts + 1,), math.nan, device=DEV)
    room[1:], other[1:] = x.view(-1).to(DEV), bias.to(DEV)
    for b in (None, bias):
        r = ecfm.ecfm_route(room[1:].view(70, experts), 6, bias=None if b is None else other[1:])
        assert r.ids.tolist() == ref.route(x.double().numpy(), 6, bias=None if b is None else b.tolist())[0]
        if b is not None:
            r = ecfm.ecfm_route(x.to(DEV), 6, bias=other[1:])
            assert r.ids.tolist() == ref.route(x.double().numpy(), 6, bias=b.tolist())[0]
