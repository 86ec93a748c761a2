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
