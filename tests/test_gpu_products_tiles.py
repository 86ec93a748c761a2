"""The products on shapes of tile that other sizes reach with short K or one tile to a workgroup only (products_tiles.py), against 64-bit products on the device."""
import pytest
import torch

import products_reference as ref
import products_tiles as sizes
from paper_2510_02676_amd import ecfm
from test_gpu_products_large import DEV, bytes_of, check, laid

pytestmark = pytest.mark.gpu


def scales(gen, rows, k, kind):
    return torch.rand((rows,) if kind == "row" else (rows, ref.blocks(k)), generator=gen, device=DEV) + 0.1


@pytest.mark.parametrize("shape,m,n,k", sizes.DENSE)
@pytest.mark.parametrize("kind,dtype", [("group", torch.bfloat16), ("row", torch.float32)])
def test_products(shape, m, n, k, kind, dtype):
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    x, w, xs, ws = bytes_of(gen, (m, k)), bytes_of(gen, (1, n, k)), scales(gen, m, k, kind), torch.rand((1, ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1
    y = torch.full((m + 2, n), 777.0, dtype=dtype, device=DEV)
    weights = ecfm.Weights(laid(w, 16)[0], ws[0])
    ecfm.ecfm_gemm(weights, laid(x, 16), xs, y=y[1:-1])
    check(y[1:-1], x, xs, w, ws, [0, m], None)
    assert (y[0] == 777).all() and (y[-1] == 777).all()
    assert torch.equal(ecfm.ecfm_gemm(weights, laid(x, 16), xs, dtype=dtype), y[1:-1])


def run(counts, first, m, n, k, kind, gather, dtype=torch.bfloat16):
    """Rows of X in order or gathered, some of them nowhere; `first` rows of Y before the first expert's and the rest behind the last one's are nobody's."""
    gen = torch.Generator(device=DEV).manual_seed(m + n)
    starts = [first]
    for c in counts:
        starts.append(starts[-1] + c)
    tokens = m // 2 + 1 if gather else m
    x, w, xs = bytes_of(gen, (tokens, k)), bytes_of(gen, (len(counts), n, k)), scales(gen, tokens, k, kind)
    ws = torch.rand((len(counts), ref.blocks(n), ref.blocks(k)), generator=gen, device=DEV) + 0.1
    rows = None
    if gather:
        rows = torch.randint(0, tokens, (m,), generator=gen, device=DEV).to(torch.int32)
        rows[5::97] = -1
        rows[11::89] = tokens
    y = torch.full((m, n), 777.0, dtype=dtype, device=DEV)
    weights, s = ecfm.Weights(laid(w, 16), ws), torch.tensor(starts, dtype=torch.int32, device=DEV)
    ecfm.ecfm_gemm_experts(weights, s, laid(x, 16), xs, rows=rows, y=y)
    check(y, x, xs, w, ws, starts, rows)
    again = torch.full((m, n), 777.0, dtype=dtype, device=DEV)
    assert torch.equal(ecfm.ecfm_gemm_experts(weights, s, laid(x, 16), xs, rows=rows, y=again), y)


@pytest.mark.parametrize("shape,counts,n,k", sizes.FEW)
@pytest.mark.parametrize("kind,gather", [("group", True), ("row", False)])
def test_experts_with_few_rows(shape, counts, n, k, kind, gather):
    run(counts, 0, sum(counts), n, k, kind, gather)


@pytest.mark.parametrize("shape,m,experts,unlike,n,k", sizes.MANY)
@pytest.mark.parametrize("kind,gather,dtype", [("group", True, torch.bfloat16), ("row", False, torch.bfloat16), ("group", False, torch.float32)])
def test_experts_with_several_tiles_to_a_workgroup(shape, m, experts, unlike, n, k, kind, gather, dtype):
    run(sizes.counts_of(m, experts, unlike), 3, m, n, k, kind, gather, dtype)
