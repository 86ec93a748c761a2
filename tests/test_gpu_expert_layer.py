"""An expert layer with compressed weights, step by step against 64 bits: every stage from what the stage before it left; captured and replayed, and two
layers that share the buffers of their weights."""
import numpy as np
import pytest
import torch

import products_reference as ref
from attention_reference import E4M3
from paper_2510_02676_amd import ecf8, ecfm, synth
from paper_2510_02676_amd.experts import CompressedExperts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def layer_weights(n, inner, hidden, seed=0):
    """(what CompressedExperts takes, {name: (bytes, scale) of each expert})."""
    g = torch.Generator().manual_seed(seed)
    packed, full = [], []
    for e in range(n):
        p, f = {}, {}
        for i, (name, rows, cols) in enumerate([("gate", inner, hidden), ("up", inner, hidden), ("down", hidden, inner)]):
            w = synth.make_weight(rows, cols, 1.7, 0.02, seed, 3 * e + i).numpy()
            scale = (torch.rand((rows // 128, cols // 128), generator=g) * 0.5 + 0.5) * 2.0 ** -9
            blob = ecf8.ecf8_encode(w, lane_syms=64)
            p[name], f[name] = (blob.header, blob.to(DEV), scale.to(DEV)), (w, scale.numpy())
        packed.append(p)
        full.append(f)
    return packed, full


def check_product(got, x8, x_scale, parts, starts, rows):
    """Rows of every expert against its weights: a list of (bytes, scale), one above the other."""
    got = got.cpu().double().numpy()
    for e, ws in enumerate(parts):
        r = rows[starts[e]:starts[e + 1]]
        if not len(r):
            continue
        at = 0
        for w, s in ws:
            want, size = ref.product(x8[r], x_scale[r], w, s)
            part = got[starts[e]:starts[e + 1], at:at + w.shape[0]]
            assert (np.abs(part - want) <= ref.product_bound(want, size, w.shape[1], 2.0 ** -8)).all()
            at += w.shape[0]


@pytest.mark.parametrize("tokens", [1, 7, 150])
@pytest.mark.parametrize("options", [{}, dict(sigmoid=True, groups=2, top_groups=1, scale=1.5)], ids=["softmax", "groups"])
def test_a_step(tokens, options):
    n, inner, hidden, top = 6, 256, 384, 3
    packed, full = layer_weights(n, inner, hidden)
    layer = CompressedExperts(packed, tokens, top, **options)
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).bfloat16().to(DEV)
    logits, add = torch.randn((tokens, n), generator=g), torch.randn((tokens, hidden), generator=g).bfloat16()
    y = layer(x, logits.to(DEV), add.to(DEV)).clone()
    torch.cuda.synchronize()
    ids, weights = ref.route(logits.double().numpy(), top, **options)
    starts, rows, place = ref.sort_pairs(ids, n)
    assert layer.routes.ids.tolist() == ids and layer.routes.starts.tolist() == starts and layer.routes.rows.tolist() == rows
    for i, f in enumerate(full):                                           # the weights as they were
        assert np.array_equal(layer.room[0][i].cpu().numpy(), np.concatenate((f["gate"][0], f["up"][0]))) and np.array_equal(layer.room[1][i].cpu().numpy(), f["down"][0])
    x8, xs = layer.x8.cpu().numpy(), layer.x_scale.cpu().numpy()
    by = np.repeat(xs.astype(np.float64), 128, 1)
    assert (np.abs(E4M3[x8] * by - x.cpu().double().numpy()) <= (2.0 ** -4 + 2.0 ** -20) * np.abs(x.cpu().double().numpy()) + 2.0 ** -10 * by).all()
    check_product(layer.mid, x8, xs, [[f["gate"], f["up"]] for f in full], starts, np.array(rows))
    mid = layer.mid.cpu().double().numpy()
    h = ref.gate(mid[:, :inner], mid[:, inner:])
    h8, hs = layer.h8.cpu().numpy(), layer.h_scale.cpu().numpy()
    by = np.repeat(hs.astype(np.float64), 128, 1)
    assert (np.abs(E4M3[h8] * by - h) <= (2.0 ** -4 + 2.0 ** -10) * np.abs(h) + 2.0 ** -10 * by * (1 + 2.0 ** -10)).all()
    check_product(layer.back, h8, hs, [[f["down"]] for f in full], starts, np.arange(len(rows)))
    back, want = layer.back.cpu().double().numpy(), add.double().numpy()
    size = np.abs(want)
    for j in range(top):
        term = np.array(weights)[:, j:j + 1] * back[np.array(place)[:, j]]
        want, size = want + term, size + np.abs(term)
    assert (np.abs(y.cpu().double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size).all()


def test_captured_with_a_shared_buffer():
    n, inner, hidden, top, tokens = 4, 128, 256, 2, 90
    layers = []
    for seed in (1, 2):
        packed, _ = layer_weights(n, inner, hidden, seed)
        layers.append(CompressedExperts(packed, tokens, top, room=layers[0].room if layers else None))
    x, logits = torch.zeros((tokens, hidden), dtype=torch.bfloat16, device=DEV), torch.zeros((2, tokens, n), device=DEV)
    run = lambda: layers[1](layers[0](x, logits[0], x), logits[1])  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g))
        logits.copy_(torch.randn(logits.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = layers[1].y.clone()
        layers[1].y.fill_(777)
        assert torch.equal(run(), got) and got.isfinite().all()


def test_on_another_stream():
    packed, _ = layer_weights(3, 128, 128, 3)
    layer = CompressedExperts(packed, 70, 2)
    g = torch.Generator().manual_seed(0)
    x, logits = torch.randn((70, 128), generator=g).to(DEV), torch.randn((70, 3), generator=g).to(DEV)
    want = layer(x, logits).clone()
    layer.y.fill_(777)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layer(x, logits, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_what_a_step_would_refuse():
    packed, _ = layer_weights(3, 128, 256, 4)
    a = ecf8.E_ARG

    def refused(*args, **more):
        with pytest.raises(ecf8.Ecf8Error) as e:
            CompressedExperts(*args, **more)
        return e.value.code == a
    swapped = [dict(packed[0], gate=packed[0]["down"])] + packed[1:]
    cut = [dict(packed[0], up=(*packed[0]["up"][:2], packed[0]["up"][2][:, :1]))] + packed[1:]
    host = [dict(packed[0], up=(packed[0]["up"][0], packed[0]["up"][1].cpu(), packed[0]["up"][2]))] + packed[1:]
    assert refused(swapped, 5, 2) and refused(packed[:1] + swapped, 5, 2) and refused(cut, 5, 2) and refused(host, 5, 2)
    assert refused(packed, 5, 4) and refused(packed, 5, 0) and refused(packed, 5, 2, groups=2) and refused(packed, 5, 2, groups=3, top_groups=1)
    assert refused(packed, 5, 2, scale=float("inf")) and refused(packed, 5, 2, bias=torch.zeros(4, device=DEV))
    assert refused(packed, 5, 2, room=tuple(torch.empty((3, 8, 8), dtype=torch.uint8, device=DEV) for _ in range(2)))
    layer = CompressedExperts(packed, 5, 2)
    for x, logits in ((torch.zeros((4, 256), device=DEV), torch.zeros((5, 3), device=DEV)), (torch.zeros((5, 256), device=DEV), torch.zeros((5, 4), device=DEV))):
        with pytest.raises(ecf8.Ecf8Error):
            layer(x, logits)
