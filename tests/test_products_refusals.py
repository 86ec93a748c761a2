"""What the products of many rows refuse, before anything reaches a device: through the C ABI and the binding, without one."""
import math

import pytest
import torch

from paper_2510_02676_amd import ecf8, ecfa, ecfm

AT = 1 << 20                                        # an address that nothing looks at
lib = ecfm._lib
A, E = ecf8.E_ARG, ecf8.E_ALIGN


def make(kind, base, more):
    f = dict(base, **more)
    return kind(*(f.get(n, 0) for n, _ in kind._fields_))


def weights(**more):
    return make(ecfm._Weights, dict(d=AT, d_scale=AT, row_stride=256, expert_stride=25600, rows=100, cols=256, experts=1), more)


def x(**more):
    return make(ecfm._X, dict(d=AT, d_scale=AT, row_stride=256, rows=5, scale_cols=2), more)


def y(**more):
    return make(ecfm._Y, dict(d=AT, row_stride=100, rows=5, dtype=ecfa.BF16), more)


def gemm(w=None, xx=None, yy=None):
    return lib.ecfm_gemm(w or weights(), xx or x(), yy or y(), None)


def experts(w=None, starts=AT, xx=None, rows=None, yy=None):
    return lib.ecfm_gemm_experts(w or weights(experts=3), starts, xx or x(), rows, yy or y(), None)


@pytest.mark.parametrize("more,code", [(dict(d=None), A), (dict(rows=0), A), (dict(rows=(1 << 24) + 1), A), (dict(cols=0), A), (dict(cols=40), A), (dict(cols=(1 << 24) + 16), A),
                                       (dict(experts=0), A), (dict(experts=4097), A), (dict(d=AT + 8), E), (dict(row_stride=264), E), (dict(d_scale=AT + 2), E),
                                       (dict(row_stride=-256), A), (dict(row_stride=(1 << 24) + 16), A)])
def test_weights(more, code):
    assert gemm(w=weights(**more)) == code
    assert experts(w=weights(**dict(dict(experts=3), **more))) == code
    assert experts(w=weights(experts=3, expert_stride=25608)) == E


@pytest.mark.parametrize("more,code", [(dict(d=None), A), (dict(d_scale=None), A), (dict(scale_cols=0), A), (dict(scale_cols=3), A), (dict(rows=4), A), (dict(rows=(1 << 28) + 1), A),
                                       (dict(d=AT + 4), E), (dict(row_stride=250), E), (dict(d_scale=AT + 1), E),
                                       (dict(row_stride=-256), A), (dict(row_stride=1 << 32), A)])
def test_x(more, code):
    assert gemm(xx=x(**more)) == code
    assert experts(xx=x(**more)) == code


@pytest.mark.parametrize("more,code", [(dict(d=None), A), (dict(dtype=0), A), (dict(dtype=ecfa.E4M3), A), (dict(rows=6), A), (dict(d=AT + 1), E), (dict(dtype=ecfa.F32, d=AT + 2), E)])
def test_y(more, code):
    assert gemm(yy=y(**more)) == code
    assert experts(yy=y(**more)) == code


def test_products():
    assert gemm(w=weights(experts=2)) == A
    assert lib.ecfm_gemm(None, x(), y(), None) == A and lib.ecfm_gemm(weights(), None, y(), None) == A and lib.ecfm_gemm(weights(), x(), None, None) == A
    assert lib.ecfm_gemm_experts(None, AT, x(), None, y(), None) == A
    assert experts(starts=None) == A and experts(starts=AT + 2) == E and experts(rows=AT + 1) == E
    assert experts(rows=AT, xx=x(rows=0)) == A
    assert gemm(xx=x(rows=0), yy=y(rows=0)) == 0 and experts(xx=x(rows=0), yy=y(rows=0)) == 0          # nothing to do, and nothing done
    assert experts(xx=x(rows=7), rows=AT, yy=y(rows=0)) == 0


def route(at=(AT,) * 5, work=AT, room=1 << 40, **more):
    o = make(ecfm._RouteOpts, dict(d_logits=AT, logit_stride=64, n_tokens=5, experts=64, top=4, dtype=ecfa.F32, groups=1, top_groups=1, scale=1.0), more)
    return lib.ecfm_route(o, *at, work, room, None)


@pytest.mark.parametrize("more,code", [(dict(d_logits=None), A), (dict(experts=0), A), (dict(experts=1025), A), (dict(top=0), A), (dict(top=33), A), (dict(experts=3), A),
                                       (dict(n_tokens=(1 << 22) + 1), A), (dict(dtype=ecfa.E4M3), A), (dict(sigmoid=2), A), (dict(normalise=2), A), (dict(groups=0), A),
                                       (dict(groups=3), A), (dict(experts=130, groups=65), A), (dict(top_groups=0), A), (dict(top_groups=2), A),
                                       (dict(groups=32, top_groups=1), A), (dict(scale=math.inf), A), (dict(scale=math.nan), A), (dict(d_logits=AT + 2), E),
                                       (dict(dtype=ecfa.BF16, d_logits=AT + 1), E), (dict(d_bias=AT + 2), E)])
def test_route(more, code):
    assert route(**more) == code


def test_route_outputs_and_workspace():
    for i in range(5):
        assert route(at=tuple(None if j == i else AT for j in range(5))) == A
        assert route(at=tuple(AT + 2 if j == i else AT for j in range(5))) == E
    assert lib.ecfm_route(None, AT, AT, AT, AT, AT, AT, 1 << 40, None) == A
    need = lib.ecfm_route_workspace_bytes
    assert need(5, 64, 4) == 0 and need(5000, 64, 4) > 0 and need(5, 0, 1) == 0 and need(5000, 2000, 4) == 0 and need(5000, 64, 65) == 0
    assert route(n_tokens=5000, work=None) == ecf8.E_CAPACITY and route(n_tokens=5000, room=need(5000, 64, 4) - 1) == ecf8.E_CAPACITY and route(work=AT + 2) == E


def gate(g=AT, u=AT, dtype=ecfa.BF16, rows=5, cols=256, gs=256, us=256, group=128, q=AT, scale=AT):
    return lib.ecfm_gate(g, u, dtype, rows, cols, gs, us, group, q, scale, None)


@pytest.mark.parametrize("more,code", [(dict(g=None), A), (dict(u=None), A), (dict(q=None), A), (dict(scale=None), A), (dict(dtype=ecfa.E4M3), A), (dict(cols=0), A), (dict(cols=200), A),
                                       (dict(cols=200, group=0), A), (dict(cols=(1 << 20) + 128), A), (dict(group=64), A), (dict(rows=(1 << 40) + 1), A), (dict(g=AT + 8), E),
                                       (dict(u=AT + 2), E), (dict(gs=257), E), (dict(us=260), E), (dict(q=AT + 4), E), (dict(scale=AT + 2), E)])
def test_gate(more, code):
    assert gate(**more) == code
    assert gate(rows=0) == 0


def combine(yy=None, place=AT, w=AT, tokens=5, top=2, cols=64, add=None, out=None):
    rows = dict(row_stride=64)
    return lib.ecfm_combine(yy or y(**rows), place, w, tokens, top, cols, add, out or y(**rows), None)


@pytest.mark.parametrize("more,code", [(dict(place=None), A), (dict(w=None), A), (dict(top=0), A), (dict(top=33), A), (dict(cols=0), A), (dict(cols=60), A),
                                       (dict(cols=(1 << 20) + 8), A), (dict(tokens=6), A), (dict(place=AT + 2), E), (dict(w=AT + 1), E),
                                       (dict(yy=dict(d=None)), A), (dict(yy=dict(dtype=0)), A), (dict(yy=dict(rows=(1 << 28) + 1)), A), (dict(yy=dict(d=AT + 8)), E),
                                       (dict(yy=dict(row_stride=68)), E), (dict(out=dict(d=None)), A), (dict(out=dict(rows=4)), A), (dict(out=dict(row_stride=66)), E),
                                       (dict(add=dict(rows=4)), A), (dict(add=dict(dtype=7)), A), (dict(add=dict(row_stride=66)), E)])
def test_combine(more, code):
    more = {k: y(**dict(dict(row_stride=64), **v)) if isinstance(v, dict) else v for k, v in more.items()}
    assert combine(**more) == code


def test_combine_of_nothing():
    assert combine(tokens=0, out=y(rows=0, row_stride=64)) == 0
    assert lib.ecfm_combine(None, AT, AT, 5, 2, 64, None, y(row_stride=64), None) == A


def refused(call):
    with pytest.raises(ecf8.Ecf8Error) as e:
        call()
    return e.value.code == A


def test_binding():
    w, s = torch.zeros((100, 256), dtype=torch.uint8), torch.zeros((1, 2))
    ok = ecfm.Weights(w, s)
    for bad in (lambda: ecfm.Weights(w.float()), lambda: ecfm.Weights(w.view(-1)), lambda: ecfm.Weights(w[:, ::2]), lambda: ecfm.Weights(w[:0]), lambda: ecfm.Weights(w, s.double()),
                lambda: ecfm.Weights(w, torch.zeros((2, 1))), lambda: ecfm.Weights(w[None], s)):
        assert refused(bad)
    xx = torch.zeros((5, 256), dtype=torch.uint8)
    # tensors on the host are refused everywhere
    assert refused(lambda: ecfm.ecfm_gemm(ok, xx)) and refused(lambda: ecfm.ecfm_gemm_experts(ecfm.Weights(w[None]), torch.zeros(2, dtype=torch.int32), xx))
    assert refused(lambda: ecfm.ecfm_gemm(ecfm.Weights(w[None]), xx)) and refused(lambda: ecfm.ecfm_gemm_experts(ok, torch.zeros(2, dtype=torch.int32), xx))
    assert refused(lambda: ecfm.ecfm_route(torch.zeros((5, 64)), 2)) and refused(lambda: ecfm.ecfm_gate(torch.zeros((5, 64)), torch.zeros((5, 64))))
    assert refused(lambda: ecfm.ecfm_combine(torch.zeros((5, 64)), torch.zeros((5, 1), dtype=torch.int32), torch.zeros((5, 1))))
    for bad in ((-1, 2, 64), (5, 0, 64), (5, 33, 64), (5, 9, 8), (5, 2, 1025), ((1 << 22) + 1, 2, 64)):
        assert refused(lambda: ecfm.Routes(*bad, device="cpu"))
    # what the operands' shapes and types have to be, told apart by the helpers that every call uses
    for bad in (lambda: ecfm._x("f", ok, xx[:, :128], None), lambda: ecfm._x("f", ok, xx.float(), None), lambda: ecfm._x("f", ok, xx, torch.zeros((5, 3))),
                lambda: ecfm._x("f", ok, xx, torch.zeros(4)), lambda: ecfm._x("f", ok, xx, torch.zeros((5, 2)).double()), lambda: ecfm._x("f", ok, xx, torch.zeros((2, 5)).t()),
                lambda: ecfm._matrix("f", torch.zeros((5, 64)).half(), 5, 64, -1), lambda: ecfm._matrix("f", torch.zeros((5, 64)), 4, 64, -1),
                lambda: ecfm._matrix("f", torch.zeros((64, 5)).t(), 5, 64, -1)):
        assert refused(bad)
