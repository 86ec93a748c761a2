"""What the products of many rows accept, without a device: a library in front of the runtime's answers for it and counts the launches."""
from test_host_launches import run_on_shim

CODE = r"""
from paper_2510_02676_amd import ecfa, ecfm
at, lib, A, E = 1 << 20, ecfm._lib, ecf8.E_ARG, ecf8.E_ALIGN             # an address that nothing looks at
def weights(rows=100, cols=256, experts=1, row=256, expert=25600):
    return ecfm._Weights(at, at, row, expert, rows, cols, experts, 0)
def x(rows=5, row=256, per=2):
    return ecfm._X(at, at if per else None, row, rows, per)
def y(rows=5, row=100, dtype=ecfa.BF16):
    return ecfm._Y(at, row, rows, dtype)
def launched(rc):
    n, var("launches").value = var("launches").value, 0
    return rc, n
def gemm(w, xx, yy): return launched(lib.ecfm_gemm(w, xx, yy, None))
def experts(w, xx, yy, rows=None): return launched(lib.ecfm_gemm_experts(w, at, xx, rows, yy, None))
assert gemm(weights(), x(), y()) == (0, 1) and experts(weights(experts=3), x(), y()) == (0, 1) and experts(weights(experts=3), x(2), y(), at) == (0, 1)
# every size has a kernel, and one launch
for m in (1, 15, 16, 17, 40, 64, 65, 100, 200, 300, 1000, 5000, 70000, 1 << 20):
    for n in (1, 16, 100, 1000, 4096, 70000):
        for k in (16, 128, 144, 4096, 1 << 20):
            w = weights(n, k, 1, k)
            assert gemm(w, x(m, k, (k + 127) // 128), y(m, n)) == (0, 1), (m, n, k)
            assert experts(weights(n, k, 64, k, n * k), x(m, k, 1), y(m, n)) == (0, 1)
assert gemm(weights(1 << 24, 16, 1, 16), x(1 << 28, 16, 1), y(1 << 28, 1 << 24)) == (A, 0)       # 2^36 tiles
assert gemm(weights(1, 16, 1, 16), x(1 << 28, 16, 1), y(1 << 28, 1)) == (0, 1)
# strides between things of which there is one
for odd in (1, -3, 255, (1 << 40) + 1):
    assert gemm(weights(1, row=odd), x(), y(row=1)) == (0, 1) and gemm(weights(expert=odd), x(), y()) == (0, 1)
    assert gemm(weights(), x(1, odd), y(1, odd)) == (0, 1)
    assert gemm(weights(row=odd), x(), y())[1] == 0 and experts(weights(experts=2, expert=odd), x(), y()) == (E, 0) and gemm(weights(), x(row=odd), y())[1] == 0
def route(tokens, per=64, experts=64, room=1 << 40):
    o = ecfm._RouteOpts(at, None, per, tokens, experts, 4, ecfa.F32, 0, 1, 1, 1, 1.0, 0)
    return launched(lib.ecfm_route(o, at, at, at, at, at, at, room, None))
assert [route(t) for t in (0, 1, 32, 33, 65535, 65536, 1 << 22)] == [(0, n) for n in (1, 1, 1, 2, 2, 3, 3)]
assert [route(t, 512, 512) for t in (16, 17, 65535, 65536)] == [(0, n) for n in (1, 2, 2, 3)]
need = lib.ecfm_route_workspace_bytes
for t in (33, 511, 513, 16384, 16385, 65535, 65536, 1 << 22):
    assert route(t, room=need(t, 64, 4)) == (0, 2 if t <= 65535 else 3) and route(t, room=need(t, 64, 4) - 1) == (ecf8.E_CAPACITY, 0)
def gate(rows, cols, stride, group): return launched(lib.ecfm_gate(at, at, ecfa.BF16, rows, cols, stride, stride, group, at, at, None))
for group in (0, 128):
    assert gate(5, 256, 256, group) == (0, 1) and gate(1, 256, 7, group) == (0, 1) and gate(2, 256, 7, group) == (E, 0)
    n, cols = 1 << 23, 1 << 11
    assert gate(n, cols, cols, group) == (0, -(-n // min(0x7fffff00 // (cols // 8), 0x1fffff)))
def combine(tokens, cols, rows=9, add=None): return launched(lib.ecfm_combine(y(rows, cols), at, at, tokens, 2, cols, add, y(tokens, cols), None))
assert combine(5, 64) == (0, 1) and combine(5, 64, 0) == (0, 1) and combine(0, 64) == (0, 0) and combine(5, 64, add=y(5, 64)) == (0, 1)
assert combine(1 << 22, 1 << 20) == (0, -(-(1 << 22) // (0x7fffff00 // (1 << 17))))
# a launch that fails
for call in (lambda: gemm(weights(), x(), y()), lambda: route(5), lambda: gate(5, 256, 256, 0), lambda: combine(5, 64)):
    var("fail_at").value = 0
    assert call()[0] == ecf8.E_HIP
    var("fail_at").value = -1
"""


def test_launches(tmp_path):
    run_on_shim(tmp_path, CODE)
