"""What the attention calls refuse, before anything reaches a device: through the C ABI, without one."""
import ctypes

import pytest
import torch

from paper_2510_02676_amd import ecf8, ecfa

AT = 1 << 20                                        # an address that nothing looks at
lib = ecfa._lib


def cache(**more):
    f = dict(d_k=AT, d_v=AT, n_pages=4, page_size=16, kv_heads=2, head_dim=64, dtype=ecfa.BF16, k=(2048, 128, 64), v=(2048, 128, 64))
    f.update(more)
    return ecfa._Cache(f["d_k"], f["d_v"], f.get("d_k_scale"), f.get("d_v_scale"), (ctypes.c_int64 * 3)(*f["k"]), (ctypes.c_int64 * 3)(*f["v"]), f["n_pages"],
                       f["page_size"], f["kv_heads"], f["head_dim"], f["dtype"], 0)


def batch(**more):
    f = dict(d_page_table=AT, d_kv_len=AT, d_q_start=AT, table_stride=4, table_width=4, n_seqs=2, n_tokens=3, max_q=0, max_kv=0)
    f.update(more)
    return ecfa._Batch(*(f[n] for n, _ in ecfa._Batch._fields_[:-1]), 0)


def rows(**more):
    f = dict(d=AT, token_stride=256, head_stride=64, heads=4, dtype=ecfa.BF16)
    f.update(more)
    return ecfa._Rows(*(f[n] for n, _ in ecfa._Rows._fields_))


def opts(**more):
    f = dict(scale=0.1, softcap=0.0, d_slopes=None, d_prefix_len=None, causal=1, window=0)
    f.update(more)
    return ecfa._AttendOpts(*(f[n] for n, _ in ecfa._AttendOpts._fields_))


def rope(**more):
    f = dict(d_freq=AT, d_pos=None, rot_dim=64, interleaved=0, scale=1.0)
    f.update(more)
    return ecfa._Rope(*(f[n] for n, _ in ecfa._Rope._fields_[:-1]), 0)


BAD_CACHES = [(dict(d_k=None), ecf8.E_ARG), (dict(d_v=None), ecf8.E_ARG), (dict(n_pages=0), ecf8.E_ARG), (dict(n_pages=2 ** 31), ecf8.E_ARG),
              (dict(page_size=0), ecf8.E_ARG), (dict(page_size=24), ecf8.E_ARG), (dict(page_size=1 << 17), ecf8.E_ARG), (dict(kv_heads=0), ecf8.E_ARG),
              (dict(head_dim=0), ecf8.E_ARG), (dict(head_dim=72), ecf8.E_ARG), (dict(head_dim=272), ecf8.E_ARG), (dict(dtype=ecfa.F32), ecf8.E_ARG),
              (dict(dtype=0), ecf8.E_ARG), (dict(d_k=AT + 8), ecf8.E_ALIGN), (dict(d_v=AT + 2), ecf8.E_ALIGN), (dict(k=(2048, 128, 60)), ecf8.E_ALIGN),
              (dict(v=(2048, 132, 64)), ecf8.E_ALIGN), (dict(dtype=ecfa.E4M3, k=(2048, 128, 72)), ecf8.E_ALIGN), (dict(d_k_scale=AT + 2), ecf8.E_ALIGN),
              (dict(d_v_scale=AT + 1), ecf8.E_ALIGN)]
BAD_BATCHES = [(dict(d_page_table=None), ecf8.E_ARG), (dict(d_kv_len=None), ecf8.E_ARG), (dict(table_width=0), ecf8.E_ARG), (dict(n_seqs=0), ecf8.E_ARG),
               (dict(table_width=1 << 27), ecf8.E_ARG), (dict(n_tokens=(1 << 22) + 1), ecf8.E_ARG), (dict(n_seqs=(1 << 22) + 1), ecf8.E_ARG),
               (dict(d_q_start=None), ecf8.E_ARG), (dict(d_page_table=AT + 2), ecf8.E_ALIGN), (dict(d_kv_len=AT + 1), ecf8.E_ALIGN), (dict(d_q_start=AT + 3), ecf8.E_ALIGN)]


def attend(c=None, b=None, o=None, q=None, out=None, work=AT, room=1 << 40):
    return lib.ecfa_attend(c or cache(), b or batch(), o or opts(), q or rows(), out or rows(), work, room, None)


def append(c=None, b=None, r=None, q=None, k=None, v=None, out=None):
    kv = dict(heads=2, token_stride=128)
    return lib.ecfa_append(c or cache(), b or batch(), r or rope(), q or rows(), k or rows(**kv), v or rows(**kv), out or rows(), None)


@pytest.mark.parametrize("more,code", BAD_CACHES)
def test_caches(more, code):
    assert attend(c=cache(**more)) == code
    assert append(c=cache(**more)) == code
    assert lib.ecfa_attend_workspace_bytes(cache(**more), batch(), 4) == 0


@pytest.mark.parametrize("more,code", BAD_BATCHES)
def test_batches(more, code):
    assert attend(b=batch(**more)) == code
    assert append(b=batch(**more)) == code


@pytest.mark.parametrize("more,code", [(dict(scale=0.0), ecf8.E_ARG), (dict(scale=-1.0), ecf8.E_ARG), (dict(scale=float("nan")), ecf8.E_ARG), (dict(scale=float("inf")), ecf8.E_ARG),
                                       (dict(softcap=-1.0), ecf8.E_ARG), (dict(softcap=float("nan")), ecf8.E_ARG), (dict(softcap=float("inf")), ecf8.E_ARG), (dict(causal=2), ecf8.E_ARG),
                                       (dict(window=5, d_prefix_len=AT), ecf8.E_ARG), (dict(d_slopes=AT + 2), ecf8.E_ALIGN), (dict(d_prefix_len=AT + 2), ecf8.E_ALIGN)])
def test_options(more, code):
    assert attend(o=opts(**more)) == code


@pytest.mark.parametrize("more,code", [(dict(heads=3), ecf8.E_ARG), (dict(heads=0), ecf8.E_ARG), (dict(d=None), ecf8.E_ARG), (dict(dtype=ecfa.F32), ecf8.E_ARG),
                                       (dict(d=AT + 8), ecf8.E_ALIGN), (dict(token_stride=252), ecf8.E_ALIGN), (dict(head_stride=65), ecf8.E_ALIGN)])
def test_rows_of_attend(more, code):
    assert attend(q=rows(**more)) == code
    assert attend(out=rows(**more)) == code
    assert attend(out=rows(heads=8)) == ecf8.E_ARG


def test_rows_and_rotation_of_append():
    kv = dict(heads=2, token_stride=128)
    assert append(k=rows(heads=4)) == ecf8.E_ARG and append(v=rows(heads=1)) == ecf8.E_ARG
    assert append(k=rows(dtype=ecfa.F32, **kv)) == ecf8.E_ARG                      # unlike types
    assert append(out=rows(dtype=ecfa.F32)) == ecf8.E_ARG and append(out=rows(heads=2)) == ecf8.E_ARG
    assert append(v=rows(**{**kv, "d": AT + 4})) == ecf8.E_ALIGN and append(q=rows(head_stride=36)) == ecf8.E_ALIGN
    assert append(q=rows(heads=0), out=rows(heads=0)) == ecf8.E_ARG
    for more in (dict(rot_dim=0), dict(rot_dim=8), dict(rot_dim=80), dict(d_freq=None), dict(interleaved=2), dict(scale=float("nan"))):
        assert append(r=rope(**more)) == ecf8.E_ARG
    assert append(r=rope(d_freq=AT + 4)) == ecf8.E_ALIGN and append(r=rope(d_pos=AT + 2)) == ecf8.E_ALIGN
    call = lambda q, k, v, o: lib.ecfa_append(cache(), batch(), None, q, k, v, o, None)  # noqa: E731
    assert call(None, None, None, None) == ecf8.E_ARG
    assert call(rows(), rows(**kv), None, rows()) == ecf8.E_ARG and call(rows(), None, rows(**kv), rows()) == ecf8.E_ARG
    assert call(rows(), rows(**kv), rows(**kv), None) == ecf8.E_ARG and call(None, rows(**kv), rows(**kv), rows()) == ecf8.E_ARG
    assert lib.ecfa_append(None, batch(), None, rows(), rows(**kv), rows(**kv), rows(), None) == ecf8.E_ARG
    assert lib.ecfa_append(cache(), None, None, rows(), rows(**kv), rows(**kv), rows(), None) == ecf8.E_ARG
    assert lib.ecfa_attend(cache(), batch(), None, rows(), rows(), AT, 1 << 40, None) == ecf8.E_ARG


def test_nothing_to_do_is_no_error():
    none = batch(n_tokens=0)
    assert attend(b=none, q=rows(d=None), out=rows(d=None), work=None, room=0) == ecf8.OK
    assert append(b=none) == ecf8.OK
    assert lib.ecfa_quant(None, ecfa.F32, 0, 256, 256, 0, None, None, None) == ecf8.OK


@pytest.mark.parametrize("dtype,rows_,cols,stride,group,x,q,s,code", [
    (ecfa.E4M3, 4, 256, 256, 0, AT, AT, AT, ecf8.E_ARG), (0, 4, 256, 256, 0, AT, AT, AT, ecf8.E_ARG), (ecfa.F32, 4, 0, 256, 0, AT, AT, AT, ecf8.E_ARG),
    (ecfa.F32, 4, 200, 256, 0, AT, AT, AT, ecf8.E_ARG), (ecfa.F32, 4, 192, 256, 128, AT, AT, AT, ecf8.E_ARG), (ecfa.F32, 4, 256, 256, 64, AT, AT, AT, ecf8.E_ARG),
    (ecfa.F32, 4, (1 << 20) + 128, 1 << 21, 0, AT, AT, AT, ecf8.E_ARG), (ecfa.F32, (1 << 40) + 1, 256, 256, 0, AT, AT, AT, ecf8.E_ARG),
    (ecfa.F32, 4, 256, 256, 0, None, AT, AT, ecf8.E_ARG), (ecfa.F32, 4, 256, 256, 0, AT, None, AT, ecf8.E_ARG), (ecfa.F32, 4, 256, 256, 0, AT, AT, None, ecf8.E_ARG),
    (ecfa.F32, 4, 256, 258, 0, AT, AT, AT, ecf8.E_ALIGN), (ecfa.BF16, 4, 256, 260, 0, AT, AT, AT, ecf8.E_ALIGN), (ecfa.BF16, 4, 256, 256, 0, AT + 2, AT, AT, ecf8.E_ALIGN),
    (ecfa.BF16, 4, 256, 256, 0, AT, AT + 4, AT, ecf8.E_ALIGN), (ecfa.BF16, 4, 256, 256, 0, AT, AT, AT + 2, ecf8.E_ALIGN)])
def test_quant(dtype, rows_, cols, stride, group, x, q, s, code):
    assert lib.ecfa_quant(x, dtype, rows_, cols, stride, group, q, s, None) == code


def test_frequencies():
    out, scale = (ctypes.c_uint64 * 64)(), ctypes.c_float()
    call = lambda rot=64, base=1e4, kind=0, factor=2.0, orig=100.0, fast=32.0, slow=1.0, f=out: lib.ecfa_rope_freq(rot, base, kind, factor, orig, fast, slow, f, scale)  # noqa: E731
    assert call() == ecf8.OK and call(kind=3) == ecf8.OK and call(factor=-1.0) == ecf8.OK
    inf, nan = float("inf"), float("nan")
    for more in (dict(rot=0), dict(rot=5), dict(base=1.0), dict(base=nan), dict(base=inf), dict(kind=4), dict(kind=1, factor=0.5), dict(kind=1, factor=nan), dict(kind=2, rot=2),
                 dict(kind=3, orig=0.0), dict(kind=3, slow=0.0), dict(kind=3, fast=1.0), dict(kind=3, fast=nan), dict(f=None), dict(kind=2, base=1e300, factor=1e300)):
        assert call(**more) == ecf8.E_ARG, more


def test_the_binding_checks_what_it_is_given():
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for k, v in ((t(2, 16, 2, 64), t(2, 16, 2, 32)), (t(2, 16, 2, 64, d=torch.float16), t(2, 16, 2, 64, d=torch.float16)), (t(2, 16, 128), t(2, 16, 128)),
                 (t(2, 16, 64, 2).transpose(2, 3), t(2, 16, 64, 2).transpose(2, 3))):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.Cache(k, v)
    with pytest.raises(ecf8.Ecf8Error):
        ecfa.Cache(t(2, 16, 2, 64), t(2, 16, 2, 64), k_scale=torch.ones(3))
    for a in ((i32(2, 4), i32(3)), (i32(2, 4), i32(2).long()), (i32(8), i32(2)), (i32(2, 4), i32(2), i32(2)), (i32(2, 4), i32(2), i32(3)), (i32(4, 2).t(), i32(2))):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.Batch(*a)
    with pytest.raises(ecf8.Ecf8Error):
        ecfa.Rope(torch.zeros(32))
    c, b = ecfa.Cache(t(2, 16, 2, 64), t(2, 16, 2, 64)), ecfa.Batch(i32(2, 4), i32(2))
    for q in (t(3, 4, 64), t(2, 4, 32), t(2, 256), t(2, 4, 64, d=torch.float16), t(2, 64, 4).transpose(1, 2)):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.ecfa_attend(c, b, q)
    for more in (dict(slopes=torch.zeros(3)), dict(prefix=i32(3)), dict(out=t(2, 2, 64))):
        with pytest.raises(ecf8.Ecf8Error):
            ecfa.ecfa_attend(c, b, t(2, 4, 64), **more)
    with pytest.raises(ecf8.Ecf8Error):
        ecfa.ecfa_append(c, b, t(2, 2, 64), t(2, 2, 64), q_out=t(2, 4, 64))
    with pytest.raises(ecf8.Ecf8Error):
        ecfa.ecfa_append(c, b, t(2, 2, 64), t(2, 2, 64), rope=ecfa.Rope(torch.zeros(32, dtype=torch.int64), pos=i32(3)))


def test_host_tensors_reach_no_kernel(monkeypatch):
    """Tensors on the host are refused before the library hears of them."""
    def reached(*a):
        raise AssertionError("reached the library")

    for name in ("_append", "_attend", "_quant"):
        monkeypatch.setattr(ecfa, name, reached)
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c, b, r = ecfa.Cache(t(2, 16, 2, 64), t(2, 16, 2, 64)), ecfa.Batch(i32(2, 4), i32(2)), ecfa.Rope(torch.zeros(32, dtype=torch.int64))
    calls = [lambda: ecfa.ecfa_attend(c, b, t(2, 4, 64)), lambda: ecfa.ecfa_attend(c, b, t(2, 4, 64), out=t(2, 4, 64), workspace=t(1 << 20, d=torch.uint8)),
             lambda: ecfa.ecfa_append(c, b, t(2, 2, 64), t(2, 2, 64)), lambda: ecfa.ecfa_append(c, b, t(2, 2, 64), t(2, 2, 64), t(2, 4, 64), t(2, 4, 64), r),
             lambda: ecfa.ecfa_quant(t(2, 256)), lambda: ecfa.ecfa_quant(t(2, 256), 128, t(2, 256, d=torch.uint8), t(2, 2, d=torch.float32))]
    for call in calls:
        with pytest.raises(ecf8.Ecf8Error) as e:
            call()
        assert e.value.code == ecf8.E_ARG


def test_a_table_of_one_column():
    table = torch.arange(12, dtype=torch.int32).view(3, 4).t()[:, :1]           # the next column, if there were one, would be 4 on
    assert table.stride() == (1, 4)
    b = ecfa.Batch(table, torch.ones(4, dtype=torch.int32))
    assert b.c.table_stride == 1 and b.c.table_width == 1
    with pytest.raises(ecf8.Ecf8Error):
        ecfa.Batch(torch.arange(12, dtype=torch.int32).view(3, 4).t()[:, :2], torch.ones(4, dtype=torch.int32))


def test_counts_that_32_bits_would_change():
    """ctypes keeps the lower 32 bits of a number and says nothing."""
    for rot in (0, -2, -64, 3, (1 << 32) + 64):
        with pytest.raises(ecf8.Ecf8Error) as e:
            ecfa.rope_freq(rot, device="cpu")
        assert e.value.code == ecf8.E_ARG
    table, lens, start = (torch.zeros(s, dtype=torch.int32) for s in ((2, 4), (2,), (3,)))
    for more in (dict(n_tokens=-1), dict(n_tokens=(1 << 32) + 2), dict(n_tokens=2, max_q=-1), dict(n_tokens=2, max_kv=1 << 32)):
        with pytest.raises(ecf8.Ecf8Error) as e:
            ecfa.Batch(table, lens, start, **more)
        assert e.value.code == ecf8.E_ARG
