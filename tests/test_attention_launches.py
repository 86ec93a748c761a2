"""What the attention calls accept, without a device: a library in front of the runtime's answers for it and counts the launches."""
from test_host_launches import run_on_shim

HEAD = r"""
from paper_2510_02676_amd import ecfa
at = 1 << 20                                                            # an address that nothing looks at
lib = ecfa._lib
def cache(k=(2048, 128, 64), v=(2048, 128, 64), pages=4, page=16, heads=2, dtype=ecfa.BF16):
    return ecfa._Cache(at, at, None, None, (ctypes.c_int64 * 3)(*k), (ctypes.c_int64 * 3)(*v), pages, page, heads, 64, dtype, 0)
def batch(tokens=3, seqs=2):
    return ecfa._Batch(at, at, at, 4, 4, seqs, tokens, 0, 0, 0)
def rows(token=256, head=64, heads=4, dtype=ecfa.BF16):
    return ecfa._Rows(at, token, head, heads, dtype)
def attend(c=None, b=None, q=None, out=None, opts=None):
    return lib.ecfa_attend(c or cache(), b or batch(), opts or ecfa._AttendOpts(0.1, 0, None, None, 1, 0), q or rows(), out or rows(), at, 1 << 40, None)
def append(c=None, b=None, q=None, k=None, v=None, out=None):
    return lib.ecfa_append(c or cache(), b or batch(), None, q or rows(), k or rows(128, heads=2), v or rows(128, heads=2), out or rows(), None)
def launched(rc):
    n, var("launches").value = var("launches").value, 0
    return rc, n
assert launched(attend()) == (0, 1) and launched(append()) == (0, 1)
"""

STRIDES = HEAD + r"""
one, A, E = batch(1, 1), ecf8.E_ALIGN, ecfa.E4M3
# between tokens, of which there is one, and between heads, of which there is one
for odd in (1, 257, -3, 0):
    assert launched(attend(b=one, q=rows(odd))) == (0, 1) and launched(attend(b=one, out=rows(odd))) == (0, 1)
    assert launched(attend(q=rows(odd))) == (A if odd else 0, 0 if odd else 1) and launched(attend(out=rows(odd))) == (A if odd else 0, 0 if odd else 1)
    alone = cache(heads=1)
    assert launched(attend(c=alone, q=rows(256, odd, 1), out=rows(256, odd, 1))) == (0, 1)
    assert launched(append(b=one, q=rows(odd), k=rows(odd, heads=2), v=rows(odd, heads=2), out=rows(odd))) == (0, 1)
    assert launched(append(c=alone, q=rows(256, odd, 1), k=rows(128, odd, 1), v=rows(128, odd, 1), out=rows(256, odd, 1))) == (0, 1)
    if odd:
        for more in (dict(q=rows(odd)), dict(k=rows(odd, heads=2)), dict(v=rows(odd, heads=2)), dict(out=rows(odd))):
            assert launched(append(**more)) == (A, 0)
    # of a cache: between pages, tokens and heads
    for dtype in (ecfa.BF16, E):
        for i, only in ((0, dict(pages=1)), (1, dict(page=1)), (2, dict(heads=1))):
            s = [2048, 128, 64]
            s[i] = odd
            for which in "kv":
                c = cache(**{which: s}, **only, dtype=dtype)
                assert launched(attend(c=c)) == (0, 1)
                assert launched(append(c=c, k=rows(128, heads=c.kv_heads), v=rows(128, heads=c.kv_heads))) == (0, 1)
                if odd:
                    assert launched(attend(c=cache(**{which: s}, dtype=dtype))) == (A, 0)
    for group in (0, 128):
        assert launched(lib.ecfa_quant(at, ecfa.BF16, 1, 256, odd, group, at, at, None)) == (0, 1)
        assert launched(lib.ecfa_quant(at, ecfa.BF16, 2, 256, odd, group, at, at, None)) == (A if odd else 0, 0 if odd else 1)
"""


def test_strides_that_lead_nowhere_do_not_count(tmp_path):
    run_on_shim(tmp_path, STRIDES)
