"""Argument checks of the 8-bit answer head that need no device: the C entry
points refuse before any CUDA call, the binding before the library's."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ct():
    from paper_2609_16742_gb300 import build
    build.build()
    import paper_2609_16742_gb300 as ct
    return ct


A, B, C, D = 0x10000, 0x20000, 0x30000, 0x40000       # addresses that are never dereferenced


def test_quantize(ct):
    f = ct.lib().ct_fp8_quantize
    good = [A, 0, 4, 64, 64, 1, B, 64, C, 1, 4, None]

    def call(**kw):
        names = ["x", "dtype", "m", "k", "ldx", "rows", "q", "ldq", "s", "sr", "sb", "stream"]
        return f(*[kw.get(n, v) for n, v in zip(names, good)])

    assert call(dtype=3) == 1 and call(dtype=-1) == 1 and call(rows=2) == 1 and call(rows=0) == 1
    assert call(x=None) == 1 and call(q=None) == 1 and call(s=None) == 1
    assert call(ldx=63) == 1 and call(ldq=63) == 1 and call(x=A + 2) == 1 and call(s=C + 1) == 1
    assert call(m=-1) == 5 and call(k=-1) == 5 and call(m=2 ** 62, k=2 ** 10, ldx=2 ** 10, ldq=2 ** 10) == 5
    assert call(m=0) == 0 and call(k=0, x=None) == 0


def test_products(ct):
    f = ct.lib().ct_fp8_matmul
    names = ["x", "ldx", "xs", "xr", "xb", "w", "ldw", "ws", "wr", "wb", "bias", "relu", "y", "yd", "ldy", "m", "n", "k", "st"]
    good = [A, 64, B, 1, 4, C, 64, D, 1, 1, None, 0, A, 0, 8, 4, 8, 64, None]

    def call(**kw):
        return f(*[kw.get(n, v) for n, v in zip(names, good)])

    for bad in (dict(yd=3), dict(ldy=7), dict(y=None), dict(y=A + 2), dict(x=None), dict(xs=None), dict(w=None), dict(ws=None),
                dict(ldx=63), dict(ldx=72), dict(ldw=48), dict(ldw=65), dict(x=A + 8), dict(w=C + 4), dict(bias=D + 2)):
        assert call(**bad) == 1, bad
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(m=2 ** 31), dict(k=2 ** 31, ldx=2 ** 31, ldw=2 ** 31)):
        assert call(**bad) == 5, bad
    assert call(m=0, x=None, y=None) == 0 and call(n=0, w=None) == 0

    g = ct.lib().ct_fp8_linear
    n = ctypes.c_size_t()
    assert ct.lib().ct_fp8_linear_workspace(4, 100, ctypes.byref(n)) == 0 and n.value >= 4 * 112 + 4 * 4
    assert ct.lib().ct_fp8_linear_workspace(-1, 100, ctypes.byref(n)) == 5
    assert ct.lib().ct_fp8_linear_workspace(1, 1, None) == 1
    good2 = [A, 0, 100, C, 112, D, 1, 1, None, 0, A, 0, 8, 4, 8, 100, B, 10000, None]
    assert g(*good2[:16], None, 10000, None) == 1
    assert g(*good2[:16], B, 4, None) == 2
    assert g(A, 7, *good2[2:]) == 1
    assert g(None, *good2[1:]) == 1
    assert g(A, 0, 99, *good2[3:]) == 1


def test_logprobs(ct):
    f = ct.lib().ct_logprobs
    names = ["x", "dtype", "ld", "ids", "rows", "vocab", "k", "lp", "h", "lse", "tl", "ti", "st"]
    good = [A, 0, 64, B, 4, 64, 2, C, C, C, D, D, None]

    def call(**kw):
        return f(*[kw.get(n, v) for n, v in zip(names, good)])

    for bad in (dict(dtype=9), dict(x=None), dict(ld=63), dict(ids=None), dict(h=None), dict(lse=None), dict(tl=None), dict(ti=None),
                dict(x=A + 2), dict(ids=B + 4), dict(ti=D + 4), dict(lse=C + 2)):
        assert call(**bad) == 1, bad
    for bad in (dict(k=33), dict(k=-1), dict(rows=-1), dict(vocab=-1), dict(vocab=2 ** 31, ld=2 ** 31), dict(rows=2 ** 31)):
        assert call(**bad) == 5, bad
    assert call(rows=0) == 0

    g = ct.lib().ct_logprobs_grad
    names = ["x", "dtype", "ld", "ids", "rows", "vocab", "lse", "h", "glp", "gh", "dx", "ldd", "st"]
    good = [A, 0, 64, B, 4, 64, C, C, C, C, D, 64, None]

    def call(**kw):
        return g(*[kw.get(n, v) for n, v in zip(names, good)])

    for bad in (dict(dtype=9), dict(x=None), dict(dx=None), dict(lse=None), dict(ids=None), dict(h=None), dict(ld=63), dict(ldd=63),
                dict(x=A + 2), dict(dx=D + 1), dict(lse=C + 2), dict(ids=B + 1)):
        assert call(**bad) == 1, bad
    assert call(rows=-1) == 5 and call(vocab=2 ** 31, ld=2 ** 31, ldd=2 ** 31) == 5
    assert call(rows=0) == 0 and call(vocab=0) == 0


def test_binding_refuses_host_tensors(ct):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64)
    v = torch.zeros(4)
    ids = torch.zeros(4, dtype=torch.int64)
    q = x.to(torch.float8_e4m3fn)
    for bad in (lambda: ct.ct_fp8_quantize(x), lambda: ct.ct_fp8_matmul(q, v[:, None], q, v[:1, None]),
                lambda: ct.ct_fp8_linear(x, q, v[:1, None]), lambda: ct.ct_logprobs(x, ids),
                lambda: ct.ct_logprobs_grad(x, ids, v, v, v, v)):
        with pytest.raises(ValueError):
            bad()
