"""Argument checks of the adapters, clipping and verification that need no device: the C entry points refuse before any CUDA
call, the binding before the library's."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def ct():
    from paper_2609_16742_gb300 import build
    build.build()
    import paper_2609_16742_gb300 as ct
    return ct


A, B, C, D, E = 0x10000, 0x20000, 0x30000, 0x40000, 0x1000000       # addresses that are never dereferenced


def caller(f, names, good):
    return lambda **kw: f(*[kw.get(n, v) for n, v in zip(names, good)])


def test_adapters(ct):
    names = ["y", "yd", "ldy", "x", "xd", "ldx", "a", "aa", "ar", "b", "ba", "br", "d", "ids", "s", "t", "count", "rank", "k", "n", "relu", "w",
             "wb", "st"]
    good = [A, 0, 8, B, 1, 16, C, 64, 16, D, 32, 4, 1, E, E, 3, 2, 4, 16, 8, 0, E, 1 << 20, None]
    call = caller(ct.lib().ct_adapters, names, good)
    for bad in (dict(yd=3), dict(d=3), dict(d=-1), dict(xd=2), dict(xd=7), dict(d=0, xd=1), dict(y=None), dict(x=None), dict(a=None), dict(b=None),
                dict(ldy=7), dict(ldx=15), dict(ar=15), dict(br=3), dict(aa=-1), dict(ba=-64), dict(y=A + 2), dict(x=B + 1), dict(a=C + 1),
                dict(b=D + 1), dict(ids=E + 4), dict(s=E + 2), dict(w=None), dict(w=E + 8), dict(ids=None, count=0)):
        assert call(**bad) == 1, bad
    for bad in (dict(t=-1), dict(count=-1), dict(rank=129), dict(rank=-1), dict(k=-1), dict(n=-1), dict(t=2 ** 31), dict(k=2 ** 31, ldx=2 ** 31),
                dict(n=2 ** 31), dict(count=65535)):
        assert call(**bad) == 5, bad
    assert call(wb=0) == 2
    assert call(t=0, y=None, x=None) == 0 and call(n=0, y=None, b=None) == 0


def test_adapters_grad(ct):
    names = ["dy", "dyd", "lddy", "x", "xd", "ldx", "a", "aa", "ar", "b", "ba", "br", "d", "ids", "s", "t", "count", "rank", "k", "n", "dx", "dxd",
             "lddx", "da", "db", "gd", "w", "wb", "st"]
    good = [A, 1, 8, B, 1, 16, C, 64, 16, D, 32, 4, 1, E, E, 3, 2, 4, 16, 8, A, 0, 16, B, C, 1, E, 1 << 20, None]
    call = caller(ct.lib().ct_adapters_grad, names, good)
    for bad in (dict(dyd=2), dict(d=3), dict(xd=2), dict(gd=2), dict(dxd=3), dict(d=0, xd=0, dyd=0), dict(dy=None), dict(x=None), dict(a=None),
                dict(b=None), dict(da=None), dict(db=None), dict(lddy=7), dict(ldx=15), dict(lddx=15), dict(ar=15), dict(br=3), dict(dy=A + 1),
                dict(dx=A + 2), dict(da=B + 1), dict(db=C + 1), dict(ids=E + 1), dict(s=E + 1), dict(w=None), dict(w=E + 4)):
        assert call(**bad) == 1, bad
    for bad in (dict(t=-1), dict(rank=129), dict(k=2 ** 31, ldx=2 ** 31, lddx=2 ** 31), dict(count=65535)):
        assert call(**bad) == 5, bad
    assert call(wb=0) == 2
    assert call(t=0, count=0) == 0


@pytest.mark.parametrize("name", ["ct_adapters_workspace", "ct_adapters_grad_workspace"])
def test_adapters_workspace(ct, name):
    f, n = getattr(ct.lib(), name), ctypes.c_size_t()
    assert f(100, 3, 16, 64, 64, ctypes.byref(n)) == 0 and n.value >= 100 * 16 * 4
    assert f(100, 3, 16, 64, 64, None) == 1
    assert f(-1, 3, 16, 64, 64, ctypes.byref(n)) == 5 and f(1, 3, 129, 64, 64, ctypes.byref(n)) == 5
    assert f(0, 0, 0, 0, 0, ctypes.byref(n)) == 0


def table(*tensors):
    """(src, dst, rows, cols, ld_src, ld_dst, dtype) each."""
    flat = [v for t in tensors for v in t]
    return (ctypes.c_int64 * len(flat))(*flat), len(tensors)


def test_clip(ct):
    f, w = ct.lib().ct_clip_grads, ctypes.c_size_t()

    def call(*tensors, kind=0, limit=1.0, norms=A, norm=A, work=B, size=1 << 30):
        t, n = table(*tensors)
        return f(t, n, kind, limit, norms, norm, work, size, None)

    good = (C, C, 4, 10, 12, 12, 0)
    for kw in (dict(kind=2), dict(kind=-1), dict(limit=-1.0), dict(limit=math.nan), dict(norms=None), dict(norm=None), dict(norm=A + 1), dict(work=None),
               dict(work=B + 8)):
        assert call(good, **kw) == 1, kw
    for bad in ((None or 0, C, 4, 10, 12, 12, 0), (C, 0, 4, 10, 12, 12, 0), (C, C, 4, 10, 9, 9, 0), (C, C, 4, 10, 12, 14, 0), (C, C, 4, 10, 12, 12, 3),
                (C + 2, C + 2, 4, 10, 12, 12, 0), (C, C + 4, 4, 10, 12, 12, 0), (C, C + 160, 1, 41, 41, 41, 0)):
        assert call(bad) == 1, bad
    for bad in ((C, C, -1, 10, 12, 12, 0), (C, C, 1, -10, 12, 12, 0), (C, C, 1 << 40, 1 << 40, 1 << 40, 1 << 40, 0)):
        assert call(bad) == 5, bad
    assert call(good, size=15) == 2
    for other in ((C, C, 4, 10, 12, 12, 0), (C + 40, C + 40, 4, 3, 12, 12, 0), (C + 4 * 45, D, 1, 5, 5, 5, 0), (D, C + 4 * 45, 1, 5, 5, 5, 0),
                  (C + 4, C + 4, 30, 2, 13, 13, 0)):
        assert call(good, other) == 1, other
    g = ct.lib().ct_clip_grads_workspace
    assert g(2, 10 ** 9, ctypes.byref(w)) == 0 and 0 < w.value < 1 << 22
    assert g(2, 40, None) == 1 and g(-1, 40, ctypes.byref(w)) == 5 and g(1, -1, ctypes.byref(w)) == 5


def test_verify(ct):
    names = ["x", "d", "ld", "q", "ldq", "ids", "off", "u", "e", "lde", "t", "b", "m", "v", "most", "acc", "tok", "lp", "w", "wb", "st"]
    good = [A, 1, 64, B, 64, C, D, C, B, 64, D, 2, 3, 64, 2, A, B, C, E, 1 << 20, None]
    call = caller(ct.lib().ct_verify_drafts, names, good)
    for bad in (dict(d=3), dict(x=None), dict(ids=None), dict(off=None), dict(u=None), dict(e=None), dict(acc=None), dict(tok=None), dict(lp=None),
                dict(ld=63), dict(ldq=63), dict(lde=63), dict(x=A + 1), dict(q=B + 1), dict(ids=C + 4), dict(off=D + 4), dict(u=C + 2),
                dict(e=B + 2), dict(t=D + 1), dict(acc=A + 4), dict(tok=B + 4), dict(lp=C + 2), dict(w=None), dict(w=E + 8)):
        assert call(**bad) == 1, bad
    for bad in (dict(b=-1), dict(m=-1), dict(v=-1), dict(most=-1), dict(most=65), dict(v=2 ** 31, ld=2 ** 31, ldq=2 ** 31, lde=2 ** 31), dict(m=2 ** 31)):
        assert call(**bad) == 5, bad
    assert call(wb=0) == 2 and call(b=0) == 0
    f, n = ct.lib().ct_verify_drafts_workspace, ctypes.c_size_t()
    assert f(2, 3, 1000, 2, ctypes.byref(n)) == 0 and n.value > 0
    assert f(2, 3, 1000, 2, None) == 1 and f(2, 3, 1000, 65, ctypes.byref(n)) == 5


def test_binding_refuses_host_tensors(ct):
    torch = pytest.importorskip("torch")
    x, a, b, y = torch.zeros(4, 16), torch.zeros(2, 3, 16), torch.zeros(2, 8, 3), torch.zeros(4, 8)
    ids, off, e = torch.zeros(4, dtype=torch.int64), torch.tensor([0, 2]), torch.ones(1, 16)
    for bad in (lambda: ct.ct_adapters(y, x, a, b, ids), lambda: ct.ct_adapters_grad(y, x, a, b, ids), lambda: ct.ct_clip_grads([x], 1.0),
                lambda: ct.ct_clip_grads([], 1.0), lambda: ct.ct_verify_drafts(x[:3], ids[:2], off, 2, torch.zeros(2), e)):
        with pytest.raises(ValueError):
            bad()
