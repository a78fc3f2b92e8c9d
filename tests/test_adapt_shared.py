"""Memory that the adapters' operands share, refused before any CUDA call: what is written must not lie on what is read after it."""
import pytest

from test_adapt_args import caller, ct  # noqa: F401

# addresses that are never dereferenced, far from one another
Y, X, A, B, IDS, DX, DA, DB, W = (i << 28 for i in range(1, 10))


def grad(ct):  # noqa: F811
    names = ["dy", "dyd", "lddy", "x", "xd", "ldx", "a", "aa", "ar", "b", "ba", "br", "d", "ids", "s", "t", "count", "rank", "k", "n", "dx", "dxd",
             "lddx", "da", "db", "gd", "w", "wb", "st"]
    good = [Y, 1, 8, X, 1, 16, A, 64, 16, B, 32, 4, 1, IDS, None, 30, 2, 4, 16, 8, DX, 0, 16, DA, DB, 1, W, 1 << 20, None]
    return caller(ct.lib().ct_adapters_grad, names, good)


def test_gradients(ct):  # noqa: F811
    call = grad(ct)
    # 30 rows: x 960 bytes, dy 480, dx 1920, a 256, da 256, db 128
    for bad in (dict(dx=X), dict(dx=X + 956), dict(dx=X - 1916), dict(dx=Y), dict(dx=Y - 4), dict(dx=A + 252), dict(da=X), dict(da=Y + 478), dict(db=X + 958),
                dict(db=Y), dict(da=DX + 1916), dict(db=DX), dict(db=DA), dict(db=DA + 254), dict(da=DB + 126),
                # rows of one matrix whose columns lie on one another
                dict(dx=X + 28, lddx=20, ldx=40), dict(dx=X + 8, lddx=20, ldx=40, x=X),
                # rows of different pitches: x's 32 of every 128 bytes, dx's 32 of every 130, which meet in their last rows
                dict(dx=X + 42, dxd=1, lddx=65, ldx=64)):
        assert call(**bad) == 1, bad


def test_forward(ct):  # noqa: F811
    names = ["y", "yd", "ldy", "x", "xd", "ldx", "a", "aa", "ar", "b", "ba", "br", "d", "ids", "s", "t", "count", "rank", "k", "n", "relu", "w",
             "wb", "st"]
    good = [Y, 0, 8, X, 1, 16, A, 64, 16, B, 32, 4, 1, IDS, None, 30, 2, 4, 16, 8, 0, W, 1 << 20, None]
    call = caller(ct.lib().ct_adapters, names, good)
    # y 960 bytes, b 128, ids 240
    for bad in (dict(y=B), dict(y=B + 124), dict(y=B - 956), dict(y=IDS), dict(y=IDS + 236), dict(y=IDS - 956)):
        assert call(**bad) == 1, bad
