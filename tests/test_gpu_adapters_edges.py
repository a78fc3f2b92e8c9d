"""Adapters and their gradients at the ends of their ranges: nothing of the rank, many rows of one adapter, very long
rows, memory that is shared, tensors' versions, the largest values."""
import pytest

import _adapt as ref
from _gpu import ct
from test_gpu_adapters import check, check_grad, like, made

pytestmark = pytest.mark.gpu

CODE = {"float32": 0, "float16": 1, "bfloat16": 2}


@pytest.mark.parametrize("wt", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("t", [5, 300])
def test_rank_0_leaves_what_it_is_added_to(t, wt):
    """Through the C entries, with a workspace that holds NaN: nothing of it goes into a result."""
    import torch
    c, count, k, n = ct(), 2, 64, 48
    dt = getattr(torch, wt)
    x, a = like(t, k, wt, 1), torch.zeros(count, 0, k, dtype=dt, device="cuda")
    b = torch.ones(count, n, 8, dtype=dt, device="cuda")[:, :, :0]       # columns of a wider matrix
    ids = torch.arange(t, device="cuda") % count
    work = torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for out in (wt, "float32"):
        y, dx = like(t, n, out, 2), like(t, k, out, 3)
        got, into = y.clone(), dx.clone()
        weights = (a.data_ptr(), a.stride(0), a.stride(1), b.data_ptr(), b.stride(0), b.stride(1), CODE[wt], ids.data_ptr(), None, t, count, 0, k, n)
        assert c.lib().ct_adapters(got.data_ptr(), CODE[out], n, x.data_ptr(), CODE[wt], k, *weights, 0, work.data_ptr(), 1 << 20, stream) == 0
        assert torch.equal(got, y)
        dy = like(t, n, wt, 4)
        assert c.lib().ct_adapters_grad(dy.data_ptr(), CODE[wt], n, x.data_ptr(), CODE[wt], k, *weights, into.data_ptr(), CODE[out], k, None, None,
                                        CODE[wt], work.data_ptr(), 1 << 20, stream) == 0
        assert torch.equal(into, dx)


def test_many_equal_rows_of_one_adapter_among_many():
    """Sums of equal positive terms, in which each addition could be rounded the same way: all rows have one adapter of so many that the kernel
    for a few rows an adapter takes them."""
    import torch
    c = ct()
    for t, count in ((8192, 512), (65536, 4096)):
        v = 1.0 + 2.0 ** -12 * (1 - 2.0 ** -8)      # just under half a step more, from 4096 on
        x = torch.full((t, 8), v, device="cuda")
        a, b = torch.zeros(count, 2, 8, device="cuda"), torch.zeros(count, 12, 2, device="cuda")
        a[7, :, 0], b[7, 0] = 1.0, 1.0
        dy = torch.zeros(t, 12, device="cuda")
        dy[:, 0] = 1.0
        ids = torch.full((t,), 7, device="cuda")
        _, da, db = c.ct_adapters_grad(dy, x, a, b, ids)
        # u = 1 and A x = v for every row: t v in every place that is not 0
        bound = (ref.UNIT * ref.steps(t) + ref.PARTS["float32"] + ref.HALF["float32"]) * t * v
        for got in (da[7], db[7, 0]):
            assert (got.double() - t * v).abs().max() <= bound
        assert (db[7, 1:] == 0).all() and (da[:7] == 0).all() and (db[8:] == 0).all()


@pytest.mark.parametrize("t", [1, 3, 40])
def test_few_rows_of_very_many_columns(t):
    """More columns than 65535 blocks of 128 have."""
    import torch
    n = 128 * 65535 + 77
    x, a = like(t, 16, "bfloat16", 1), like(8, 16, "bfloat16", 2).view(8, 1, 16)
    b = torch.zeros(8, n, 1, dtype=torch.bfloat16, device="cuda")
    b[:, ::1000003] = 1.0
    b[:, -1] = 2.0
    y = torch.zeros(t, n, dtype=torch.float32, device="cuda")
    ids = torch.arange(t, device="cuda") % 8
    v = (x.double() * a[ids, 0].double()).sum(dim=1)
    ct().ct_adapters(y, x, a, b, ids)
    want = torch.zeros(t, n, device="cuda")
    want[:, ::1000003] = 1.0
    want[:, -1] = 2.0
    bound = (ref.UNIT * ref.steps(16) + ref.PARTS["float32"]) * 2 * (x.double() * a[ids, 0].double()).abs().sum(dim=1)
    for r in range(t):
        at = torch.nonzero(want[r])[:, 0]
        assert torch.equal(torch.nonzero(y[r])[:, 0], at) or float(v[r]) == 0
        assert (y[r, at].double() - want[r, at].double() * v[r]).abs().max() <= bound[r]


def test_tensors_that_share_memory():
    """dx is written while x, dy and a are still to be read: it may lie beside them in one matrix, but not on them."""
    import torch
    c = ct()
    for t in (20, 300):
        x, a, b, ids, scale = made(t, 24, 40, 4, 2, "float32", "float32")
        y = like(t, 40, "float32", 1)
        for dx in (x, x[:, :24]):
            with pytest.raises(c.CtError):
                c.ct_adapters_grad(y, x, a, b, ids, scale, dx=dx)
        big = torch.zeros(t, 100, device="cuda")
        dy, x2, dx = big[:, :40].copy_(y), big[:, 40:64].copy_(x), big[:, 64:88].copy_(like(t, 24, "float32", 2))
        with pytest.raises(c.CtError):
            c.ct_adapters_grad(dy, x2, a, b, ids, scale, dx=big[:, 39:63])
        with pytest.raises(c.CtError):
            c.ct_adapters_grad(dy, x2, a, b, ids, scale, dx=big[:, 63:87])
        with pytest.raises(c.CtError):
            c.ct_adapters_grad(dy[:-1], x2[:-1], a, b, ids[:-1], scale, dx=big[1:, 30:54])
        with pytest.raises(c.CtError):
            c.ct_adapters(big[:, 8:48], x, a, big.view(-1)[:320].view(2, 40, 4), ids, scale)
        before = dx.clone()
        check_grad(dy, x2, a, b, ids, scale, before, c.ct_adapters_grad(dy, x2, a, b, ids, scale, dx=dx))
        assert (big[:, 88:] == 0).all()
        # rows of different pitches in one store, one behind the other's values
        store = torch.zeros(4 * t, 32, device="cuda")
        x3, dx3 = store[::2][:t, :24].copy_(x), store[1::2][:t, 4:28].copy_(before)
        check_grad(y, x3, a, b, ids, scale, before, c.ct_adapters_grad(y, x3, a, b, ids, scale, dx=dx3))
        x4, dx4 = store[::4][:t, :24].copy_(x), store[1::2][:t, 8:32].copy_(before)
        check_grad(y, x4, a, b, ids, scale, before, c.ct_adapters_grad(y, x4, a, b, ids, scale, dx=dx4))
        with pytest.raises(c.CtError):
            c.ct_adapters_grad(y, store[::4][:t, :24], a, b, ids, scale, dx=store[::2][:t, 8:32])


def test_y_that_is_x():
    """x has been read before y is written: a layer that adds to its own input."""
    for t in (3, 300):
        x, a, b, ids, scale = made(t, 64, 64, 8, 3, "bfloat16", "bfloat16")
        y = x.clone()
        assert (ct().ct_adapters(y, y, a, b, ids, scale) == ct().ct_adapters(x.clone(), x, a, b, ids, scale)).all()


def test_results_in_place_raise_the_tensors_versions():
    """So that autograd notices where a graph still wants what was there."""
    import torch
    c = ct()
    for t in (4, 300):
        x, a, b, ids, scale = made(t, 32, 24, 4, 2, "float32", "float32")
        y, dx = like(t, 24, "float32", 1), like(t, 32, "float32", 2)
        at = y._version, dx._version, x._version
        c.ct_adapters(y, x, a, b, ids, scale)
        c.ct_adapters_grad(y, x, a, b, ids, scale, dx=dx)
        assert y._version == at[0] + 1 and dx._version == at[1] + 1 and x._version == at[2]
        c.ct_adapters(y, x, a, b, ids, scale, stream=torch.cuda.Stream())
        assert y._version == at[0] + 2
        torch.cuda.synchronize()
        w = torch.ones(t, 24, device="cuda", requires_grad=True)
        loss = (w * y).sum()
        with torch.no_grad():
            c.ct_adapters(y, x, a, b, ids, scale)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        z = torch.zeros(4, 24, device="cuda")
        c.ct_adapters(z, x[:4].clone(), a, b, ids[:4].clone(), scale)
    c.ct_adapters(z, x[:4], a, b, ids[:4], scale)                       # no version to raise


@pytest.mark.parametrize("xt,wt", [("float32", "float32"), ("float32", "float16"), ("float32", "bfloat16")])
@pytest.mark.parametrize("t", [6, 300])
def test_the_largest_values_stay_finite(t, xt, wt):
    """The largest finite FP32 values are nearer to infinity than to any smaller BF16 value: their products with small numbers are finite."""
    import torch
    c, k, n, rank = ct(), 40, 24, 4
    top = torch.finfo(torch.float32).max
    small, a, b, ids, scale = made(t, k, n, rank, 3, xt, wt)
    ids.clamp_(min=0)
    x = small.clone()
    x[:, 3], x[1, 7], x[:, 11] = top, -top, top * (1 - 2.0 ** -9)
    a *= 2.0 ** -10
    b *= 2.0 ** -10
    for yt in ("float32", wt) if wt != "float16" else ("float32",):
        y = like(t, n, yt, 1)
        got = c.ct_adapters(y.clone(), x, a, b, ids, scale)
        assert got.isfinite().all()
        check(y, x, a, b, ids, scale, False, got)
    small_dy = like(t, n, "float32", 3) * 2.0 ** -20
    dy = small_dy.clone()
    dy[2, 5], dy[:, 9] = -top, top
    dx = like(t, k, "float32", 4)
    for g, h in ((dy, small * 2.0 ** -20), (small_dy, x)):
        got = c.ct_adapters_grad(g, h, a, b, ids, scale, dx=dx.clone(), grad_dtype=torch.float32)
        assert all(v.isfinite().all() for v in got)
        check_grad(g, h, a, b, ids, scale, dx, got)


@pytest.mark.parametrize("t", [6, 300])
def test_the_largest_weights_and_vectors_stay_finite(t):
    import torch
    c, k, n, rank = ct(), 40, 24, 4
    top = torch.finfo(torch.float32).max
    x = torch.zeros(t, k, device="cuda")
    x[:, 3] = 1.0
    x[1, 3] = -1.0
    a = like(rank, k, "float32", 1).view(1, rank, k) * 2.0 ** -10
    a[0, 1, 3], a[0, 2, 3] = top, -top                  # v is as large
    b = like(n, rank, "float32", 2).view(1, n, rank) * 2.0 ** -10
    y = like(t, n, "float32", 1)
    got = c.ct_adapters(y.clone(), x, a, b)
    assert got.isfinite().all()
    check(y, x, a, b, None, None, False, got)
    dy, dx = like(t, n, "float32", 3) * 2.0 ** -20, torch.zeros(t, k, device="cuda")
    got = c.ct_adapters_grad(dy, x, a, b, dx=dx.clone())
    assert all(g.isfinite().all() for g in got)
    check_grad(dy, x, a, b, None, None, dx, got)
