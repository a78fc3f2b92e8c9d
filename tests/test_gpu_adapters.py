"""Low-rank adapters and their gradients against the definition in 64 bits: types, odd sizes, pitches, ids in any order,
rows without an adapter, ids out of range, shared matrices, streams and graphs."""
import math

import numpy as np
import pytest

import _adapt as ref
from _gpu import ct

pytestmark = pytest.mark.gpu

PAIRS = [("float32", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"), ("float32", "float16"), ("float32", "bfloat16")]
# rows, k, n, rank, adapters
SIZES = [(1, 16, 10, 1, 1), (1, 4096, 512, 16, 8), (3, 257, 129, 5, 4), (17, 64, 64, 8, 17), (33, 1000, 31, 20, 3), (64, 128, 256, 16, 64),
         (130, 72, 264, 64, 1), (200, 520, 1000, 128, 2), (257, 320, 96, 33, 5), (700, 136, 200, 32, 3), (1500, 48, 40, 4, 2)]
# rows that can be copied as they lie, the long axes shared by several CTAs
WHOLE = [(300, 4104, 72, 16, 1), (400, 1032, 136, 8, 3), (129, 8, 2056, 24, 2), (3000, 136, 264, 64, 2), (150, 2120, 648, 128, 1), (2000, 520, 24, 40, 300), (300, 72, 520, 16, 40)]


def np64(t):
    return t.detach().double().cpu().numpy()


def made(t, k, n, rank, count, xt, wt, seed=0, bare=0.1, pad=0):
    """x, a, b, ids, scale; matrices with `pad` columns more than they show."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = lambda s: getattr(torch, s)  # noqa: E731

    def mat(*shape):
        v = torch.randn(*shape[:-1], shape[-1] + pad, generator=g)
        return v
    x = (mat(t, k) * torch.exp(0.5 * torch.randn(t, 1, generator=g))).to(dt(xt)).cuda()[:, pad // 2:pad // 2 + k]
    a = (mat(count, rank, k) * max(k, 1) ** -0.5).to(dt(wt)).cuda()[:, :, pad // 2:pad // 2 + k]
    b = mat(count, n, rank).to(dt(wt)).cuda()[:, :, pad // 2:pad // 2 + rank]
    ids = torch.randint(0, max(count, 1), (t,), generator=g)
    ids[torch.rand(t, generator=g) < bare] = -1
    return x, a, b, ids.cuda(), (torch.rand(count, generator=g) + 0.5).cuda()


def like(t, n, dtype, seed, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn(t, n + pad, generator=g).to(getattr(torch, dtype)).cuda()[:, pad // 2:pad // 2 + n]


def check(y, x, a, b, ids, scale, relu, got):
    want, mag, part = ref.adapters(np64(y), np64(x), np64(a), np64(b), None if ids is None else ids.cpu().numpy(),
                                   None if scale is None else np64(scale), relu)
    err = np.abs(np64(got) - want)
    lost = np.isnan(want)
    assert (np.isnan(np64(got)) == lost).all()
    assert (err <= ref.adapters_bound(want, mag, part, x.shape[1], a.shape[1], got.dtype))[~lost].all(), \
        (err / ref.adapters_bound(want, mag, part, x.shape[1], a.shape[1], got.dtype))[~lost].max()


def check_grad(dy, x, a, b, ids, scale, dx, got):
    want, mag = ref.adapters_grad(np64(dy), np64(x), np64(a), np64(b), None if ids is None else ids.cpu().numpy(),
                                  None if scale is None else np64(scale), np64(dx))
    t, k, n, rank = x.shape[0], x.shape[1], dy.shape[1], a.shape[1]
    for g, w, m, lengths in zip(got, want, mag, ((n, rank), (n, t), (k, t))):
        err, bound = np.abs(np64(g) - w), ref.grad_bound(w, m, lengths, g.dtype)
        lost = np.isnan(w)
        assert (np.isnan(np64(g)) == lost).all()
        assert (err <= bound)[~lost].all(), (err / bound)[~lost].max()


@pytest.mark.parametrize("xt,wt", PAIRS)
@pytest.mark.parametrize("size", SIZES)
def test_adapters(size, xt, wt):
    import torch
    t, k, n, rank, count = size
    for yt, relu, pad in ((wt, False, 0), ("float32", True, 0), (wt, True, 7), ("float32", False, 8)):
        x, a, b, ids, scale = made(t, k, n, rank, count, xt, wt, pad=pad)
        y = like(t, n, yt, 1, pad)
        whole = torch.full((t, n + pad), 7.0, dtype=y.dtype, device="cuda")
        got = whole[:, pad // 2:pad // 2 + n].copy_(y)
        assert ct().ct_adapters(got, x, a, b, ids, scale, relu=relu) is got
        check(y, x, a, b, ids, scale, relu, got)
        assert (whole[:, :pad // 2] == 7).all() and (whole[:, pad // 2 + n:] == 7).all()
        if not relu:
            assert (got[ids == -1] == y[ids == -1]).all()


@pytest.mark.parametrize("xt,wt", PAIRS)
@pytest.mark.parametrize("size", SIZES)
def test_gradients(size, xt, wt):
    import torch
    t, k, n, rank, count = size
    for gt, dxt, pad in ((wt, wt, 0), ("float32", "float32", 0), (wt, "float32", 5), ("float32", wt, 8)):
        x, a, b, ids, scale = made(t, k, n, rank, count, xt, wt, seed=2, pad=pad)
        dy = like(t, n, gt, 3, pad)
        dx = like(t, k, dxt, 4, pad)
        into = torch.zeros(t, k + pad, dtype=dx.dtype, device="cuda")[:, pad // 2:pad // 2 + k].copy_(dx)
        got = ct().ct_adapters_grad(dy, x, a, b, ids, scale, dx=into, grad_dtype=torch.float32 if gt == "float32" else None)
        assert got[0] is into and got[1].shape == a.shape and got[2].shape == b.shape
        check_grad(dy, x, a, b, ids, scale, dx, got)
        assert (into[ids == -1] == dx[ids == -1]).all()
        alone = ct().ct_adapters_grad(dy, x, a, b, ids, scale, grad_dtype=torch.float32 if gt == "float32" else None)
        assert alone[0] is None and (alone[1] == got[1]).all() and (alone[2] == got[2]).all()


@pytest.mark.parametrize("wt", ["bfloat16", "float16"])
@pytest.mark.parametrize("size", WHOLE)
def test_whole_rows(size, wt):
    import torch
    t, k, n, rank, count = size
    x, a, b, ids, scale = made(t, k, n, rank, count, wt, wt, seed=6)
    y = like(t, n, "float16", 1)
    check(y, x, a, b, ids, scale, False, ct().ct_adapters(y.clone(), x, a, b, ids, scale))
    for dt in (wt, "float32"):
        y, dx = like(t, n, dt, 1), like(t, k, dt, 4)
        for relu in (False, True):
            check(y, x, a, b, ids, scale, relu, ct().ct_adapters(y.clone(), x, a, b, ids, scale, relu=relu))
        dy = like(t, n, wt, 3)
        got = ct().ct_adapters_grad(dy, x, a, b, ids, scale, dx=dx.clone(), grad_dtype=getattr(torch, dt))
        check_grad(dy, x, a, b, ids, scale, dx, got)
    assert ct().ct_ops_device_error() == 0


def test_many_rows_of_one_adapter_among_many_adapters():
    """Rows enough for one adapter of many: the kernels for few rows an adapter on many of one."""
    import torch
    x, a, b, ids, scale = made(700, 136, 300, 12, 64, "bfloat16", "bfloat16", seed=4)
    ids[ids > 2] = 7
    dx = like(700, 136, "float32", 4)
    dy = like(700, 300, "bfloat16", 3)
    check_grad(dy, x, a, b, ids, scale, dx, ct().ct_adapters_grad(dy, x, a, b, ids, scale, dx=dx.clone(), grad_dtype=torch.float32))


def test_gradients_agree_with_differences():
    """The loss sum(dy * y) is linear in each of a, b and x, so a difference over any step gives its slope; in 64 bits of the
    definition the slope is exact to 1e-9, the kernel's gradient to its bound."""
    import torch
    t, k, n, rank, count = 40, 24, 18, 4, 3
    x, a, b, ids, scale = made(t, k, n, rank, count, "float32", "float32", seed=9)
    dy, dx = like(t, n, "float32", 5), torch.zeros(t, k, device="cuda")
    got = ct().ct_adapters_grad(dy, x, a, b, ids, scale, dx=dx)
    X, A, B, I, S, D = np64(x), np64(a), np64(b), ids.cpu().numpy(), np64(scale), np64(dy)
    loss = lambda X, A, B: (D * ref.adapters(np.zeros((t, n)), X, A, B, I, S, False)[0]).sum()  # noqa: E731
    _, mag = ref.adapters_grad(D, X, A, B, I, S, np.zeros((t, k)))
    rng = np.random.default_rng(0)
    for which, (g, m, lengths) in enumerate(zip(got, mag, ((n, rank), (n, t), (k, t)))):
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in g.shape)
            args = [X.copy(), A.copy(), B.copy()]
            args[which][at] += 0.5
            up = loss(*args)
            args[which][at] -= 1.0
            slope = up - loss(*args)
            assert abs(float(g[at]) - slope) <= ref.grad_bound(slope, m[at], lengths, torch.float32) + 1e-9, (which, at)


@pytest.mark.parametrize("wt", ["float32", "float16", "bfloat16"])
def test_one_adapter_without_ids(wt):
    import torch
    for t in (1, 100, 300):
        x, a, b, _, scale = made(t, 136, 72, 12, 1, wt, wt)
        y = like(t, 72, wt, 1)
        got = ct().ct_adapters(y.clone(), x, a, b)
        check(y, x, a, b, None, None, False, got)
        ids = torch.zeros(t, dtype=torch.int64, device="cuda")
        assert (ct().ct_adapters(y.clone(), x, a, b, ids) == got).all()
        dx = like(t, 136, wt, 2)
        into = dx.clone()
        check_grad(y, x, a, b, None, scale, dx, ct().ct_adapters_grad(y, x, a, b, None, scale, dx=into))


@pytest.mark.parametrize("t", [5, 300])
def test_ids_out_of_range_and_infinities_stay_in_their_rows(t):
    import torch
    x, a, b, ids, scale = made(t, 64, 48, 8, 3, "bfloat16", "bfloat16", bare=0)
    ids[0], ids[2] = 3, -2
    ids[3] = -1
    y = like(t, 48, "bfloat16", 1)
    x2 = x.clone()
    x2[1, 5], x2[3, 7] = math.inf, math.nan          # row 3 has no adapter: its x is not looked at
    got = ct().ct_adapters(y.clone(), x2, a, b, ids, scale)
    want = ct().ct_adapters(y.clone(), x, a, b, ids, scale)
    assert got[0].isnan().all() and got[2].isnan().all() and not got[1].isfinite().any() and (got[3] == y[3]).all()
    assert (got[4:] == want[4:]).all()
    dx = torch.zeros(t, 64, device="cuda")
    bad_dy = y.clone()
    bad_dy[0], bad_dy[2], bad_dy[3] = math.nan, math.inf, math.nan
    _, da, db = ct().ct_adapters_grad(bad_dy, x, a, b, ids, scale, dx=dx)
    assert dx[0].isnan().all() and dx[2].isnan().all() and (dx[3] == 0).all() and dx[4:].isfinite().all()
    _, da2, db2 = ct().ct_adapters_grad(y, x, a, b, ids, scale)
    assert (da == da2).all() and (db == db2).all()
    # an adapter with a NaN loses its own rows only
    a2 = a.clone()
    a2[1, 2, 3] = math.nan
    got = ct().ct_adapters(y.clone(), x, a2, b, ids, scale)
    mine = ids == 1
    assert got[mine].isnan().all()
    rest = ~mine & (ids >= 0) & (ids < 3)
    assert (got[rest] == want[rest]).all()


def test_adapters_that_share_a_matrix():
    import torch
    x, a, b, ids, scale = made(50, 40, 24, 6, 1, "float16", "float16")
    ids = torch.randint(0, 4, (50,), device="cuda")
    scale = torch.rand(4, device="cuda") + 0.5
    wide = a.expand(4, 6, 40), b.expand(4, 24, 6)
    y = like(50, 24, "float16", 1)
    check(y, x, *wide, ids, scale, False, ct().ct_adapters(y.clone(), x, *wide, ids, scale))
    dx = torch.zeros(50, 40, device="cuda")
    check_grad(y, x, *wide, ids, scale, dx, ct().ct_adapters_grad(y, x, *wide, ids, scale, dx=dx.clone()))


@pytest.mark.parametrize("t,k,n,rank,count", [(0, 8, 8, 4, 2), (5, 0, 8, 4, 2), (5, 8, 0, 4, 2), (5, 8, 8, 0, 2), (300, 8, 8, 0, 2), (5, 8, 8, 4, 0)])
def test_nothing_of_a_size(t, k, n, rank, count):
    import torch
    x, a, b, ids, scale = made(t, k, n, rank, count, "float32", "float32")
    ids.fill_(-1 if count == 0 else 0)
    y = like(t, n, "float32", 1)
    got = ct().ct_adapters(y.clone(), x, a, b, ids, scale, relu=True)
    assert (got == y.clamp(min=0)).all()
    dx = like(t, k, "float32", 2)
    into = dx.clone()
    _, da, db = ct().ct_adapters_grad(y, x, a, b, ids, scale, dx=into)
    assert (into == dx).all() and (da == 0).all() and (db == 0).all()


def test_adapters_without_rows_get_zeros():
    import torch
    x, a, b, ids, scale = made(300, 40, 24, 6, 5, "bfloat16", "bfloat16")
    ids[ids == 3] = 1
    _, da, db = ct().ct_adapters_grad(like(300, 24, "bfloat16", 1), x, a, b, ids, scale)
    assert (da[3] == 0).all() and (db[3] == 0).all() and (da[1] != 0).any()
    ids.fill_(-1)
    _, da, db = ct().ct_adapters_grad(like(300, 24, "bfloat16", 1), x, a, b, ids, scale)
    assert (da == 0).all() and (db == 0).all()


@pytest.mark.parametrize("t", [7, 600])
def test_captured_and_replayed(t):
    import torch
    c = ct()
    x, a, b, ids, scale = made(t, 264, 136, 16, 3, "bfloat16", "bfloat16")
    y, dx = like(t, 136, "bfloat16", 1), like(t, 264, "float32", 2)

    def both(y, dx):
        out = c.ct_adapters(y, x, a, b, ids, scale, relu=True)
        return (out,) + c.ct_adapters_grad(y, x, a, b, ids, scale, dx=dx)

    y1, dx1 = y.clone(), dx.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(y1.clone(), dx1.clone())
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                          # two graphs, replayed one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = both(y1, dx1)
        graphs.append((g, outs))
    for seed in (5, 6):
        x2, _, _, ids2, _ = made(t, 264, 136, 16, 3, "bfloat16", "bfloat16", seed=seed)
        x.copy_(x2), ids.copy_(ids2)
        for g, outs in graphs:
            y1.copy_(y), dx1.copy_(dx)
            g.replay()
            want = both(y.clone(), dx.clone())
            torch.cuda.synchronize()
            for o, w in zip(outs, want):
                assert (o == w).all()


def test_streams_at_once():
    """Calls on several streams at a time, each with what it allocated itself."""
    import torch
    c = ct()
    work = []
    for i in range(4):
        t = (3, 200, 900, 64)[i]
        x, a, b, ids, scale = made(t, 512, 256, 16, 4, "float16", "float16", seed=i)
        y = like(t, 256, "float16", i)
        work.append((y, x, a, b, ids, scale, c.ct_adapters(y.clone(), x, a, b, ids, scale), c.ct_adapters_grad(y, x, a, b, ids, scale)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(5):
        outs = []
        for s, (y, x, a, b, ids, scale, _, _) in zip(streams, work):
            z = y.clone()
            s.wait_stream(torch.cuda.current_stream())
            outs.append((c.ct_adapters(z, x, a, b, ids, scale, stream=s), c.ct_adapters_grad(y, x, a, b, ids, scale, stream=s.cuda_stream)))
        torch.cuda.synchronize()
        for (o, g), w in zip(outs, work):
            assert (o == w[6]).all() and (g[1] == w[7][1]).all() and (g[2] == w[7][2]).all()


def test_offsets_beyond_32_bits():
    """Rows whose pitch puts the later ones more than 2^31 values behind the first."""
    import torch
    ld = (1 << 30) + 8
    store = torch.zeros(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    x, a, b, ids, scale = made(3, 64, 48, 8, 2, "bfloat16", "bfloat16")
    far = store.as_strided((3, 64), (ld, 1)).copy_(x)
    y = like(3, 48, "bfloat16", 1)
    assert (ct().ct_adapters(y.clone(), far, a, b, ids, scale) == ct().ct_adapters(y.clone(), x, a, b, ids, scale)).all()
    g, w = ct().ct_adapters_grad(y, far, a, b, ids, scale), ct().ct_adapters_grad(y, x, a, b, ids, scale)
    assert (g[1] == w[1]).all() and (g[2] == w[2]).all()
    yfar = store.as_strided((3, 48), (ld, 1)).copy_(y)
    assert (ct().ct_adapters(yfar, x, a, b, ids, scale) == ct().ct_adapters(y.clone(), x, a, b, ids, scale)).all()


def test_refusals():
    import torch
    c = ct()
    x, a, b, ids, scale = made(4, 16, 8, 2, 3, "float16", "float16")
    y = like(4, 8, "float16", 1)
    for bad in (lambda: c.ct_adapters(y, x, a, b), lambda: c.ct_adapters(y[:3], x, a, b, ids), lambda: c.ct_adapters(y, x.bfloat16(), a, b, ids),
                lambda: c.ct_adapters(y, x, a.float(), b, ids), lambda: c.ct_adapters(y, x, a, b[:, :, :1], ids),
                lambda: c.ct_adapters(y, x, a, b.transpose(1, 2).contiguous().transpose(1, 2), ids), lambda: c.ct_adapters(y, x[:, :8], a, b, ids),
                lambda: c.ct_adapters(y, x, a, b, ids.int()), lambda: c.ct_adapters(y, x, a, b, ids[:3]),
                lambda: c.ct_adapters(y, x, a, b, ids, scale.double()), lambda: c.ct_adapters(y, x, a, b, ids, scale[:2]),
                lambda: c.ct_adapters(y, x, a[0], b, ids), lambda: c.ct_adapters(y.cpu(), x, a, b, ids),
                lambda: c.ct_adapters(y, x, torch.zeros(3, 129, 16, dtype=torch.float16, device="cuda"),
                                      torch.zeros(3, 8, 129, dtype=torch.float16, device="cuda"), ids),
                lambda: c.ct_adapters_grad(y.bfloat16(), x, a, b, ids), lambda: c.ct_adapters_grad(y, x, a, b, ids, dx=x[:3]),
                lambda: c.ct_adapters_grad(y, x, a, b, ids, grad_dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(c.CtError):
        c.ct_adapters(y[:1].expand(4, 8), x, a, b, ids)               # rows of y that lie on one another
    for who in ("y", "x", "a", "b", "scale"):
        args = dict(y=y.clone(), x=x, a=a, b=b, scale=scale)
        args[who] = args[who].detach().clone().requires_grad_()
        with pytest.raises(ValueError, match=who + r".*gradient"):
            c.ct_adapters(args["y"], args["x"], args["a"], args["b"], ids, args["scale"])
