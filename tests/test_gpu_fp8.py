"""8-bit quantisation and block-scaled products against plain 64-bit
implementations.  Tolerances are derived, not fitted:
  - the quantiser rounds each value once (its scale is a power of two), so its
    outputs are compared for equality;
  - products: every FP32 addition and multiplication adds at most 2^-23 of
    the magnitudes it sums (also when it truncates), 128 of them inside a
    block, one per block, a few for scales and bias, so
    |error| <= (128 + blocks + 8) 2^-23 sum |x||w| + half a unit of y's type;
  - integer operands whose sums stay below 2^24 are exact."""
import numpy as np
import pytest

import _ops
from _gpu import ct

pytestmark = pytest.mark.gpu

HALF_UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}


def torch_():
    import torch
    return torch


def rand_fp8(rng, m, k, pad=0):
    """(device e4m3 tensor, its values): bytes drawn over all finite codes."""
    torch = torch_()
    b = rng.integers(0, 256, (m, k)).astype(np.uint8)
    b[(b & 0x7F) == 0x7F] = 0                                  # no NaN
    pitch = (k + 15) // 16 * 16 + pad
    d = torch.full((m, pitch), 0x7F, dtype=torch.uint8, device="cuda")[:, :k]   # NaN beyond k: must not be read as data
    d.copy_(torch.from_numpy(b))
    q = d.view(torch.float8_e4m3fn)
    return q, q.float().cpu().numpy().astype(np.float64)


def check_product(y, out, xv, wv, bias, relu, kb):
    ref = _ops.product(xv, wv, bias, relu)
    mag = np.abs(xv) @ np.abs(wv).T + (0 if bias is None else np.abs(bias))
    tol = (128 + kb + 8) * 2.0 ** -23 * mag + HALF_UNIT[out] * np.abs(ref) + TINY[out]
    err = np.abs(y.double().cpu().numpy() - ref)
    assert y.shape == ref.shape and (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 128), (3, 127), (5, 129), (130, 300), (257, 16), (64, 1000)])
def test_quantize_is_the_definition(dtype, block_rows, m, k):
    torch = torch_()
    rng = np.random.default_rng(m * 1000 + k)
    x = rng.standard_normal((m, k)) * np.exp(3 * rng.standard_normal((m, 1)))
    x[rng.random((m, k)) < 0.05] = 0.0
    x[0, 0] = 448.0                                            # the largest value: exactly scale 1 for a small row
    xt = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    q, s = ct().ct_fp8_quantize(xt, block_rows)
    torch.cuda.synchronize()
    qr, sr = _ops.quantize(xt.double().cpu().numpy(), block_rows)
    assert np.array_equal(s.cpu().numpy(), sr)
    np.testing.assert_array_equal(q.float().cpu().numpy(), qr)     # float16 rows may hold infinities: NaN on both sides
    assert q.stride(0) % 16 == 0 or m == 1


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_special_values(block_rows):
    torch = torch_()
    x = np.zeros((3, 400))
    x[0, 5], x[0, 6], x[0, 130], x[0, 131] = np.inf, 3.0, np.nan, -np.inf
    x[1, 0], x[1, 129], x[1, 300] = 1e-45, 3.4028e38, 2.0 ** -130
    x[2, 0], x[2, 1], x[2, 128], x[2, 256] = 449.0, 224.5, np.nextafter(np.float32(448), np.float32(500)), 2.0 ** -126
    xt = torch.from_numpy(x.astype(np.float32)).cuda()
    q, s = ct().ct_fp8_quantize(xt, block_rows)
    qr, sr = _ops.quantize(xt.double().cpu().numpy(), block_rows)
    assert np.array_equal(s.cpu().numpy(), sr)
    np.testing.assert_array_equal(q.float().cpu().numpy(), qr)


def test_quantize_strides_and_offsets():
    """Rows that start anywhere, wide pitches, given outputs, a scale order of
    the caller's; nothing outside the outputs is written."""
    torch = torch_()
    base = torch.randn(37, 1003, device="cuda").half()
    for lo, hi in [(0, 1003), (1, 700), (3, 4), (8, 1000)]:
        x = base[1:, lo:hi]
        m, k = x.shape
        qb = torch.full((m + 2, 1100), 7, dtype=torch.uint8, device="cuda")
        sb = torch.full((m, (k + 127) // 128, 2), -1.0, device="cuda")
        q, s = ct().ct_fp8_quantize(x, 1, q=qb[1:m + 1, 3:3 + k].view(torch.float8_e4m3fn), scale=sb[:, :, 0])
        qr, sr = _ops.quantize(x.double().cpu().numpy(), 1)
        assert np.array_equal(q.float().cpu().numpy(), qr) and np.array_equal(s.cpu().numpy(), sr)
        inside = torch.zeros_like(qb, dtype=torch.bool)
        inside[1:m + 1, 3:3 + k] = True
        assert (qb[~inside] == 7).all() and (sb[:, :, 1] == -1).all()


@pytest.mark.parametrize("m", [1, 2, 16, 17, 33, 64, 65, 128, 129, 256, 257, 400, 1000])
@pytest.mark.parametrize("n,k", [(1, 1), (10, 84), (129, 128), (1000, 512), (130, 1290), (300, 4096)])
def test_matmul_sizes(m, n, k):
    torch = torch_()
    rng = np.random.default_rng(m + 7 * n + 31 * k)
    xq, xv = rand_fp8(rng, m, k)
    wq, wv = rand_fp8(rng, n, k, pad=16)
    kb = (k + 127) // 128
    xs = np.exp(rng.standard_normal((m, kb))).astype(np.float32)
    ws = np.exp(rng.standard_normal(((n + 127) // 128, kb))).astype(np.float32)
    bias = rng.standard_normal(n).astype(np.float32)
    out = ["float32", "float16", "bfloat16"][(m + n) % 3]
    if out == "float16":
        xs *= 1e-4                                             # results within the type's range
        ws *= 1e-3
    relu = bool(k % 2)
    y = ct().ct_fp8_matmul(xq, torch.from_numpy(xs).cuda(), wq, torch.from_numpy(ws).cuda(),
                           bias=torch.from_numpy(bias).cuda(), relu=relu, out_dtype=getattr(torch, out))
    assert ct().ct_ops_device_error() == 0
    check_product(y, out, xv * _ops.widen(xs.astype(np.float64), 1, m, k), wv * _ops.widen(ws.astype(np.float64), 128, n, k),
                  bias.astype(np.float64), relu, kb)


@pytest.mark.parametrize("m", [1, 20, 50, 100, 256, 300, 700])
def test_matmul_long_k(m):
    """K long enough that every stage of the pipeline is used many times, on
    few tiles and on many, called back to back."""
    torch = torch_()
    rng = np.random.default_rng(m)
    for n, k in [(130, 30000), (4400, 9000)]:
        xq, xv = rand_fp8(rng, m, k)
        wq, wv = rand_fp8(rng, n, k)
        kb = (k + 127) // 128
        xs = torch.rand(m, kb, device="cuda")
        ws = torch.rand((n + 127) // 128, kb, device="cuda")
        ys = [ct().ct_fp8_matmul(xq, xs, wq, ws) for _ in range(20)]
        assert ct().ct_ops_device_error() == 0
        check_product(ys[0], "float32", xv * _ops.widen(xs.double().cpu().numpy(), 1, m, k),
                      wv * _ops.widen(ws.double().cpu().numpy(), 128, n, k), None, False, kb)
        assert all(torch.equal(y, ys[0]) for y in ys)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (8, 520, 4096), (200, 1000, 1152), (300, 516, 640), (1300, 770, 400)])
def test_matmul_exact_on_integers(m, n, k):
    """Small integers and power-of-two scales: every sum is exact, so all
    shapes give the exact result, twice the same."""
    torch = torch_()
    rng = np.random.default_rng(5)
    xv, wv = rng.integers(-4, 5, (m, k)).astype(np.float64), rng.integers(-4, 5, (n, k)).astype(np.float64)

    def dev(v):
        t = torch.zeros(v.shape[0], (k + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :k]
        t.copy_(torch.from_numpy(v).float())
        return t

    kb = (k + 127) // 128
    xs = 2.0 ** rng.integers(-1, 2, (m, kb))
    ws = 2.0 ** rng.integers(-1, 2, ((n + 127) // 128, kb))
    args = (dev(xv), torch.from_numpy(xs).float().cuda(), dev(wv), torch.from_numpy(ws).float().cuda())
    ref = (xv * _ops.widen(xs, 1, m, k)) @ (wv * _ops.widen(ws, 128, n, k)).T
    assert np.abs(ref).max() < 2 ** 22
    for _ in range(2):
        y = ct().ct_fp8_matmul(*args)
        assert np.array_equal(y.cpu().numpy(), ref)


@pytest.mark.parametrize("out", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("m,n,k", [(1777, 2999, 1300), (1100, 4001, 300), (2050, 3501, 130), (530, 9600, 256)])
@pytest.mark.parametrize("lo,pad", [(0, 0), (1, 2), (3, 5), (8, 0)])
def test_matmul_many_tiles_anywhere(out, m, n, k, lo, pad):
    """More tiles than the GPU takes at once, into a matrix whose rows start
    anywhere; nothing beside it is written.  Integers: exact before the one
    rounding to y's type."""
    torch = torch_()
    g = torch.Generator(device="cuda").manual_seed(n + lo)

    def ints(rows):
        v = torch.randint(-4, 5, (rows, k), device="cuda", generator=g)
        t = torch.zeros(rows, (k + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :k]
        t.copy_(v.float())
        return t, v.double()

    kb = (k + 127) // 128
    (xq, xv), (wq, wv) = ints(m), ints(n)
    xs = 2.0 ** torch.randint(-1, 2, (m, kb), device="cuda", generator=g).float()
    ws = 2.0 ** torch.randint(-1, 2, ((n + 127) // 128, kb), device="cuda", generator=g).float()
    big = torch.full((m + 1, lo + n + pad), 7.0, dtype=getattr(torch, out), device="cuda")
    y = ct().ct_fp8_matmul(xq, xs, wq, ws, out=big[:m, lo:lo + n])
    wide = lambda s, block, rows: s.double().repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :k]
    ref = (xv * wide(xs, 1, m)) @ (wv * wide(ws, 128, n)).T
    assert ref.abs().max() < 2 ** 22 and torch.equal(y, ref.float().to(y.dtype))
    assert ct().ct_ops_device_error() == 0
    assert (big[m] == 7).all() and (big[:m, :lo] == 7).all() and (big[:m, lo + n:] == 7).all()


@pytest.mark.parametrize("m", [3, 40, 300])
def test_matmul_strides_scale_orders_and_untouched_memory(m):
    torch = torch_()
    rng = np.random.default_rng(m)
    n, k = 261, 777
    xq, xv = rand_fp8(rng, m, k, pad=64)
    wq, wv = rand_fp8(rng, n, k)
    kb = (k + 127) // 128
    xs = torch.rand(kb, m, 3, device="cuda")[:, :, 1].t()       # [m, kb], strides (3, 3 m)
    ws = torch.rand(kb, (n + 127) // 128, device="cuda").t()
    for out in ("float32", "bfloat16"):
        buf = torch.full((m + 2, n + 5), 5.0, dtype=getattr(torch, out), device="cuda")
        for lo in (0, 1, 3):
            buf.fill_(5.0)
            y = ct().ct_fp8_matmul(xq, xs, wq, ws, out=buf[1:m + 1, lo:lo + n])
            check_product(y, out, xv * _ops.widen(xs.double().cpu().numpy(), 1, m, k),
                          wv * _ops.widen(ws.double().cpu().numpy(), 128, n, k), None, False, kb)
            buf[1:m + 1, lo:lo + n] = 5.0
            assert (buf == 5.0).all()


def test_matmul_nan_stays_in_its_rows_and_columns():
    torch = torch_()
    rng = np.random.default_rng(3)
    for m in (20, 300):
        n, k = 200, 300
        xq, xv = rand_fp8(rng, m, k)
        wq, wv = rand_fp8(rng, n, k)
        xq.view(torch.uint8)[7, 290] = 0x7F
        wq.view(torch.uint8)[150, 3] = 0xFF
        y = ct().ct_fp8_matmul(xq, torch.ones(m, 3, device="cuda"), wq, torch.ones(2, 3, device="cuda"), relu=True)
        want = np.zeros((m, n), bool)
        want[7], want[:, 150] = True, True
        assert np.array_equal(np.isnan(y.cpu().numpy()), want)


def test_sizes_of_zero():
    torch = torch_()
    c = ct()
    e8 = torch.float8_e4m3fn
    for m, n in [(0, 5), (5, 0), (0, 0)]:
        y = c.ct_fp8_matmul(torch.zeros(m, 16, device="cuda").to(e8), torch.ones(m, 1, device="cuda"),
                            torch.zeros(n, 16, device="cuda").to(e8), torch.ones((n + 127) // 128, 1, device="cuda"))
        assert y.shape == (m, n)
    b = torch.tensor([1.0, -2.0, float("nan")], device="cuda")
    for m in (2, 300):
        y = c.ct_fp8_linear(torch.empty(m, 0, device="cuda"), torch.empty(3, 0, device="cuda").to(e8),
                            torch.empty(1, 0, device="cuda"), bias=b, relu=True)
        assert (y[:, 0] == 1).all() and (y[:, 1] == 0).all() and y[:, 2].isnan().all()
    q, s = c.ct_fp8_quantize(torch.empty(0, 300, device="cuda"))
    assert q.shape == (0, 300) and s.shape == (0, 3)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("m,n,k", [(1, 1000, 4096), (5, 257, 129), (64, 300, 1024), (150, 10, 512), (513, 384, 260)])
def test_linear_is_quantize_then_matmul(dtype, m, n, k):
    """Bit for bit the two calls', whatever the shape; and near the product of
    the unquantised operands (each e4m3 value is within 2^-4 of its own)."""
    torch = torch_()
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn(m, k, device="cuda", generator=g).to(getattr(torch, dtype))
    w = torch.randn(n, k, device="cuda", generator=g) / k ** 0.5
    wq, ws = c.ct_fp8_quantize(w, 128)
    bias = torch.randn(n, device="cuda", generator=g)
    y = c.ct_fp8_linear(x, wq, ws, bias=bias)
    assert y.dtype == x.dtype
    q, s = c.ct_fp8_quantize(x)
    z = c.ct_fp8_matmul(q, s, wq, ws, bias=bias, out_dtype=x.dtype)
    assert torch.equal(y, z)
    ref = x.double() @ w.double().t() + bias.double()
    mag = x.double().abs() @ w.double().abs().t()
    assert ((y.double() - ref).abs() <= 0.13 * mag + 0.01 * ref.abs() + 1e-3).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 130, 5003), (7, 1000, 25088), (16, 128, 128), (17, 129, 127), (33, 64, 3000),
                                   (100, 500, 300), (256, 1000, 512), (500, 500, 500), (1000, 100, 1000)])
def test_linear_of_rows_anywhere(dtype, m, n, k):
    """The two calls' bits, from rows that start anywhere beside values that must
    not be read as theirs, with masked, empty and poisoned rows; called back to
    back."""
    torch = torch_()
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(m + k)
    base = torch.full((m, k + 9), float("nan"), device="cuda").to(getattr(torch, dtype))
    wq, ws = c.ct_fp8_quantize(torch.randn(n, k, device="cuda", generator=g), 128)
    bias = torch.randn(n, device="cuda", generator=g)
    for lo in (0, 1, 4, 8):
        x = base[:, lo:lo + k]
        x.copy_(torch.randn(m, k, device="cuda", generator=g))
        x[m // 2, :k // 2] = 0
        if m > 3:
            x[1], x[2, k // 3], x[3, k - 1] = 0, float("inf"), float("nan")
        z = c.ct_fp8_matmul(*c.ct_fp8_quantize(x), wq, ws, bias=bias, relu=True, out_dtype=x.dtype)
        for _ in range(5):
            y = c.ct_fp8_linear(x, wq, ws, bias=bias, relu=True)
            assert torch.equal(y.nan_to_num(7.0), z.nan_to_num(7.0)) and torch.equal(y.isnan(), z.isnan())
        assert c.ct_ops_device_error() == 0
        if m > 3:
            assert y[2:4].isnan().all() and not y[1].isnan().any()
        x.fill_(float("nan"))


def test_input_gradient_is_the_product_with_transposed_weights():
    """dx = dy W from the transposed 8-bit weights: the same numbers as the
    64-bit product with the weights the forward pass used, and the directional
    derivative of the layer that they imply."""
    torch = torch_()
    c = ct()
    rng = np.random.default_rng(8)
    n, k, m = 300, 200, 40
    wq, wv = rand_fp8(rng, n, k)
    ws = torch.rand(3, 2, device="cuda") * 0.01
    wv = wv * _ops.widen(ws.double().cpu().numpy(), 128, n, k)
    wt = torch.zeros(k, (n + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :n]
    wt.copy_(wq.view(torch.uint8).t())
    dyq, dyv = rand_fp8(rng, m, n)
    dys = torch.rand(m, 3, device="cuda")
    dyv = dyv * _ops.widen(dys.double().cpu().numpy(), 1, m, n)
    dx = c.ct_fp8_matmul(dyq, dys, wt, ws.t())
    check_product(dx, "float32", dyv, wv.T, None, False, 3)
    # d/dt of sum(dy * (x + t v) W^T) along v is sum(dx * v); the layer is linear, so any step shows it
    xq, xv = rand_fp8(rng, m, k)
    vq, vv = rand_fp8(rng, m, k)
    one = torch.ones(m, 2, device="cuda")
    f0 = (dyv * c.ct_fp8_matmul(xq, one * 0, wq, ws).double().cpu().numpy()).sum()
    f1 = (dyv * c.ct_fp8_matmul(vq, one, wq, ws).double().cpu().numpy()).sum()
    slope = (dx.double().cpu().numpy() * vv).sum()
    mag = (np.abs(dyv) * (np.abs(vv) @ np.abs(wv).T)).sum()
    assert abs((f1 - f0) - slope) <= 2 * (128 + 3 + 8) * 2.0 ** -23 * mag


def test_streams_of_the_callers():
    """Inputs made on a side stream, the call on that stream, interleaved with
    work on the default one: same bits as in order."""
    torch = torch_()
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(48, 1024, device="cuda", generator=g)
    wq, ws = c.ct_fp8_quantize(torch.randn(640, 1024, device="cuda", generator=g), 128)
    want = c.ct_fp8_linear(x, wq, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for i in range(8):
        with torch.cuda.stream(side):
            xi = x * 2.0
            got.append(c.ct_fp8_linear(xi, wq, ws))
        c.ct_fp8_linear(x, wq, ws)
        got.append(c.ct_fp8_linear(x, wq, ws, stream=torch.cuda.current_stream()))
    torch.cuda.synchronize()
    for i in range(8):
        assert torch.equal(got[2 * i], want * 2) and torch.equal(got[2 * i + 1], want)
    side.wait_stream(torch.cuda.current_stream())
    y = c.ct_fp8_linear(x, wq, ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)


def test_refusals():
    torch = torch_()
    c = ct()
    x = torch.zeros(4, 64, device="cuda")
    e8 = torch.float8_e4m3fn
    q, s = c.ct_fp8_quantize(x)
    w, ws = c.ct_fp8_quantize(x, 128)
    for bad in (lambda: c.ct_fp8_quantize(x.double()), lambda: c.ct_fp8_quantize(x.t()), lambda: c.ct_fp8_quantize(x, 64),
                lambda: c.ct_fp8_quantize(x[0]), lambda: c.ct_fp8_matmul(q, s, w[:, :32], ws),
                lambda: c.ct_fp8_matmul(q, s[:2], w, ws), lambda: c.ct_fp8_matmul(q.cpu(), s, w, ws),
                lambda: c.ct_fp8_matmul(q, s, w, ws, bias=torch.zeros(5, device="cuda")),
                lambda: c.ct_fp8_matmul(q, s, w, ws, out_dtype=torch.float64),
                lambda: c.ct_fp8_linear(x, w, ws, out=torch.zeros(4, 5, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    # operands that the copy engine cannot address
    raw = torch.zeros(4, 72, dtype=torch.uint8, device="cuda").view(e8)
    for bad in (lambda: c.ct_fp8_matmul(raw[:, :64], s, w, ws),            # pitch 72
                lambda: c.ct_fp8_matmul(torch.zeros(4, 80, dtype=torch.uint8, device="cuda")[:, 8:72].view(e8), s, w, ws)):
        with pytest.raises(c.CtError) as ei:
            bad()
        assert ei.value.status == 1
    assert c.ct_ops_device_error() == 0


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes of activations and of results: the rows at the end
    are the same as those rows alone."""
    torch = torch_()
    c = ct()
    m, n, k = 140000, 16400, 16000
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    x[-40:] = torch.randn(40, k, device="cuda", generator=g).bfloat16()
    q, s = c.ct_fp8_quantize(x)
    del x
    ql, sl = q[-40:].clone(), s[-40:].clone()
    w, ws = c.ct_fp8_quantize(torch.randn(n, k, device="cuda", generator=g), 128)
    y = c.ct_fp8_matmul(q, s, w, ws, out_dtype=torch.bfloat16)
    assert c.ct_ops_device_error() == 0
    assert q.numel() > 2 ** 31 and y.numel() > 2 ** 31
    assert (y[:-40] == 0).all()
    xv = ql.float().cpu().numpy().astype(np.float64) * _ops.widen(sl.double().cpu().numpy(), 1, 40, k)
    wv = w.float().cpu().numpy().astype(np.float64) * _ops.widen(ws.double().cpu().numpy(), 128, n, k)
    check_product(y[-40:], "bfloat16", xv, wv, None, False, (k + 127) // 128)
