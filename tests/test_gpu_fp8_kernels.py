"""Every kernel that a product or a linear layer can take, by sizes that take it
(asked of the library, so that another choice is noticed): ragged sizes, all
output types, rows of y that start anywhere.  Integers and power-of-two scales:
every sum is exact, so the result is, before its one rounding; what is
quantised in the launch has the two calls' bits."""
import ctypes

import numpy as np
import pytest

import _ops
from _gpu import ct
from test_gpu_fp8 import check_product

pytestmark = pytest.mark.gpu

# (m, n, k), (wide, columns of a tile), K split
PRODUCTS = [((711, 18, 711), (0, 16), False), ((203, 283, 2218), (0, 16), True), ((128, 49, 2932), (0, 16), True),
            ((17, 10781, 1658), (0, 32), False), ((107, 1271, 4664), (0, 32), True), ((351, 265, 5598), (0, 32), True),
            ((495, 2296, 82), (0, 64), False), ((1660, 328, 673), (0, 64), False), ((580, 408, 3957), (0, 64), True),
            ((42, 1824, 8091), (0, 64), True), ((1356, 1098, 251), (0, 128), False), ((700, 2000, 128), (0, 128), False),
            ((1568, 156, 5544), (0, 128), True), ((117, 5768, 4353), (0, 128), True),
            ((3000, 300, 1000), (1, 64), False), ((700, 1000, 2000), (1, 64), False), ((7269, 33, 5011), (1, 64), True),
            ((6838, 11, 5042), (1, 64), True), ((700, 2000, 1000), (1, 128), False), ((6499, 549, 402), (1, 128), False),
            ((1243, 796, 6318), (1, 128), True), ((3933, 197, 5705), (1, 128), True), ((417, 11892, 162), (1, 192), False),
            ((1818, 1626, 985), (1, 192), False), ((193, 16071, 167), (1, 256), False), ((3869, 2119, 427), (1, 256), False),
            ((182, 5321, 7519), (1, 256), True), ((6673, 149, 7341), (1, 256), True)]

# type of x, (m, n, k), columns of a tile, K split
LINEARS = [("float32", (259, 1422, 154), 32, False), ("float16", (259, 1422, 154), 32, False), ("bfloat16", (206, 2000, 154), 32, False),
           ("float32", (1330, 155, 214), 32, False), ("float32", (682, 41, 4402), 32, True), ("float16", (585, 42, 4575), 32, True),
           ("bfloat16", (833, 71, 2325), 32, True), ("float32", (67, 416, 1697), 16, True), ("float16", (147, 218, 3206), 16, True),
           ("bfloat16", (242, 20, 4653), 16, True), ("float32", (356, 67, 266), 16, False), ("float16", (59, 266, 534), 16, False),
           ("bfloat16", (55, 99, 1594), 16, False)]


def kernel(m, n, k, x_dtype=-1):
    """(quantises in the launch, wide, columns, splits)"""
    import torch
    torch.zeros(1, device="cuda")                              # the device is current
    f = ct().lib().ct_internal_fp8_kernel
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    got = (ctypes.c_int32 * 4)()
    assert f(m, n, k, x_dtype, got) == 0
    return tuple(got)


def test_the_lists_reach_every_kernel():
    kinds = {(w, s) for _, w, s in PRODUCTS}
    assert kinds == {((0, bn), s) for bn in (16, 32, 64, 128) for s in (False, True)} | \
        {((1, bn), s) for bn in (64, 128, 256) for s in (False, True)} | {((1, 192), False)}
    assert {(d, bn, s) for d, _, bn, s in LINEARS} == {(d, bn, s) for d in ("float32", "float16", "bfloat16") for bn in (16, 32)
                                                       for s in (False, True)}
    for size, (wide, bn), split in PRODUCTS:
        q, w, b, s = kernel(*size)
        assert (q, w, b, s > 1) == (0, wide, bn, split), (size, (q, w, b, s))
    for dtype, size, bn, split in LINEARS:
        q, w, b, s = kernel(*size, x_dtype=["float32", "float16", "bfloat16"].index(dtype))
        assert (q, w, b, s > 1) == (1, 0, bn, split), (dtype, size, (q, w, b, s))


def ints(g, rows, k):
    import torch
    v = torch.randint(-4, 5, (rows, k), device="cuda", generator=g)
    t = torch.full((rows, (k + 15) // 16 * 16), float("nan"), device="cuda").to(torch.float8_e4m3fn)[:, :k]   # NaN beyond k
    t.copy_(v.float())
    return t, v.double()


@pytest.mark.parametrize("size", [p[0] for p in PRODUCTS], ids=lambda s: "%dx%dx%d" % s)
def test_products(size):
    import torch
    m, n, k = size
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(m + n)
    kb = (k + 127) // 128
    (xq, xv), (wq, wv) = ints(g, m, k), ints(g, n, k)
    xs = 2.0 ** torch.randint(-1, 2, (m, kb), device="cuda", generator=g).float()
    ws = 2.0 ** torch.randint(-1, 2, ((n + 127) // 128, kb), device="cuda", generator=g).float()
    bias = torch.randint(-50, 51, (n,), device="cuda", generator=g).float()
    wide = lambda s, block, rows: s.double().repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :k]
    plain = (xv * wide(xs, 1, m)) @ (wv * wide(ws, 128, n)).t()
    assert plain.abs().max() < 2 ** 22
    for out in (torch.float32, torch.float16, torch.bfloat16):
        for lo, pad, b, relu in [(0, (-n) % 8, None, False), (8, 8 + (-n) % 8, bias, True), (1, 2, bias, False), (3, 5, None, True)]:
            big = torch.full((m + 1, lo + n + pad), 7.0, dtype=out, device="cuda")
            y = c.ct_fp8_matmul(xq, xs, wq, ws, bias=b, relu=relu, out=big[:m, lo:lo + n])
            want = plain if b is None else plain + b.double()
            want = (want.clamp(min=0) if relu else want).float().to(out)
            assert torch.equal(y, want), (out, lo)
            assert (big[m] == 7).all() and (big[:m, :lo] == 7).all() and (big[:m, lo + n:] == 7).all()
    assert c.ct_ops_device_error() == 0


@pytest.mark.parametrize("dtype,size", [(d, s) for d, s, _, _ in LINEARS])
def test_linear_layers_in_one_launch(dtype, size):
    import torch
    m, n, k = size
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(m + n)
    wq, ws = c.ct_fp8_quantize(torch.randn(n, k, device="cuda", generator=g) / k ** 0.5, 128)
    bias = torch.randn(n, device="cuda", generator=g)
    base = torch.full((m, k + 9), float("nan"), device="cuda").to(getattr(torch, dtype))
    weights = wq.float().cpu().numpy().astype(np.float64) * _ops.widen(ws.double().cpu().numpy(), 128, n, k)
    for lo in (0, 1, 8):
        x = base[:, lo:lo + k]
        x.copy_(torch.randn(m, k, device="cuda", generator=g) * torch.randn(m, 1, device="cuda", generator=g).exp())
        x[m // 2] = 0
        qr, sr = _ops.quantize(x.double().cpu().numpy(), 1)
        for out in ("float32", "float16", "bfloat16"):
            y = c.ct_fp8_linear(x, wq, ws, bias=bias, relu=lo == 1, out_dtype=getattr(torch, out))
            z = c.ct_fp8_matmul(*c.ct_fp8_quantize(x), wq, ws, bias=bias, relu=lo == 1, out_dtype=getattr(torch, out))
            assert torch.equal(y, z), (lo, out)
            check_product(y, out, qr * _ops.widen(sr, 1, m, k), weights, bias.double().cpu().numpy(), lo == 1, (k + 127) // 128)
        x.fill_(float("nan"))
    assert c.ct_ops_device_error() == 0
