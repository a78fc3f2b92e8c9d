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

# sizes by the kernel that they take on a GB300, several of each: how many clusters a device holds at once may move one
PRODUCTS = [(711, 18, 711), (36, 26, 110), (203, 283, 2218), (128, 49, 2932),              # narrow, 16 columns: whole K, split K
            (17, 10781, 1658), (2984, 13, 20), (107, 1271, 4664), (351, 265, 5598),        # 32
            (495, 2296, 82), (1660, 328, 673), (580, 408, 3957), (42, 1824, 8091),         # 64
            (1356, 1098, 251), (700, 2000, 128), (1568, 156, 5544), (117, 5768, 4353),     # 128
            (3000, 300, 1000), (700, 1000, 2000), (7269, 33, 5011), (6838, 11, 5042),      # wide, 64 columns
            (700, 2000, 1000), (6499, 549, 402), (1243, 796, 6318), (3933, 197, 5705),     # 128
            (417, 11892, 162), (1818, 1626, 985),                                          # 192: whole K only
            (193, 16071, 167), (3869, 2119, 427), (182, 5321, 7519), (6673, 149, 7341)]    # 256

# type of x, (m, n, k): quantised in the launch, 32 columns, whole K and split K, then 16 columns
LINEARS = [("float32", (259, 1422, 154)), ("float16", (259, 1422, 154)), ("bfloat16", (206, 2000, 154)),
           ("float32", (1330, 155, 214)), ("float16", (2465, 65, 73)), ("bfloat16", (1232, 474, 46)),
           ("float32", (682, 41, 4402)), ("float16", (585, 42, 4575)), ("bfloat16", (833, 71, 2325)),
           ("float32", (421, 62, 3969)), ("float16", (293, 100, 4006)), ("bfloat16", (665, 32, 6467)),
           ("float32", (67, 416, 1697)), ("float16", (147, 218, 3206)), ("bfloat16", (242, 20, 4653)),
           ("float32", (356, 67, 266)), ("float16", (59, 266, 534)), ("bfloat16", (55, 99, 1594))]


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
    """(wide, columns, K split), and (type, columns, K split) of what quantises in the launch."""
    products = [kernel(*size) for size in PRODUCTS]
    assert {(w, bn, s > 1) for _, w, bn, s in products} == {(0, bn, s) for bn in (16, 32, 64, 128) for s in (False, True)} | \
        {(1, bn, s) for bn in (64, 128, 256) for s in (False, True)} | {(1, 192, False)}
    types = ["float32", "float16", "bfloat16"]
    linears = [(d, kernel(*size, x_dtype=types.index(d))) for d, size in LINEARS]
    assert {(d, bn, s > 1) for d, (q, _, bn, s) in linears if q} == {(d, bn, s) for d in types for bn in (16, 32) for s in (False, True)}


def ints(g, rows, k):
    import torch
    v = torch.randint(-4, 5, (rows, k), device="cuda", generator=g)
    t = torch.full((rows, (k + 15) // 16 * 16), float("nan"), device="cuda").to(torch.float8_e4m3fn)[:, :k]   # NaN beyond k
    t.copy_(v.float())
    return t, v.double()


@pytest.mark.parametrize("size", PRODUCTS, ids=lambda s: "%dx%dx%d" % s)
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


@pytest.mark.parametrize("dtype,size", LINEARS)
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
