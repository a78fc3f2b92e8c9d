"""Products into columns of a wider matrix whose rows start at 16-byte boundaries and
end inside a 16-byte unit: what lies beside them is not written."""
import pytest

from _gpu import ct

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("m,k", [(3, 300), (70, 300), (300, 300), (1500, 300), (1500, 4000)])
@pytest.mark.parametrize("n", [9, 130, 301, 999, 1626, 3003])
def test_columns_beside_the_output(out, m, n, k):
    import torch
    c = ct()
    g = torch.Generator(device="cuda").manual_seed(m + n)
    e8 = torch.float8_e4m3fn

    def ints(rows):
        v = torch.randint(-4, 5, (rows, k), device="cuda", generator=g)
        t = torch.zeros(rows, (k + 15) // 16 * 16, dtype=e8, device="cuda")[:, :k]
        t.copy_(v.float())
        return t, v.double()

    kb = (k + 127) // 128
    (xq, xv), (wq, wv) = ints(m), ints(n)
    one = torch.ones(m, kb, device="cuda"), torch.ones((n + 127) // 128, kb, device="cuda")
    big = torch.full((m + 1, (n + 15) // 8 * 8 + 16), 7.0, dtype=getattr(torch, out), device="cuda")
    for lo in (0, 8):
        y = c.ct_fp8_matmul(xq, one[0], wq, one[1], out=big[:m, lo:lo + n])
        assert torch.equal(y, (xv @ wv.t()).float().to(y.dtype))
        big[:m, lo:lo + n] = 7
        assert (big == 7).all()
    assert c.ct_ops_device_error() == 0
