"""Scales at the ends of their range: the two scales of a block are one FP32
factor, exact results as long as it is a normal number."""
import numpy as np
import pytest

from _gpu import ct

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 20, 100, 300])
@pytest.mark.parametrize("ex,ew", [(100, 27), (-50, 140 - 13), (127, 0), (-126, 0), (-60, -66), (-140, 30), (120, -149)])
def test_powers_of_two(m, ex, ew):
    import torch
    rng = np.random.default_rng(m)
    n, k = 150, 130
    e = ex + ew
    xv = rng.integers(-4, 5, (m, k)).astype(np.float64) * (2.0 ** -9 if e > 100 else 1.0)    # results within FP32's range
    wv = rng.integers(-4, 5, (n, k)).astype(np.float64) * (2.0 ** -9 if e > 100 else 1.0)
    xv[0] = 0
    wv[3] = 0

    def dev(v):
        t = torch.zeros(v.shape[0], (k + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :k]
        t.copy_(torch.from_numpy(v).float())
        return t

    xs, ws = torch.full((m, 2), 2.0 ** ex, device="cuda"), torch.full((2, 2), 2.0 ** ew, device="cuda")
    y = ct().ct_fp8_matmul(dev(xv), xs, dev(wv), ws).cpu().numpy()
    assert np.array_equal(y, (xv @ wv.T) * 2.0 ** e)


def test_a_factor_beyond_the_range():
    """2^128 and more is infinity, in the rows whose scales make it."""
    import torch
    e8 = torch.float8_e4m3fn
    x = torch.ones(4, 128, device="cuda").to(e8)
    xs = torch.tensor([[1.0], [2.0 ** 100], [2.0 ** 127], [1.0]], device="cuda")
    y = ct().ct_fp8_matmul(x, xs, x, torch.full((1, 1), 2.0 ** 20, device="cuda"))
    assert (y[[0, 3]] == 2.0 ** 27).all() and (y[1] == 2.0 ** 127).all() and torch.isinf(y[2]).all()
