"""Entropy of rows whose best token is far ahead, with few tokens left: it is
next to 0, and must keep its digits.  Tolerances are derived, not fitted, with
u = 2^-23: Z = 1 + s is within 10 u (2 u for each of the function's value of the
best token, the factor that takes the reference's rounding out, and the
factors of two joins of sums; half a u for each of the 4 additions of what is
not 0), so log Z is within 10 u plus its own rounding; s and
T / Z have relative errors of u (16 + 2 D), D the range of the tokens left.
|error| <= u (12 + (16 + 2 D) entropy)."""
import math

import numpy as np
import pytest

import _ops
from _gpu import ct

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,step", [(400, 1000, 128), (400, 1000, 256), (1300, 7001, 4096), (700, 30011, 8192), (600, 70001, 8192),
                                             (40, 70001, 8192), (2, 300001, 8192)])
def test_entropy_of_confident_rows(dtype, rows, vocab, step):
    """The runner-up lies `step` tokens before the best one, where the same lane
    of the kernel meets it first, for several kinds of rows and splits."""
    import torch
    rng = np.random.default_rng(vocab + step)
    x = np.full((rows, vocab), -math.inf)
    r = np.arange(rows)
    best = rng.integers(step, vocab, rows)
    top = rng.integers(0, 64, rows) / 4.0 - 8
    x[r, rng.integers(0, vocab, rows)] = top - rng.integers(20, 48, rows) / 4.0
    x[r, rng.integers(0, vocab, rows)] = top - rng.integers(28, 48, rows) / 4.0
    x[r, best - step] = top - rng.integers(16, 33, rows) / 4.0
    x[r, best] = top
    xt = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    x = xt.double().cpu().numpy()
    _, h, _, _, _ = _ops.logprobs(x, best, 0)
    live = np.where(np.isfinite(x), x, np.nan)
    d = np.nanmax(live, axis=1) - np.nanmin(live, axis=1)
    lp, got, lse, _, _ = [None if t is None else t.double().cpu().numpy() for t in ct().ct_logprobs(xt, torch.from_numpy(best).cuda())]
    err, tol = np.abs(got - h), U * (12 + (16 + 2 * d) * h)
    assert ct().ct_ops_device_error() == 0
    assert (got >= 0).all() and (err <= tol).all(), (err / tol).max()
