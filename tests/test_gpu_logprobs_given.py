"""The gradient where the given token cannot occur (its logit is -inf): the token's
own term g_logprob stands at its place, as the formula has it with p = 0; the
other tokens that cannot occur have 0."""
import math

import numpy as np
import pytest

from _gpu import ct
from test_gpu_logprobs import DTYPES, check_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 9, 40, 777, 9001])
@pytest.mark.parametrize("in_place", [False, True])
def test_given_tokens_that_cannot_occur(dtype, vocab, in_place):
    import torch
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((6, vocab)) * 3
    ids = np.array([0, vocab - 1, vocab // 2, vocab // 2, -1, vocab // 2])
    x[0] = -math.inf                                   # nothing left, at either end and inside
    x[1] = -math.inf
    x[2] = -math.inf
    x[3, ::2] = -math.inf                              # a part left
    x[3, ids[3]] = -math.inf
    x[4] = -math.inf                                   # nothing left, nothing given
    x[5, ids[5]] = float(torch.finfo(getattr(torch, dtype)).min)
    g = rng.standard_normal(6).astype(np.float32).astype(np.float64)
    gh = rng.standard_normal(6).astype(np.float32).astype(np.float64)
    xt = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    d = check_grad(xt, ids, g, gh, in_place=in_place).double().cpu().numpy()
    own = torch.from_numpy(g).to(getattr(torch, dtype)).double().numpy()
    for r in range(4):
        assert d[r, ids[r]] == own[r]
        assert (np.delete(d[r], ids[r])[np.delete(x[r], ids[r]) == -math.inf] == 0).all()
    assert (d[4] == 0).all()
    assert ct().ct_ops_device_error() == 0
