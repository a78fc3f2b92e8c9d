"""Clipping beside autograd."""
import pytest

from _gpu import ct
from test_gpu_clip import TYPES, made

pytestmark = pytest.mark.gpu


def test_results_raise_the_tensors_versions():
    import torch
    c = ct()
    for grads in (made([1000, 7], TYPES), [torch.randn(9, 8, device="cuda")[:, :5], torch.randn(4, 6, device="cuda").t()]):
        out = [torch.zeros_like(g) for g in grads]
        at = [t._version for t in grads + out]
        c.ct_clip_grads(grads, 0.5, out=out)
        assert [t._version for t in grads + out] == at[:len(grads)] + [v + 1 for v in at[len(grads):]]
        c.ct_clip_grads(grads, 0.5)
        assert [t._version for t in grads] == [v + 1 for v in at[:len(grads)]]
