"""Clipping at the ends of its ranges, and beside autograd."""
import math

import pytest

from _gpu import ct
from test_gpu_clip import TYPES, check, made

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


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale,max_norm", [(1e20, 1e-20), (1e30, 1e-12), (1e36, 1e-36), (1e-2, 1e-41), (1e36, 1e-300), (1e3, 1e-34), (1e30, 5e-324)])
def test_factors_below_the_range_of_32_bits(scale, max_norm, dtype, kind):
    """max_norm / norm has no normal 32-bit number, the values times it have."""
    import torch
    for sizes in ([5, 70001], [1]):
        grads = made(sizes, [dtype], scale=scale)
        before = [g.clone() for g in grads]
        out = [torch.full_like(g, 3.0) for g in grads]
        got = ct().ct_clip_grads(grads, max_norm, kind, out=out)
        check(before, out, max_norm, kind, got)
        assert all(torch.equal(g, b) for g, b in zip(grads, before))
        ct().ct_clip_grads(grads, max_norm, kind)
        assert all(torch.equal(g, o) for g, o in zip(grads, out))
    pitched = made([300], [dtype], scale=scale)[0].view(20, 15)[:, 2:13]
    before = [pitched.clone()]
    check(before, [pitched], max_norm, kind, ct().ct_clip_grads([pitched], max_norm, kind))


def test_tensors_between_one_another():
    """Tensors of one store whose ranges cross and which share no value: a row in the gap of a matrix's rows, matrices of different pitches."""
    import torch
    c = ct()
    store = torch.zeros(24, 30, device="cuda")
    picks = ([store[:, :4], store[3, 5:9], store[7, 10:30]], [store[::2, :10], store[1::2, 3:20], store[::4, 12:16], store[2, 25:30]],
             [store[::3, 1:9], store[1::2, 20:30], store[::6, 10:20]], [store.view(-1)[:600].view(20, 30)[:, 29:], store[1:, :29]])
    for grads in picks:
        store.copy_(torch.randn(24, 30))
        before = [g.clone() for g in grads]
        rest = torch.ones(24, 30, dtype=torch.bool, device="cuda")
        for g in grads:
            rest.as_strided(g.shape, g.stride(), g.storage_offset()).fill_(False)
        was = store.clone()
        check(before, grads, 0.5, 2, c.ct_clip_grads(grads, 0.5))
        assert torch.equal(store[rest], was[rest])
    flat = store.view(-1)
    for bad in ([store[::2, :10], store[::4, 9:12]], [store[:, :4], store[3, 3:9]], [store[::3, 1:9], store[1::2, 8:30]],
                [store[:, 2:9], flat[30 * 23 + 8:30 * 23 + 12]], [flat[23 * 30:], store[5:, 29:]]):
        with pytest.raises(c.CtError):
            c.ct_clip_grads(bad, 1.0)
