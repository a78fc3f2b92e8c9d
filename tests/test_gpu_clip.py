"""The norm of many tensors and clipping, against the definition in 64 bits."""
import math

import numpy as np
import pytest

import _adapt as ref
from _gpu import ct

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]
# A thread adds at most 1024 squares in 32 bits, each rounded once with its addition: relative 1024 x 2^-24 of a sum of positive terms,
# half of that of its root; the root is rounded to 32 bits.
NORM = 1024 * 2.0 ** -24 / 2 + 2.0 ** -24


def made(sizes, types, seed=0, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(getattr(torch, types[i % len(types)])).cuda() for i, n in enumerate(sizes)]


def check(before, after, max_norm, kind, got):
    norm, norms, c = ref.clip([g.double().cpu().numpy().reshape(-1) for g in before], max_norm, kind)
    assert abs(float(got[0]) - norm) <= (NORM if kind == 2 else 2.0 ** -24) * norm, (float(got[0]), norm)
    assert (np.abs(got[1].double().cpu().numpy() - norms) <= (NORM if kind == 2 else 0) * norms).all()
    for b, a in zip(before, after):
        want = b.double().cpu().numpy() * c
        d = ref.name(a.dtype)
        if c == 1.0:
            assert (a == b).all()
            continue
        # the factor has the norm's error and a rounding, the product one in 32 bits and one in the type
        bound = (NORM + 3 * 2.0 ** -24) * np.abs(want) * 1.01 + ref.HALF[d] * np.abs(want) + ref.TINY[d]
        assert (np.abs(a.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("types", [["float32"], ["float16"], ["bfloat16"], TYPES])
@pytest.mark.parametrize("sizes", [[1], [5, 0, 1, 4097], [100003], [7] * 60, [1, 40000, 3, 270001, 8, 0], list(range(0, 1100, 2)), [3000001, 5, 1 << 20]])
def test_clip(sizes, types, kind):
    import torch
    c = ct()
    for max_norm in (0.5, 1e9, 0.0):
        grads = made(sizes, types)
        before = [g.clone() for g in grads]
        got = c.ct_clip_grads(grads, max_norm, kind)
        assert got[0].shape == () and got[1].shape == (len(sizes),)
        check(before, grads, max_norm, kind, got)
        out = [torch.full_like(g, 3.0) for g in before]
        again = c.ct_clip_grads(before, max_norm, kind, out=out)
        assert again[0] == got[0] and (again[1] == got[1]).all()
        assert all((o == g).all() for o, g in zip(out, grads))


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale", [1e30, 1e36, 1e-25, 1e-36])
def test_values_whose_squares_leave_the_range(scale, dtype, kind):
    grads = made([5, 70001], [dtype], scale=scale)
    before = [g.clone() for g in grads]
    got = ct().ct_clip_grads(grads, scale / 2, kind)
    check(before, grads, scale / 2, kind, got)


def test_one_large_value_among_small_ones():
    import torch
    g = torch.full((100000,), 1e-30, device="cuda")
    g[777] = 1e25
    h = torch.full((3000,), 1e-20, device="cuda")
    before = [g.clone(), h.clone()]
    check(before, [g, h], 1e24, 2.0, ct().ct_clip_grads([g, h], 1e24))


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_not_finite_scales_nothing(bad, kind):
    import torch
    grads = made([1000, 50000, 17], TYPES)
    grads[1][1234] = bad
    before = [g.clone() for g in grads]
    norm, norms = ct().ct_clip_grads(grads, 0.1, kind)
    want = math.nan if bad != bad else math.inf
    assert str(float(norm)) == str(want) and str(float(norms[1])) == str(want) and norms[0].isfinite() and norms[2].isfinite()
    for g, b in zip(grads, before):
        assert torch.equal(g.nan_to_num(5.0), b.nan_to_num(5.0)) and torch.equal(g.isnan(), b.isnan())
    out = [torch.zeros_like(g) for g in grads]
    ct().ct_clip_grads(grads, 0.1, kind, out=out)
    for o, b in zip(out, before):
        assert torch.equal(o.nan_to_num(5.0), b.nan_to_num(5.0)) and torch.equal(o.isnan(), b.isnan())


def test_a_norm_beyond_the_range_scales_nothing():
    import torch
    g = torch.full((5000,), 3e38, device="cuda")
    before = g.clone()
    norm, norms = ct().ct_clip_grads([g], 1.0)
    assert float(norm) == math.inf and float(norms[0]) == math.inf and (g == before).all()


def test_layouts():
    """Pitches, transposed and channels-last tensors, tensors that start anywhere, columns of one matrix."""
    import torch
    c = ct()
    store = torch.randn(90, 64, device="cuda")
    grads = [store[:40, 3:24], store[:40, 24:25], store[:40, 30:64], torch.randn(33, 20, device="cuda").t(),
             torch.randn(4, 6, 5, 7, device="cuda").contiguous(memory_format=torch.channels_last), torch.randn(1001, device="cuda").half()[1:],
             torch.randn(3, 1, device="cuda"), torch.randn(70, 9, device="cuda")[::2, :8]]
    before = [g.clone() for g in grads]
    rest = store[40:].clone()
    got = c.ct_clip_grads(grads, 1.5)
    check(before, grads, 1.5, 2, got)
    assert (store[40:] == rest).all()
    out = [torch.zeros(40, 50, device="cuda")[:, 5:26], torch.zeros(40, 1, device="cuda"), torch.zeros(40, 34, device="cuda")] + \
          [torch.zeros_like(b) for b in before[3:]]
    out[3] = torch.zeros(33, 20, device="cuda").t()
    out[4] = torch.zeros_like(grads[4])
    source = [g.copy_(b) for g, b in zip(grads, before)]
    c.ct_clip_grads(source, 1.5, out=out)
    check(before, out, 1.5, 2, got)


def test_more_values_than_32_bits_count():
    import torch
    n = (1 << 31) + 1027
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[-1], g[1 << 31] = 3.0, 4.0, 12.0
    norm, norms = ct().ct_clip_grads([g], 6.5)
    assert float(norm) == 13.0 and float(norms[0]) == 13.0
    assert g[0] == 1.5 and g[-1] == 2.0 and g[1 << 31] == 6.0 and int((g != 0).sum()) == 3


def test_captured_and_on_streams():
    import torch
    c = ct()
    grads = made([1000, 300001, 5], TYPES)
    out = [torch.zeros_like(g) for g in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.ct_clip_grads(grads, 0.7, out=out)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        norm, norms = c.ct_clip_grads(grads, 0.7, out=out)
    for seed in (3, 4):
        for a, b in zip(grads, made([1000, 300001, 5], TYPES, seed=seed)):
            a.copy_(b)
        g.replay()
        kept = [o.clone() for o in out]
        check(grads, kept, 0.7, 2, (norm, norms))
        out2 = [torch.zeros_like(x) for x in grads]
        side.wait_stream(torch.cuda.current_stream())
        n2, ns2 = c.ct_clip_grads(grads, 0.7, out=out2, stream=side)
        torch.cuda.synchronize()
        assert n2 == norm and (ns2 == norms).all() and all((a == b).all() for a, b in zip(out2, kept))


def test_refusals():
    import torch
    c = ct()
    g = torch.randn(10, 10, device="cuda")
    for bad in (lambda: c.ct_clip_grads([], 1.0), lambda: c.ct_clip_grads([g], -1.0), lambda: c.ct_clip_grads([g], math.nan),
                lambda: c.ct_clip_grads([g], 1.0, 1.0), lambda: c.ct_clip_grads([g.cpu()], 1.0), lambda: c.ct_clip_grads([g.double()], 1.0),
                lambda: c.ct_clip_grads([g[:, ::2]], 1.0), lambda: c.ct_clip_grads([g[:1].expand(4, 10)], 1.0),
                lambda: c.ct_clip_grads([g], 1.0, out=[]), lambda: c.ct_clip_grads([g], 1.0, out=[g.half()]),
                lambda: c.ct_clip_grads([g], 1.0, out=[torch.zeros(10, 10, device="cuda").t()]), lambda: c.ct_clip_grads([g, g.cpu()], 1.0),
                lambda: c.ct_clip_grads([g.clone().requires_grad_()], 1.0)):
        with pytest.raises(ValueError):
            bad()
    flat = torch.randn(100, device="cuda")
    for bad in ([g, g], [flat[:60], flat[50:]], [g[:, :6], g[:, 5:]]):
        with pytest.raises(c.CtError):
            c.ct_clip_grads(bad, 1.0)
    with pytest.raises(c.CtError):
        c.ct_clip_grads([flat[:50]], 1.0, out=[flat[10:60]])
