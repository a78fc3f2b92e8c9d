"""The adapted answer head as a whole: 8-bit layers with adapters, their answers, the adapters' gradients, clipping and the
verification of drawn answers, each step against the 64-bit definition of what it was given; and the command."""
import numpy as np
import pytest

import _adapt as ref
from _cache import params
from _gpu import ct
from test_gpu_adapters import check, check_grad, np64
from test_gpu_clip import check as check_clip

pytestmark = pytest.mark.gpu


def made(name, dtype, rank, adapters, seed=0):
    import torch
    import synth
    ct()
    from paper_2609_16742_gb300 import answer_head
    wl = synth.workload(name)
    layers, _ = answer_head.layers_of(wl, params(name))
    dt = getattr(torch, dtype)
    head = answer_head.AdaptedHead(layers, rank, adapters, dt, scale=0.5, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for _, b in head.adapters:
        b.copy_(torch.randn(b.shape, device="cuda", generator=g) * 0.1)
    x = torch.randn(37, layers[0][0].shape[1], device="cuda", generator=g).abs().to(dt)
    ids = torch.randint(-1, adapters, (37,), device="cuda", generator=g)
    return head, x, ids


@pytest.mark.parametrize("name,dtype,rank,adapters", [("lenet5", "float32", 4, 3), ("resnet18_cifar", "float16", 8, 1), ("lenet5", "bfloat16", 16, 5)])
def test_layers_gradients_and_clipping(name, dtype, rank, adapters):
    import torch
    c = ct()
    head, x, ids = made(name, dtype, rank, adapters)
    acts = head.forward(x, ids)
    for (q, s, _, _, bias, relu), (a, b), t, y in zip(head.layers, head.adapters, acts, acts[1:]):
        shared = c.ct_fp8_linear(t, q, s, bias=bias, out_dtype=y.dtype)
        check(shared, t, a, b, ids, head.scale, relu, y)
    chosen = torch.arange(37, device="cuda") % acts[-1].shape[1]
    _, h, lse, _, _ = c.ct_logprobs(acts[-1], chosen)
    d = c.ct_logprobs_grad(acts[-1], chosen, lse, h, torch.ones(37, device="cuda"))
    dx, grads = head.gradients(acts, d, ids)
    for i in reversed(range(len(head.layers))):
        (q, s, qt, st, _, relu), (a, b) = head.layers[i], head.adapters[i]
        if relu:
            d = torch.where(acts[i + 1] > 0, d, torch.zeros_like(d))
        shared = c.ct_fp8_linear(d, qt, st, out_dtype=torch.float32)
        again = c.ct_adapters_grad(d, acts[i], a, b, ids, head.scale, dx=shared.clone(), grad_dtype=torch.float32)
        check_grad(d, acts[i], a, b, ids, head.scale, shared, again)
        assert (again[1] == grads[i][0]).all() and (again[2] == grads[i][1]).all()
        d = again[0]
    assert (d == dx).all()
    flat = [t for pair in grads for t in pair]
    before = [t.clone() for t in flat]
    check_clip(before, flat, 0.01, 2, c.ct_clip_grads(flat, 0.01))
    assert c.ct_ops_device_error() == 0


def test_adapters_that_add_nothing_leave_the_head_as_it_was():
    import torch
    import synth
    ct()
    from paper_2609_16742_gb300 import answer_head
    layers, _ = answer_head.layers_of(synth.workload("lenet5"), params("lenet5"))
    head = answer_head.AdaptedHead(layers, 4)
    x = torch.randn(9, layers[0][0].shape[1], device="cuda")
    for a, b in zip(head.forward(x), answer_head.Head(layers).forward(x)):
        assert (a == b).all()


def test_tuning_follows_the_clipped_gradients():
    """Two steps, written out from the calls that other tests hold against the definition."""
    import torch
    c = ct()
    head, x, _ = made("lenet5", "float32", 4, 1)
    chosen = torch.arange(37, device="cuda") % 10
    want = [[t.clone() for t in pair] for pair in head.adapters]
    start = [[t.clone() for t in pair] for pair in head.adapters]
    losses = []
    for _ in range(2):
        acts = head.forward(x)
        lp, h, lse, _, _ = c.ct_logprobs(acts[-1], chosen)
        losses.append(float(-lp.mean()))
        _, grads = head.gradients(acts, c.ct_logprobs_grad(acts[-1], chosen, lse, h, torch.full((37,), -1 / 37, device="cuda")))
        norm, norms, f = ref.clip([np64(t).reshape(-1) for pair in grads for t in pair], 0.3, 2)
        for pair, gs, own in zip(want, grads, head.adapters):
            for w, gr, t in zip(pair, gs, own):
                w -= 0.25 * (gr.double() * f).float()
                t.copy_(w)
    for pair, s in zip(head.adapters, start):
        for t, w in zip(pair, s):
            t.copy_(w)
    got = head.tune(x, chosen, 2, rate=0.25, max_norm=0.3)
    # a gradient's own bound is in the product's tests; here a factor and a product are rounded once more for each step, and the second
    # step's logits answer to that with factors far below 2^6
    assert np.allclose(got, losses, rtol=2.0 ** -16)
    for pair, w2 in zip(head.adapters, want):
        for t, w in zip(pair, w2):
            assert (t - w).abs().max() <= 2.0 ** -16 * w.abs().max()


def test_drawn_answers():
    import torch
    ct()
    from paper_2609_16742_gb300 import answer_head
    g = torch.Generator(device="cuda").manual_seed(2)
    target = torch.randn(500, 10, device="cuda", generator=g) * 2
    draft = target + torch.randn(500, 10, device="cuda", generator=g) * 0.5
    for heat in (None, torch.zeros(500, device="cuda")):
        answers, stood = answer_head.draw_answers(draft, target, seed=3, temperature=heat)
        assert answers.min() >= 0 and answers.max() < 10 and 0 < int(stood.sum()) < 500
        if heat is not None:
            assert (answers == target.argmax(dim=1)).all()
    same, stood = answer_head.draw_answers(target, target, seed=3)
    assert stood.all()


@pytest.mark.parametrize("argv", [["--workload", "lenet5", "--batch", "8", "--tune", "3", "--draw"],
                                  ["--workload", "resnet18_cifar", "--batch", "4", "--tune", "2", "--rank", "4"],
                                  ["--workload", "lenet5", "--batch", "8", "--draw"]])
def test_command(argv, capsys):
    ct()
    from paper_2609_16742_gb300 import answer_head
    assert answer_head.main(argv) == 0
    out = capsys.readouterr().out
    assert "answers are the protected network's" in out
    assert ("tuned" in out) == ("--tune" in argv) and ("drafts stand" in out) == ("--draw" in argv)
