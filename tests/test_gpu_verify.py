"""Verification of drafted tokens against the definition in 64 bits, the tokens' distribution, masks, bad rows and offsets."""
import math

import numpy as np
import pytest

import _adapt as ref
from _gpu import ct

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


def made(lengths, vocab, dtype, seed=0, point=False, masked=0.0, heat=None, spread=4.0, pad=0):
    """Arguments of ct_verify_drafts, a draft row near each target row."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)
    batch, count = len(lengths), sum(lengths)
    offsets = torch.tensor([sum(lengths[:b]) for b in range(batch + 1)])
    rows = torch.tensor([offsets[b].item() + b + j for b in range(batch) for j in range(lengths[b])], dtype=torch.int64)
    x = torch.randn(count + batch, vocab + pad, generator=g) * spread
    q = (x[rows] + 0.7 * torch.randn(count, vocab + pad, generator=g))
    if masked:
        x[torch.rand(x.shape, generator=g) < masked] = -math.inf
    x, q = x.to(dt).cuda()[:, pad // 2:pad // 2 + vocab], q.to(dt).cuda()[:, pad // 2:pad // 2 + vocab]
    e = torch.empty(count, vocab).exponential_(generator=g).clamp_(min=1e-20).cuda()
    from_ = x[rows.cuda()] if point else q
    drafts = (from_.float() - torch.log(e)).argmax(dim=1) if vocab else torch.zeros(count, dtype=torch.int64, device="cuda")
    u = torch.rand(count, generator=g).cuda()
    noise = torch.empty(batch, vocab + pad).exponential_(generator=g).clamp_(min=1e-20).cuda()[:, :vocab]
    t = None if heat is None else torch.tensor([heat[b % len(heat)] for b in range(batch)]).cuda()
    return x, drafts, offsets.cuda(), u, noise, None if point else q, t


def run(c, args, most):
    x, drafts, offsets, u, noise, q, t = args
    return c.ct_verify_drafts(x, drafts, offsets, most, u, noise, draft_logits=q, temperature=t)


def check(args, most, got):
    x, drafts, offsets, u, noise, q, t = args
    ref.same_as_defined(got, x, q, drafts, offsets, most, u, noise, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 10, 129, 1000, 5003, 32003, 70001])
def test_verify(vocab, dtype):
    for lengths, most in (([4], 4), ([0], 0), ([3, 0, 1, 5, 2, 5, 0], 5), ([1] * 13, 3), ([0, 0], 2)):
        for seed, (point, masked, heat) in enumerate(((False, 0.0, None), (True, 0.0, [0.0, 0.7, 1.3]), (False, 0.5, [1.0, 0.0]), (False, 0.02, [0.3, 2.0]))):
            for pad in (0, 3):
                args = made(lengths, vocab, dtype, seed, point, masked, heat, pad=pad)
                check(args, most, run(ct(), args, most))


@pytest.mark.parametrize("batch,most,vocab", [(1, 64, 500), (300, 2, 333), (40, 8, 9000), (2, 4, 200000), (170, 3, 4099)])
def test_many_sequences_and_drafts(batch, most, vocab):
    lengths = [(5 * b + 3) % (most + 1) if batch > 1 else most for b in range(batch)]
    for dtype, point in (("bfloat16", False), ("float32", True)):
        args = made(lengths, vocab, dtype, 7, point, 0.0, [0.0, 1.0, 0.8])
        check(args, most, run(ct(), args, most))


def test_ties_go_to_the_lowest_index():
    import torch
    c = ct()
    for vocab in (40, 3000, 50000):
        x = torch.zeros(3, vocab, device="cuda")
        x[:, vocab // 3] = x[:, vocab // 2] = x[:, vocab - 1] = 5.0
        zero, offsets = torch.zeros(2, device="cuda"), torch.tensor([0, 2], device="cuda")
        drafts = torch.tensor([vocab // 3, vocab // 2], device="cuda")
        noise = torch.ones(1, vocab, device="cuda")
        got = c.ct_verify_drafts(x, drafts, offsets, 2, zero, noise, temperature=torch.zeros(1, device="cuda"))
        assert got[0].tolist() == [1] and got[1].tolist() == [[vocab // 3, vocab // 3, -1]]
        # equal weights and noise; the draft's own token is out
        got = c.ct_verify_drafts(x, drafts, offsets, 2, zero + 0.9999, noise)
        assert got[0].tolist() == [0] and got[1].tolist() == [[vocab // 2, -1, -1]]
        got = c.ct_verify_drafts(x, drafts, offsets, 2, zero, noise)
        assert got[0].tolist() == [2] and got[1].tolist() == [[vocab // 3, vocab // 2, vocab // 3]]


def test_tokens_are_distributed_as_the_target():
    """One draft, many sequences: the counts of the first token against the target's probabilities.  Chi-squared over 8 tokens with
    200,000 draws: 7 degrees of freedom exceed 40 with probability 1.3e-6."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    n, vocab = 200000, 8
    p = torch.tensor([0.5, -1.0, 2.0, 0.0, 1.0, -2.0, 1.5, 0.3], device="cuda")
    q = torch.tensor([1.5, 0.0, 1.0, 0.5, -1.0, 0.0, 2.0, 0.3], device="cuda")
    x = p.expand(2 * n, vocab).contiguous()
    drafts = (q - torch.log(torch.empty(n, vocab, device="cuda").exponential_(generator=g))).argmax(dim=1)
    u = torch.rand(n, device="cuda", generator=g)
    noise = torch.empty(n, vocab, device="cuda").exponential_(generator=g)
    for draft_logits in (q.expand(n, vocab).contiguous(), None):
        acc, tok, _ = ct().ct_verify_drafts(x, drafts, torch.arange(n + 1, device="cuda"), 1, u, noise, draft_logits=draft_logits)
        if draft_logits is None:
            # certain drafts: each stands with its own p
            first = torch.bincount(tok[:, 0], minlength=vocab).double() / n
            share = torch.bincount(drafts, minlength=vocab).double() / n
            pp = torch.softmax(p.double(), 0)
            want = share * pp + sum(share[i] * (1 - pp[i]) * torch.where(torch.arange(vocab, device="cuda") == i, 0.0, pp / (1 - pp[i])) for i in range(vocab))
        else:
            first, want = torch.bincount(tok[:, 0], minlength=vocab).double() / n, torch.softmax(p.double(), 0)
        chi = float((n * (first - want) ** 2 / want).sum())
        assert chi < 40, (chi, first, want)


@pytest.mark.parametrize("vocab", [50, 4000, 40000])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_and_bad_rows(vocab, dtype):
    import torch
    c = ct()
    lowest = torch.finfo(getattr(torch, dtype)).min
    for case in range(9):
        args = made([2] * 6, vocab, dtype, case, heat=[1.0, 0.5] if case % 2 else None)
        x, drafts, offsets, u, noise, q, t = args
        if case == 0:
            x[3] = -math.inf                     # nothing can occur
            x[8] = -math.inf
        elif case == 1:
            x[:, vocab // 2:] = lowest           # masked by the type's lowest value
            q[:, vocab // 2:] = lowest
        elif case == 2:
            x[0, 3], x[4, 7], x[8, 1], q[6, 2], q[9, 0] = math.nan, math.inf, math.nan, math.inf, math.nan
        elif case == 3:
            q[2], q[5] = -math.inf, -math.inf
        elif case == 4:
            drafts[0], drafts[3], drafts[6] = -1, vocab, 1 << 40
        elif case == 5:
            t = torch.tensor([-1.0, math.nan, math.inf, 1e-31, 1e-25, 1e20], device="cuda")
        elif case == 6:
            q.copy_(x[torch.tensor([0, 1, 3, 4, 6, 7, 9, 10, 12, 13, 15, 16], device="cuda")])   # equal: every draft stands
            u.fill_(0.999)
        elif case == 7:
            # drafts of equal probabilities fall, and nothing is left of p - q: p.  At u = 1 the two sides would be equal, and sums of the
            # same numbers in two orders (rows that start on other boundaries) differ by up to 2^-23: 2^-10 more decides.
            u.fill_(1.0 + 2.0 ** -10)
            q.copy_(x[torch.tensor([0, 1, 3, 4, 6, 7, 9, 10, 12, 13, 15, 16], device="cuda")])
        elif case == 8:
            x[:, 5:] = -math.inf
            q[:, :5] = -math.inf                 # nothing in common
        args = (x, drafts, offsets, u, noise, q, t)
        got = run(c, args, 2)
        if case in (6, 7):                       # equal up to the rounding of two sums of the same numbers: the same bits
            assert got[0].tolist() == [2 if case == 6 else 0] * 6
        check(args, 2, got)


def test_offsets_out_of_order_or_range():
    """What is outside is clamped; nothing beside the tensors is read or written (the results are those of the clamped offsets)."""
    import torch
    c = ct()
    x, drafts, _, u, noise, q, _ = made([3, 3, 3], 700, "float32")
    for off in ([0, 20, 9, 9], [-5, 3, 6, 9], [4, 2, 9, 1], [9, 9, 9, 9], [0, 1, 5, 9], [-(1 << 60), 1 << 60, 3, 1 << 62]):
        args = (x, drafts, torch.tensor(off, device="cuda"), u, noise, q, None)
        check(args, 5, run(c, args, 5))


def test_clamped_offsets_with_temperatures():
    """Ascending offsets that begin before 0 and end behind the drafts: each row goes by its own sequence's temperature."""
    import torch
    x, drafts, _, u, noise, q, _ = made([3, 3, 3], 3000, "float32")
    for off, heat in (([-7, -2, 4, 9], [0.3, 0.0, 1.0]), ([0, 4, 30, 40], [0.0, 0.5, 0.0]), ([-9, -8, -7, 2], [0.0, 0.7, 0.0]), ([12, 13, 14, 15], [0.0, 1.0, 0.2])):
        args = (x, drafts, torch.tensor(off, device="cuda"), u, noise, q, torch.tensor(heat, device="cuda"))
        check(args, 5, run(ct(), args, 5))


def test_descending_offsets_among_greedy_sequences_touch_nothing_else():
    import torch
    x, drafts, _, u, noise, q, _ = made([3, 3, 3], 3000, "float32")
    for off in ([9, 5, 2, 0], [4, 2, 9, 1], [0, 20, 9, 9]):
        for heat in ([0.0, 1.0, 0.0], [1.0, 0.0, 1.0]):
            n, token, lp = run(ct(), (x, drafts, torch.tensor(off, device="cuda"), u, noise, q, torch.tensor(heat, device="cuda")), 5)
            assert 0 <= int(n.min()) and int(n.max()) <= 5 and int(token.min()) >= -1 and int(token.max()) < 3000


def test_more_drafts_than_are_looked_at():
    args = made([6, 2, 9], 300, "float32")
    check(args, 3, run(ct(), args, 3))


def test_offsets_beyond_32_bits():
    import torch
    x, drafts, offsets, u, noise, q, t = made([2], 90, "bfloat16")
    ld = (1 << 30) + 8
    far = torch.zeros(2 * ld + 96, dtype=torch.bfloat16, device="cuda").as_strided((3, 90), (ld, 1)).copy_(x)
    a, b = run(ct(), (far, drafts, offsets, u, noise, q, t), 2), run(ct(), (x, drafts, offsets, u, noise, q, t), 2)
    assert all((i == j).all() for i, j in zip(a, b))


@pytest.mark.parametrize("vocab,batch", [(600, 5), (40000, 2)])
def test_captured_and_on_streams(vocab, batch):
    import torch
    c = ct()
    lengths = [3] * batch
    args = made(lengths, vocab, "float16")
    run(c, args, 3)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run(c, args, 3)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for seed in (4, 5):
        for a, b in zip(args, made(lengths, vocab, "float16", seed)):
            if a is not None:
                a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        check(args, 3, got)
        x, drafts, offsets, u, noise, q, t = args
        many = [c.ct_verify_drafts(x, drafts, offsets, 3, u, noise, draft_logits=q, temperature=t, stream=s) for s in streams for _ in range(3)]
        torch.cuda.synchronize()
        for m in many:
            assert all((i == j).all() for i, j in zip(m, got))


def test_refusals():
    import torch
    c = ct()
    x, drafts, offsets, u, noise, q, t = made([2, 1], 30, "float16", heat=[1.0])
    for bad in (lambda: c.ct_verify_drafts(x[:4], drafts, offsets, 2, u, noise), lambda: c.ct_verify_drafts(x, drafts.int(), offsets, 2, u, noise),
                lambda: c.ct_verify_drafts(x, drafts, offsets, 65, u, noise), lambda: c.ct_verify_drafts(x, drafts, offsets, -1, u, noise),
                lambda: c.ct_verify_drafts(x, drafts, offsets, 2, u[:2], noise), lambda: c.ct_verify_drafts(x, drafts, offsets, 2, u, noise[:, :29]),
                lambda: c.ct_verify_drafts(x, drafts, offsets, 2, u, noise, draft_logits=q.float()),
                lambda: c.ct_verify_drafts(x, drafts, offsets, 2, u, noise, draft_logits=q[:2]),
                lambda: c.ct_verify_drafts(x, drafts, offsets, 2, u, noise, temperature=t[:1]),
                lambda: c.ct_verify_drafts(x, drafts, offsets[:0], 2, u, noise), lambda: c.ct_verify_drafts(x.cpu(), drafts, offsets, 2, u, noise),
                lambda: c.ct_verify_drafts(x.clone().requires_grad_(), drafts, offsets, 2, u, noise)):
        with pytest.raises(ValueError):
            bad()
    none = c.ct_verify_drafts(x[:0], drafts[:0], offsets[:1], 2, u[:0], noise[:0])
    assert [tuple(n.shape) for n in none] == [(0,), (0, 3), (0, 3)]
