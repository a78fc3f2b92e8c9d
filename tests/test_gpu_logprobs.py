"""Log probabilities, entropy, top tokens and their gradient against plain
64-bit implementations.  Tolerances are derived, not fitted, with u = 2^-23:
  - e^(x - m) has a relative error of a few u from the function and |x - m| u
    from its argument, where |x - m| <= D = min(104, range of the row) (beyond
    it the term is 0 in FP32); a sum of n terms by one thread and a tree adds at
    most n u / 128 + 16 u; so lse is within u (16 + n / 128 + 2 D + 4 |m|), the
    entropy within u (16 + n / 128 + 2 D) (1 + entropy);
  - a log probability adds one rounding of x - lse;
  - the gradient is the formula of the given lse and entropy, with p within
    u (8 + 2 |log p|), and one rounding to its type.
Top tokens are compared for equality."""
import math

import numpy as np
import pytest

import _ops
from _gpu import ct

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF_UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}
DTYPES = ["float32", "float16", "bfloat16"]


def torch_():
    import torch
    return torch


def row_tols(x):
    with np.errstate(invalid="ignore"):
        live = np.where(np.isfinite(x), x, np.nan)
        empty = np.isnan(live).all(axis=1)
        live[empty] = 0.0
        m = np.nanmax(live, axis=1)
        d = np.minimum(104.0, m - np.nanmin(live, axis=1))
    base = 16 + x.shape[1] / 128 + 2 * d
    return U * (base + 4 * np.abs(m)), U * base


def same_or_near(got, want, tol):
    """Equal where not finite, within tol elsewhere."""
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine])
    err = np.abs(got[fine] - want[fine])
    tol = np.broadcast_to(tol, want.shape)[fine]
    assert (err <= tol).all(), (err / tol).max()


def check_forward(xt, ids, k):
    torch = torch_()
    x = xt.double().cpu().numpy()
    got = [None if t is None else t.cpu().numpy() for t in ct().ct_logprobs(xt, torch.from_numpy(ids).cuda(), k)]
    lp, h, lse, top_lp, top_id = _ops.logprobs(x, ids, k)
    tl, th = row_tols(x) if x.shape[1] else (np.zeros(len(x)), np.zeros(len(x)))
    same_or_near(got[2].astype(np.float64), lse, tl)
    same_or_near(got[1].astype(np.float64), h, th * (1 + np.where(np.isfinite(h), h, 0)))
    same_or_near(got[0].astype(np.float64), lp, tl + U * np.where(np.isfinite(lp), np.abs(lp), 0))
    np.testing.assert_array_equal(got[4], top_id)
    same_or_near(got[3].astype(np.float64), top_lp, (tl[:, None] + U * np.where(np.isfinite(top_lp), np.abs(top_lp), 0)))
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 5), (256, 10, 3), (70, 33, 32), (9, 1000, 5), (5, 1003, 20),
                                          (2, 4097, 8), (3, 32003, 32), (1, 131072, 20), (2, 70001, 0), (1, 300001, 7)])
def test_forward(dtype, rows, vocab, k):
    torch = torch_()
    rng = np.random.default_rng(rows + vocab)
    x = rng.standard_normal((rows, vocab)) * rng.uniform(0.3, 6, (rows, 1)) + 5 * rng.standard_normal((rows, 1))
    ids = rng.integers(0, vocab, rows)
    ids[rng.random(rows) < 0.2] = -1
    check_forward(torch.from_numpy(x).to(getattr(torch, dtype)).cuda(), ids, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [7, 1000, 9001, 70000])
def test_masks_infinities_and_empty_rows(dtype, vocab):
    torch = torch_()
    rng = np.random.default_rng(vocab)
    low = float(torch.finfo(getattr(torch, dtype)).min)
    high = float(torch.finfo(getattr(torch, dtype)).max)
    x = rng.standard_normal((14, vocab)) * 3
    x[0] = -math.inf                                  # nothing left
    x[1] = -math.inf; x[1, vocab - 1] = -2.0          # one token left
    x[2, rng.random(vocab) < 0.9] = -math.inf
    x[3, rng.random(vocab) < 0.9] = low               # masked by the type's lowest value
    x[4] = low                                        # all of them: a uniform row
    x[5, vocab // 2] = math.inf                       # poisoned rows
    x[6, vocab - 1] = math.nan
    x[7, 0], x[7, 1] = math.nan, -math.inf
    x[8] = 1.5                                        # all equal: the lowest indices
    x[9] = 0.0; x[9, ::2] = -0.0                      # signed zeros are equal
    x[10] = -1e4; x[10, 2] = 50.0                     # everything else vanishes
    x[11] = np.sort(x[11])[::-1]                      # the best tokens side by side
    x[12] = np.sort(x[12])                            # ... at the end
    x[13] = low; x[13, 3] = high                      # the whole range of the type
    ids = np.array([0, vocab - 1, 3, 3, 5, 2, 2, 2, vocab - 1, 1, 2, 0, vocab, -2])
    check_forward(torch.from_numpy(x).to(getattr(torch, dtype)).cuda(), ids, 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,k", [(1025, 5), (2047, 32), (4096, 8), (8001, 20)])
def test_many_rows(dtype, vocab, k):
    """More rows than the GPU has warps for at first, of moderate length: as
    few rows do, with odd starts, masks, ties, poisoned and empty rows."""
    torch = torch_()
    rng = np.random.default_rng(vocab)
    rows = 1300
    low = float(torch.finfo(getattr(torch, dtype)).min)
    x = rng.standard_normal((rows, vocab + 3)) * rng.uniform(0.3, 6, (rows, 1))
    x[0] = -math.inf
    x[1] = 1.5
    x[2] = low
    x[3, ::3] = math.nan
    x[4, 700] = math.inf
    x[5] = rng.integers(0, 3, vocab + 3)
    x[6] = np.sort(x[6])
    x[7] = np.sort(x[7])[::-1]
    x[8, rng.random(vocab + 3) < 0.99] = -math.inf
    x[9] = -math.inf; x[9, 100:140] = 1.0
    ids = rng.integers(-1, vocab, rows)
    xt = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    check_forward(xt[:, 1:vocab + 1], ids, k)
    check_forward(xt[:, :vocab].contiguous(), ids, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [31, 64, 65, 257, 1000, 1024])
@pytest.mark.parametrize("k", [16, 17, 32])
def test_short_rows_many_tokens(dtype, vocab, k):
    """As many tokens as a warp has lanes, from rows that one warp holds: spread
    out, side by side, nearly all masked, equal."""
    torch = torch_()
    rng = np.random.default_rng(vocab + k)
    x = rng.standard_normal((40, vocab)) * 2
    x[0] = np.sort(x[0])
    x[1] = np.sort(x[1])[::-1]
    x[2, rng.random(vocab) < 0.95] = -math.inf
    x[3] = 0.25
    x[4] = rng.integers(0, 4, vocab)
    x[5, : vocab // 2] = -math.inf
    check_forward(torch.from_numpy(x).to(getattr(torch, dtype)).cuda(), rng.integers(-1, vocab, 40), k)


def test_few_values_many_ties():
    """Logits of three values: every choice among the top is a tie."""
    torch = torch_()
    rng = np.random.default_rng(2)
    for vocab in (50, 5000, 66000):
        x = rng.integers(0, 3, (4, vocab)).astype(np.float32)
        x[1, : vocab // 2] = 0
        check_forward(torch.from_numpy(x).cuda(), np.full(4, 1), 32)
        check_forward(torch.from_numpy(x).bfloat16().cuda(), np.full(4, 1), 32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_offsets(dtype):
    torch = torch_()
    rng = np.random.default_rng(4)
    base = torch.from_numpy(rng.standard_normal((12, 5003)) * 4).to(getattr(torch, dtype)).cuda()
    for lo, hi in [(0, 5003), (1, 5003), (3, 4000), (7, 8), (2, 1026)]:
        x = base[1::2, lo:hi]
        want = check_forward(x, np.arange(6) % (hi - lo), 9)
        alone = [t.cpu().numpy() for t in ct().ct_logprobs(x.contiguous(), torch.arange(6, device="cuda") % (hi - lo), 9)]
        for a, b in zip(want, alone):
            np.testing.assert_array_equal(a, b)        # the same bits from rows that start elsewhere


def test_sizes_of_zero_and_no_ids():
    torch = torch_()
    check_forward(torch.zeros(0, 5, device="cuda"), np.zeros(0, np.int64), 2)
    check_forward(torch.zeros(3, 0, device="cuda"), np.array([-1, 0, -1]), 2)
    x = torch.randn(4, 100, device="cuda")
    lp, h, lse, tl, ti = ct().ct_logprobs(x)
    assert lp is None and tl.shape == (4, 0) and torch.equal(lse, ct().ct_logprobs(x, top_k=3)[2])
    d = ct().ct_logprobs_grad(torch.zeros(0, 5, device="cuda"), None, torch.zeros(0, device="cuda"), None)
    assert d.shape == (0, 5)


def check_grad(xt, ids, g, gh, in_place=False):
    torch = torch_()
    dtype = str(xt.dtype).replace("torch.", "")
    idt = torch.from_numpy(ids).cuda()
    _, h, lse, _, _ = ct().ct_logprobs(xt, idt)
    gt, ght = torch.from_numpy(g).float().cuda(), torch.from_numpy(gh).float().cuda()
    x = xt.double().cpu().numpy()
    d = ct().ct_logprobs_grad(xt, idt, lse, h, gt, ght, out=xt if in_place else None)
    ln, hn = lse.double().cpu().numpy(), h.double().cpu().numpy()
    want = _ops.grad(x, ids, ln, hn, g, gh)
    with np.errstate(invalid="ignore", over="ignore"):
        lp = np.where(np.isfinite(x), x - ln[:, None], 0.0)
        mag = np.exp(np.minimum(lp, 1)) * (np.abs(g)[:, None] + np.abs(gh)[:, None] * (np.abs(lp) + np.abs(hn)[:, None]))
        tol = U * (8 + 2 * np.minimum(np.abs(lp), 110)) * mag + 2 * U * np.abs(g)[:, None] + HALF_UNIT[dtype] * np.abs(want) + TINY[dtype] + 1e-37
    same_or_near(d.double().cpu().numpy(), want, tol)
    return d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (4, 2), (256, 10), (7, 1003), (3, 32003), (1, 131072), (600, 129)])
def test_gradient(dtype, rows, vocab):
    torch = torch_()
    rng = np.random.default_rng(rows * vocab)
    x = torch.from_numpy(rng.standard_normal((rows, vocab)) * 3).to(getattr(torch, dtype)).cuda()
    ids = rng.integers(-1, vocab, rows)
    g = rng.standard_normal(rows).astype(np.float32).astype(np.float64)
    gh = rng.standard_normal(rows).astype(np.float32).astype(np.float64)
    d = check_grad(x, ids, g, gh)
    xc = x.clone()
    assert torch.equal(check_grad(xc, ids, g, gh, in_place=True), d)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_masks(dtype):
    torch = torch_()
    low = float(torch.finfo(getattr(torch, dtype)).min)
    rng = np.random.default_rng(6)
    x = rng.standard_normal((9, 777)) * 3
    x[0] = -math.inf
    x[1, ::2] = -math.inf
    x[2, ::2] = low
    x[3] = low
    x[4, 5] = math.nan
    x[5, 5] = math.inf
    x[6] = -math.inf; x[6, 700] = 3.0
    ids = np.array([-1, 1, 1, 1, 1, 1, 700, -7, 777])
    check_grad(torch.from_numpy(x).to(getattr(torch, dtype)).cuda(), ids, np.ones(9), np.full(9, 0.5))


def test_gradient_strides():
    torch = torch_()
    rng = np.random.default_rng(1)
    base = torch.from_numpy(rng.standard_normal((10, 1500))).bfloat16().cuda()
    ids = rng.integers(0, 900, 5)
    x = base[::2, 3:1203]
    d = check_grad(x, ids, np.ones(5), np.ones(5))
    _, h, lse, _, _ = ct().ct_logprobs(x)
    buf = torch.full((7, 1300), 9.0, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(5, device="cuda")
    ct().ct_logprobs_grad(x, torch.from_numpy(ids).cuda(), lse, h, one, one, out=buf[1:6, 5:1205])
    assert torch.equal(buf[1:6, 5:1205], d)
    buf[1:6, 5:1205] = 9.0
    assert (buf == 9.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 5, 40, 300, 2500, 9001])
@pytest.mark.parametrize("lo,to", [(0, 1), (1, 0), (3, 5), (7, 7), (2, 10)])
def test_gradient_starts(dtype, vocab, lo, to):
    """Logits and gradients whose rows start anywhere: what contiguous ones
    give, and nothing beside it."""
    torch = torch_()
    rows = 67
    base = torch.randn(rows, vocab + 11, device="cuda").to(getattr(torch, dtype))
    ids = torch.arange(rows, device="cuda") % vocab
    one = torch.ones(rows, device="cuda")
    x = base[:, lo:lo + vocab]
    _, h, lse, _, _ = ct().ct_logprobs(x, ids)
    buf = torch.full((rows, vocab + 13), 9.0, dtype=x.dtype, device="cuda")
    ct().ct_logprobs_grad(x, ids, lse, h, one, one, out=buf[:, to:to + vocab])
    assert torch.equal(buf[:, to:to + vocab], ct().ct_logprobs_grad(x.contiguous(), ids, lse, h, one, one))
    buf[:, to:to + vocab] = 9.0
    assert (buf == 9.0).all()


def test_gradient_against_differences():
    """Central differences of the forward kernel, step e = 2^-6: truncation
    e^2 / 6 times a third derivative of at most 6 (|g| + |gh| (8 + entropy)),
    and twice the forward tolerance over 2 e."""
    torch = torch_()
    rng = np.random.default_rng(12)
    vocab, e = 40, 2.0 ** -6
    x = np.round(rng.standard_normal((1, vocab)) * 2 * 1024) / 1024
    ids = np.array([11])
    g, gh = 0.7, -0.4
    rows = np.repeat(x, 2 * vocab, 0)
    rows[np.arange(vocab), np.arange(vocab)] += e
    rows[vocab + np.arange(vocab), np.arange(vocab)] -= e
    lp, h, _, _, _ = ct().ct_logprobs(torch.from_numpy(rows).float().cuda(), torch.full((2 * vocab,), 11, device="cuda"))
    f = g * lp.double().cpu().numpy() + gh * h.double().cpu().numpy()
    slope = (f[:vocab] - f[vocab:]) / (2 * e)
    d = check_grad(torch.from_numpy(x).float().cuda(), ids, np.array([np.float32(g)], float), np.array([np.float32(gh)], float))
    tl, th = row_tols(rows)
    tol = e * e * (abs(g) + abs(gh) * (8 + math.log(vocab))) + (tl.max() * 2 + th.max() * 5) / (2 * e)
    assert np.abs(slope - d.double().cpu().numpy()[0]).max() <= tol


def test_one_of_the_gradients_alone():
    torch = torch_()
    x = torch.randn(5, 300, device="cuda")
    ids = torch.arange(5, device="cuda")
    _, h, lse, _, _ = ct().ct_logprobs(x, ids)
    one, zero = torch.ones(5, device="cuda"), torch.zeros(5, device="cuda")
    a = ct().ct_logprobs_grad(x, ids, lse, h, one, zero)
    assert torch.equal(a, ct().ct_logprobs_grad(x, ids, lse, None, one, None))
    b = ct().ct_logprobs_grad(x, ids, lse, h, zero, one)
    assert torch.equal(b, ct().ct_logprobs_grad(x, None, lse, h, None, one))


def test_refusals():
    torch = torch_()
    c = ct()
    x = torch.zeros(4, 64, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    v = torch.zeros(4, device="cuda")
    for bad in (lambda: c.ct_logprobs(x.double(), ids), lambda: c.ct_logprobs(x.t(), ids), lambda: c.ct_logprobs(x, ids.int()),
                lambda: c.ct_logprobs(x, ids[:3]), lambda: c.ct_logprobs(x, ids, 33), lambda: c.ct_logprobs(x, ids, -1),
                lambda: c.ct_logprobs(x, ids.cpu()), lambda: c.ct_logprobs_grad(x, None, v, v, v),
                lambda: c.ct_logprobs_grad(x, ids, v, None, None, v), lambda: c.ct_logprobs_grad(x, ids, v, v, v, out=x.half())):
        with pytest.raises(ValueError):
            bad()


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes of logits: the last rows are the same as those rows alone."""
    torch = torch_()
    rows, vocab = 24000, 131077
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[-300:] = torch.randn(300, vocab, device="cuda").bfloat16() * 3
    assert x.numel() > 2 ** 31
    ids = torch.full((rows,), 131076, device="cuda")
    got = ct().ct_logprobs(x, ids, 5)
    want = check_forward(x[-7:].clone(), ids[-7:].cpu().numpy(), 5)
    np.testing.assert_array_equal(got[4][-7:].cpu().numpy(), want[4])
    for a, b in zip(got[:4], want[:4]):
        np.testing.assert_allclose(a[-7:].cpu().numpy(), b, rtol=0, atol=1e-4)
    one = torch.ones(rows, device="cuda")
    d = ct().ct_logprobs_grad(x, ids, got[2], got[1], one, one, out=x)
    assert torch.isfinite(d[-300:].float()).all() and (d[-300:, -1] > 0).all() and (d[:3, 0] < 0).all()
