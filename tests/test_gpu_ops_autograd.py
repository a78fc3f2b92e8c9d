"""The 8-bit answer head and autograd: results are not tracked, so a tensor that
requires a gradient is refused while autograd records, by name, and taken
where the caller has said that no gradient is wanted."""
import pytest

from _gpu import ct

pytestmark = pytest.mark.gpu


def calls():
    import torch
    c = ct()
    x = torch.randn(4, 256, device="cuda")
    v = torch.randn(4, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    q, s = c.ct_fp8_quantize(x)
    w, ws = c.ct_fp8_quantize(torch.randn(4, 256, device="cuda"), 128)
    _, h, lse, _, _ = c.ct_logprobs(x, ids)
    return [("x", x, lambda t: c.ct_fp8_quantize(t)), ("x", x, lambda t: c.ct_fp8_linear(t, w, ws)),
            ("bias", v, lambda t: c.ct_fp8_linear(x, w, ws, bias=t)), ("ws", ws, lambda t: c.ct_fp8_linear(x, w, t)),
            ("xs", s, lambda t: c.ct_fp8_matmul(q, t, w, ws)), ("bias", v, lambda t: c.ct_fp8_matmul(q, s, w, ws, bias=t)),
            ("out", torch.empty(4, 4, device="cuda"), lambda t: c.ct_fp8_matmul(q, s, w, ws, out=t)),
            ("logits", x, lambda t: c.ct_logprobs(t, ids, 2)), ("logits", x, lambda t: c.ct_logprobs_grad(t, ids, lse, h, v, v)),
            ("lse", lse, lambda t: c.ct_logprobs_grad(x, ids, t, h, v, v)), ("entropy", h, lambda t: c.ct_logprobs_grad(x, ids, lse, t, v, v)),
            ("g_logprob", v, lambda t: c.ct_logprobs_grad(x, ids, lse, h, t, v)), ("g_entropy", v, lambda t: c.ct_logprobs_grad(x, ids, lse, h, v, t))]


def flat(y):
    return [t for t in (y if isinstance(y, tuple) else (y,)) if t is not None]


def same(got, want):
    return all((a.float() == b.float()).all() for a, b in zip(got, want)) and len(got) == len(want)


def test_tensors_that_require_a_gradient():
    import torch
    for name, t, f in calls():
        want = [y.clone() for y in flat(f(t))]
        leaf = t.detach().clone().requires_grad_()
        for tracked in (leaf, leaf * 1) if name != "out" else (leaf,):
            with pytest.raises(ValueError, match=name + r".*gradient"):
                f(tracked)
            with torch.no_grad():
                got = flat(f(tracked))
            assert same(got, want)
        assert same(flat(f(leaf.detach())), want)
