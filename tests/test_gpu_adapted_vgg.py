"""The adapted head at VGG-16's fully-connected sizes, with the types that tuning it has: FP16 activations and adapters, FP32 gradients."""
import pytest

from _gpu import ct
from test_gpu_adapters import check, check_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [5, 37, 160])
def test_layers_and_gradients(rows):
    import torch
    c = ct()
    from paper_2609_16742_gb300 import answer_head
    g = torch.Generator(device="cuda").manual_seed(rows)
    sizes = [(25088, 4096), (4096, 4096), (4096, 1000)]
    layers = [(torch.randn(n, k, device="cuda", generator=g) * (2 / k) ** 0.5, torch.randn(n, device="cuda", generator=g) * 0.1, n != 1000)
              for k, n in sizes]
    head = answer_head.AdaptedHead(layers, 8, dtype=torch.float16)
    for _, b in head.adapters:
        b.copy_(torch.randn(b.shape, device="cuda", generator=g) * 0.1)
    acts = head.forward(torch.randn(rows, 25088, device="cuda", generator=g).abs().half())
    d = torch.randn(rows, 1000, device="cuda", generator=g) * 0.01
    dx, grads = head.gradients(acts, d)
    for i in reversed(range(3)):
        (q, s, qt, st, bias, relu), (a, b) = head.layers[i], head.adapters[i]
        shared = c.ct_fp8_linear(acts[i], q, s, bias=bias, out_dtype=acts[i + 1].dtype)
        check(shared, acts[i], a, b, None, head.scale, relu, acts[i + 1])
        if relu:
            d = torch.where(acts[i + 1] > 0, d, torch.zeros_like(d))
        shared = c.ct_fp8_linear(d, qt, st, out_dtype=torch.float32)
        again = c.ct_adapters_grad(d, acts[i], a, b, None, head.scale, dx=shared.clone(), grad_dtype=torch.float32)
        check_grad(d, acts[i], a, b, None, head.scale, shared, again)
        assert (again[1] == grads[i][0]).all() and (again[2] == grads[i][1]).all()
        d = again[0]
    assert (d == dx).all()
    assert c.ct_ops_device_error() == 0
