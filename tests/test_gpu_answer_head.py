"""The 8-bit answer head as a whole (answer_head.py): each layer forward and
backward against the 64-bit product of what it was given (tolerances of
test_gpu_fp8.py), the answers against the 64-bit definitions (test_gpu_logprobs.py),
and the command on two networks."""
import numpy as np
import pytest

import _ops
from _cache import params
from _gpu import ct
from test_gpu_fp8 import check_product
from test_gpu_logprobs import check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,dtype", [("lenet5", "float32"), ("resnet18_cifar", "float16")])
def test_layers_forward_and_backward(name, dtype):
    import torch
    import synth
    ct()
    from paper_2609_16742_gb300 import answer_head
    wl = synth.workload(name)
    head, _ = answer_head.head_of(wl, params(name))
    g = torch.Generator(device="cuda").manual_seed(0)
    k = head.layers[0][0].shape[1]
    x = torch.randn(21, k, device="cuda", generator=g).abs().to(getattr(torch, dtype))
    acts = head.forward(x)

    def values(t):
        q, s = _ops.quantize(t.double().cpu().numpy(), 1)
        return q * _ops.widen(s, 1, *t.shape)

    def weights(q, s):
        return q.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64) * \
            _ops.widen(s.double().cpu().numpy(), 128, *q.shape)

    for a, y, (q, s, qt, st, b, relu) in zip(acts, acts[1:], head.layers):
        check_product(y, str(y.dtype).replace("torch.", ""), values(a), weights(q, s),
                      None if b is None else b.double().cpu().numpy(), relu, (a.shape[1] + 127) // 128)
        np.testing.assert_array_equal(weights(qt, st), weights(q, s).T)
    chosen = acts[-1].argmax(dim=1)
    check_forward(acts[-1], chosen.cpu().numpy(), 3)
    _, h, lse, _, _ = ct().ct_logprobs(acts[-1], chosen)
    d = ct().ct_logprobs_grad(acts[-1], chosen, lse, h, torch.ones(21, device="cuda"))
    grads = head.backward(acts, d) + [d]
    for i, (q, s, _, _, _, relu) in enumerate(head.layers):
        up = grads[i + 1]
        up = torch.where(acts[i + 1] > 0, up, torch.zeros_like(up)) if relu else up
        check_product(grads[i], "float32", values(up), weights(q, s).T, None, False, (q.shape[0] + 127) // 128)


@pytest.mark.parametrize("argv", [["--workload", "lenet5", "--batch", "8"], ["--workload", "resnet18_cifar", "--batch", "4"]])
def test_command(argv, capsys):
    ct()
    from paper_2609_16742_gb300 import answer_head
    assert answer_head.main(argv) == 0
    assert "answers are the protected network's" in capsys.readouterr().out
