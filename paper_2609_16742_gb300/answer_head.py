"""The 8-bit answer head on a protected network: run a named synthetic
workload on cuda:0, take the features its fully-connected layers read, run
those layers again in 8 bits, and read the answers:

    python -m paper_2609_16742_gb300.answer_head --workload vgg16 --batch 64

For each image: the class the protected network chose, its log probability
under the 8-bit head, the entropy of the answer and the best alternatives.
Then, per image, the features the answer hangs on: the gradient of that log
probability with respect to the features (through the layers, transposed),
times the feature -- the first-order change of the answer if a fault cleared
that feature.

Weights are quantised once (e4m3, a scale for each 128 x 128 block), with a
transposed copy for the gradient; activations on the way through the layers.
"""
import argparse
import os
import sys

from . import (ct_build_workload, ct_copy_activation, ct_device_error, ct_fp8_linear, ct_fp8_quantize, ct_infer, ct_logprobs,
               ct_logprobs_grad, ct_ops_device_error)


class Head:
    """The fully-connected layers at the end of a network, in 8 bits.

    layers: [(weight [n, k] float32, bias [n] float32 or None, relu), ...] as
    CUDA tensors, in order."""

    def __init__(self, layers):
        import torch
        self.layers = []
        for w, b, relu in layers:
            q, s = ct_fp8_quantize(w, 128)
            n, k = q.shape
            # transposing an e4m3 matrix and its square blocks of scales is exact
            qt = torch.empty(k, (n + 15) // 16 * 16, dtype=torch.uint8, device=q.device)[:, :n]
            qt.copy_(q.view(torch.uint8).t())
            self.layers.append((q, s, qt, s.t(), b, relu))

    def forward(self, x):
        """[x, the output of each layer]; the last is the logits, in float32."""
        import torch
        acts = [x]
        for i, (q, s, _, _, b, relu) in enumerate(self.layers):
            last = i + 1 == len(self.layers)
            acts.append(ct_fp8_linear(acts[-1], q, s, bias=b, relu=relu, out_dtype=torch.float32 if last else x.dtype))
        return acts

    def backward(self, acts, dlogits):
        """Gradient of each layer's input, the features' first."""
        import torch
        grads = [dlogits]
        for (q, s, qt, st, b, relu), y in zip(reversed(self.layers), reversed(acts[1:])):
            d = torch.where(y > 0, grads[0], torch.zeros_like(grads[0])) if relu else grads[0]
            grads.insert(0, ct_fp8_linear(d, qt, st, out_dtype=torch.float32))
        return grads[:-1]


def head_of(wl, params, device="cuda"):
    """(Head, slot of its features) of a workload's trailing fully-connected layers."""
    import torch
    first = len(wl.layers)
    while first > 0 and wl.layers[first - 1].op == "fc":
        first -= 1
    if first == len(wl.layers):
        raise ValueError("workload %s does not end in fully-connected layers" % wl.name)
    layers = []
    for L, p in zip(wl.layers[first:], params[first:]):
        b = torch.from_numpy(p["b"]).to(device) if "b" in p else None
        layers.append((torch.from_numpy(p["w"]).reshape(L.cout, L.cin).to(device), b, bool(L.relu)))
    return Head(layers), wl.layers[first].src


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="vgg16")
    ap.add_argument("--batch", type=int, default=None)
    ap.add_argument("--top", type=int, default=5)
    ap.add_argument("--show", type=int, default=4, help="images to print")
    args = ap.parse_args(argv)

    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    import torch
    import synth

    wl = synth.workload(args.workload)
    B = args.batch or wl.batch
    params = synth.make_params(wl.layers, wl.seed)
    m = ct_build_workload(wl, params, max_batch=B, layerwise=True)    # the features are a stored tensor
    x = torch.from_numpy(synth.make_input(wl, batch=B)).cuda()
    logits = torch.empty(B, wl.n_classes, device="cuda")
    ct_infer(m, x, B, logits)
    head, slot = head_of(wl, params)
    # data channels, in the (C, H, W) order of the layers' weights
    data, _ = ct_copy_activation(m, slot, B)
    features = torch.from_numpy(data.reshape(B, -1)).cuda().to(torch.float16 if wl.precision == "fp16" else torch.float32)

    chosen = logits.argmax(dim=1)
    acts = head.forward(features)
    logprob, entropy, lse, top_logprob, top_id = ct_logprobs(acts[-1], chosen, min(args.top, wl.n_classes))
    dlogits = ct_logprobs_grad(acts[-1], chosen, lse, entropy, torch.ones_like(logprob))
    weight = (head.backward(acts, dlogits)[0] * features.float()).abs()
    torch.cuda.synchronize()

    same = int((top_id[:, 0] == chosen).sum())
    print("workload %s batch %d: %d of %d answers are the protected network's; mean log probability %.4f, mean entropy %.4f"
          % (wl.name, B, same, B, logprob.mean().item(), entropy.mean().item()))
    for i in range(min(args.show, B)):
        best = " ".join("%d:%.3f" % (t, p) for t, p in zip(top_id[i].tolist(), top_logprob[i].tolist()))
        w, f = weight[i].topk(min(5, weight.shape[1]))
        print("image %d class %d log p %.4f entropy %.4f top %s | features %s"
              % (i, chosen[i], logprob[i], entropy[i], best, " ".join("%d:%.4f" % (a, b) for a, b in zip(f.tolist(), w.tolist()))))
    err = ct_device_error(m) | ct_ops_device_error()
    m.close()
    return 0 if err == 0 else 1


if __name__ == "__main__":
    sys.exit(main())
