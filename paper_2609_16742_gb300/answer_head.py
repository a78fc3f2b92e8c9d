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

With --tune N the head is adapted: low-rank adapters beside its frozen layers
learn for N steps to answer as the protected network does (their gradients are
clipped to a norm of 1).  With --draw an answer is drawn instead of taken: the
8-bit head drafts a class for each image and the protected network's
probabilities decide whether it stands, so that what is answered is distributed as
the protected network's answers are.  That shows how ct_verify_drafts is called; with the
protected network's logits at hand for one answer an image, a draw from them would
do, and drafts save time only where several of them go before one run of the target.
"""
import argparse
import os
import sys

from . import (ct_adapters, ct_adapters_grad, ct_build_workload, ct_clip_grads, ct_copy_activation, ct_device_error, ct_fp8_linear,
               ct_fp8_quantize, ct_infer, ct_logprobs, ct_logprobs_grad, ct_ops_device_error, ct_verify_drafts)


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


class AdaptedHead(Head):
    """A head with low-rank adapters beside its frozen layers: each layer is
    act(W x + b + scale B_i A_i x), i the adapter of the row.

    rank, adapters: of every layer; dtype: of the adapters (that of the
    activations).  A starts random, B at 0: at first the adapters add nothing."""

    def __init__(self, layers, rank, adapters=1, dtype=None, scale=1.0, seed=0):
        import torch
        super().__init__(layers)
        g = torch.Generator().manual_seed(seed)
        self.adapters = []
        for w, _, _ in layers:
            n, k = w.shape
            a = torch.randn(adapters, rank, k, generator=g) * k ** -0.5
            self.adapters.append((a.to(device=w.device, dtype=dtype or torch.float32),
                                  torch.zeros(adapters, n, rank, device=w.device, dtype=dtype or torch.float32)))
        self.scale = torch.full((adapters,), float(scale), device=layers[0][0].device)

    def forward(self, x, ids=None):
        """[x, the output of each layer]; ids int64 [rows]: the adapter of each row (-1: none; None: the only one)."""
        import torch
        acts = [x]
        for i, ((q, s, _, _, bias, relu), (a, b)) in enumerate(zip(self.layers, self.adapters)):
            last = i + 1 == len(self.layers)
            y = ct_fp8_linear(acts[-1], q, s, bias=bias, out_dtype=torch.float32 if last else x.dtype)
            acts.append(ct_adapters(y, acts[-1], a, b, ids, self.scale, relu=relu))
        return acts

    def gradients(self, acts, dlogits, ids=None):
        """(gradient of the features, [(dA, dB) of each layer], in float32)."""
        import torch
        found, d = [], dlogits
        for (q, s, qt, st, _, relu), (a, b), x, y in zip(reversed(self.layers), reversed(self.adapters), reversed(acts[:-1]), reversed(acts[1:])):
            if relu:
                d = torch.where(y > 0, d, torch.zeros_like(d))
            d, da, db = ct_adapters_grad(d, x, a, b, ids, self.scale, dx=ct_fp8_linear(d, qt, st, out_dtype=torch.float32),
                                         grad_dtype=torch.float32)
            found.insert(0, (da, db))
        return d, found

    def tune(self, x, chosen, steps, rate=0.05, ids=None, max_norm=1.0):
        """Gradient descent on the mean of -log p(chosen): [its value before each step].  Gradients are clipped together."""
        import torch
        master = [[t.float() for t in pair] for pair in self.adapters]
        g = torch.full((x.shape[0],), -1.0 / x.shape[0], device=x.device)
        losses = []
        for _ in range(steps):
            acts = self.forward(x, ids)
            logprob, entropy, lse, _, _ = ct_logprobs(acts[-1], chosen)
            losses.append(-logprob.mean())
            _, grads = self.gradients(acts, ct_logprobs_grad(acts[-1], chosen, lse, entropy, g), ids)
            flat = [t for pair in grads for t in pair]
            ct_clip_grads(flat, max_norm)
            for w, t, d in zip((w for pair in master for w in pair), (t for pair in self.adapters for t in pair), flat):
                w.sub_(d, alpha=rate)
                t.copy_(w)
        return torch.stack(losses).tolist() if losses else []


def draw_answers(draft_logits, target_logits, seed=0, temperature=None):
    """(answers, which drafts stood) [rows]: one class for each row, drafted from draft_logits' probabilities and verified against
    target_logits', as which it is distributed."""
    import torch
    rows, n = target_logits.shape
    g = torch.Generator(device=target_logits.device).manual_seed(seed)
    draft_logits = draft_logits.to(target_logits.dtype)
    # drafts are drawn from what they are verified by; below 1e-30 the most probable class is taken
    heat = 1.0 if temperature is None else temperature[:, None].clamp(min=1e-30)
    first = torch.empty(rows, n, device=draft_logits.device).exponential_(generator=g)
    x = draft_logits.float()
    drafts = ((x - x.amax(dim=1, keepdim=True)) / heat - torch.log(first)).argmax(dim=1)
    noise = torch.empty(rows, n, device=draft_logits.device).exponential_(generator=g)
    uniform = torch.rand(rows, device=draft_logits.device, generator=g)
    # each row is a sequence of one draft; the row after it, which a longer answer would go on from, is the same again
    token = ct_verify_drafts(target_logits.repeat_interleave(2, dim=0), drafts, torch.arange(rows + 1, device=drafts.device), 1, uniform, noise,
                             draft_logits=draft_logits, temperature=temperature)
    return token[1][:, 0], token[0] > 0


def layers_of(wl, params, device="cuda"):
    """([(weight, bias, relu), ...], slot of the features they read) of a workload's trailing fully-connected layers."""
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
    return layers, wl.layers[first].src


def head_of(wl, params, device="cuda"):
    """(Head, slot of its features) of a workload's trailing fully-connected layers."""
    layers, slot = layers_of(wl, params, device)
    return Head(layers), slot


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="vgg16")
    ap.add_argument("--batch", type=int, default=None)
    ap.add_argument("--top", type=int, default=5)
    ap.add_argument("--show", type=int, default=4, help="images to print")
    ap.add_argument("--tune", type=int, default=0, metavar="N", help="adapt the head for N steps first")
    ap.add_argument("--rank", type=int, default=8, help="of the adapters")
    ap.add_argument("--rate", type=float, default=0.05, help="of the steps")
    ap.add_argument("--draw", action="store_true", help="draw answers: drafted by the head, verified by the protected network")
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
    layers, slot = layers_of(wl, params)
    # data channels, in the (C, H, W) order of the layers' weights
    data, _ = ct_copy_activation(m, slot, B)
    features = torch.from_numpy(data.reshape(B, -1)).cuda().to(torch.float16 if wl.precision == "fp16" else torch.float32)

    chosen = logits.argmax(dim=1)
    if args.tune > 0:
        head = AdaptedHead(layers, args.rank, dtype=features.dtype)
        losses = head.tune(features, chosen, args.tune, args.rate)
        print("tuned %d steps at rank %d: mean -log p of the protected network's answers %.4f at first, %.4f at last"
              % (args.tune, args.rank, losses[0], losses[-1]))
    else:
        head = Head(layers)
    acts = head.forward(features)
    logprob, entropy, lse, top_logprob, top_id = ct_logprobs(acts[-1], chosen, min(args.top, wl.n_classes))
    dlogits = ct_logprobs_grad(acts[-1], chosen, lse, entropy, torch.ones_like(logprob))
    weight = ((head.gradients(acts, dlogits)[0] if args.tune > 0 else head.backward(acts, dlogits)[0]) * features.float()).abs()
    if args.draw:
        answers, stood = draw_answers(acts[-1], logits)
    torch.cuda.synchronize()

    same = int((top_id[:, 0] == chosen).sum())
    print("workload %s batch %d: %d of %d answers are the protected network's; mean log probability %.4f, mean entropy %.4f"
          % (wl.name, B, same, B, logprob.mean().item(), entropy.mean().item()))
    if args.draw:
        print("drawn answers: %d of %d drafts stand, %d answers are the most probable ones"
              % (int(stood.sum()), B, int((answers == chosen).sum())))
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
