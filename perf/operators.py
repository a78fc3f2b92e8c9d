"""The 8-bit answer head: quantisation, block-scaled products, log probabilities and their gradient, measured one call at a time.

A classifier (or any model that answers with one of many tokens) ends in wide
fully-connected layers and a row of logits for each answer.  The operators
here run that end in 8 bits and read the answer:

  quantize   x -> 8-bit floating point (e4m3) with one power-of-two scale for
             each run of 128 values of a row (activations) or each 128 x 128
             block (weights)
  linear     y = act(dequant(quant(x)) W^T + b), W in e4m3 with a scale for
             each 128 x 128 block; matmul: the same from an x that is already
             in 8 bits.  A layer's input gradient is the same product with
             the transposed weights.
  logprobs   for each row of logits: the log probability of a given token,
             the entropy, the log of the normaliser and the k most probable
             tokens
  grad       the gradient of the log probability and the entropy with respect
             to the logits

Where ``own`` is false, ``run`` computes them from elementary tensor
operations in 32 bits; where it is true it calls the framework.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # the flattened feature maps of 64 images on their way into the first fully-connected layer
        {"name": "quantize_features", "op": "quantize", "m": 64, "k": 25088, "block_rows": 1, "dtype": "f16"},
        # that layer's weights, laid out once when a model is loaded
        {"name": "quantize_weights", "op": "quantize", "m": 4096, "k": 25088, "block_rows": 128, "dtype": "f32"},
        # one image through the first fully-connected layer of VGG-16: latency, bound by the weights
        {"name": "linear_one", "op": "linear", "m": 1, "n": 4096, "k": 25088, "dtype": "f16", "out": "f16", "bias": True, "relu": True},
        # the classifier of the 1000-class ResNet on its usual batch: the smallest product
        {"name": "linear_classes", "op": "linear", "m": 256, "n": 1000, "k": 512, "dtype": "f32", "out": "f32", "bias": True, "relu": False},
        # a batch of 64 images through VGG-16's first fully-connected layer
        {"name": "linear_batch", "op": "linear", "m": 64, "n": 4096, "k": 25088, "dtype": "f16", "out": "f16", "bias": True, "relu": True},
        # many answers at once (a prompt's tokens, a campaign's images) through a square-ish layer
        {"name": "matmul_prompt", "op": "matmul", "m": 8192, "n": 8192, "k": 4096, "out": "bf16", "bias": False, "relu": False},
        # the gradient of an odd layer's input: the product with the transposed weights, every size ragged
        {"name": "input_grad_ragged", "op": "matmul", "m": 1777, "n": 2999, "k": 5003, "out": "f32", "bias": False, "relu": False},
        # one answer from a large vocabulary, with its 20 best alternatives: latency
        {"name": "logprobs_one", "op": "logprobs", "rows": 1, "vocab": 131072, "dtype": "f16", "top_k": 20, "masked": 0.0},
        # the answers of a 1000-class network on its usual batch
        {"name": "logprobs_classes", "op": "logprobs", "rows": 256, "vocab": 1000, "dtype": "f32", "top_k": 5, "masked": 0.0},
        # a prompt's rows over a large vocabulary, some tokens forbidden
        {"name": "logprobs_prompt", "op": "logprobs", "rows": 2048, "vocab": 131072, "dtype": "bf16", "top_k": 8, "masked": 0.02},
        # training a small odd vocabulary in 32 bits
        {"name": "grad_ragged", "op": "grad", "rows": 517, "vocab": 32003, "dtype": "f32", "masked": 0.0},
        # training on a prompt's rows over a large vocabulary
        {"name": "grad_prompt", "op": "grad", "rows": 2048, "vocab": 131072, "dtype": "bf16", "masked": 0.02},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "matmul", "logprobs", "logprobs", "grad"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "quantize":
        block_rows = rng.choice([1, 128])
        k = _log(rng, 16, 25088)
        return {"op": op, "m": _log(rng, 1, min(16384, (1 << 26) // k)), "k": k, "block_rows": block_rows, "dtype": dtype}
    if op in ("linear", "matmul"):
        n, k = _log(rng, 10, 16384), _log(rng, 16, 25088)
        m = _log(rng, 1, max(1, min(8192, int(2.5e11 / (n * k)))))
        case = {"op": op, "m": m, "n": n, "k": k, "out": rng.choice(["f32", "f16", "bf16"]),
                "bias": rng.random() < 0.5, "relu": rng.random() < 0.3}
        return dict(case, dtype=dtype) if op == "linear" else case
    vocab = _log(rng, 10, 200000)
    rows = _log(rng, 1, max(1, min(8192, (1 << 27) // vocab)))
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "masked": rng.choice([0.0, 0.02, 0.5])}
    return dict(case, top_k=rng.choice([0, 1, 5, 8, 20, 32])) if op == "logprobs" else case


# ---------------------------------------------------------------- inputs

def _pitch(k):
    return (k + 15) // 16 * 16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _to_e4m3(x):
    """8-bit values in rows whose pitch is a multiple of 16 bytes."""
    m, k = x.shape
    q = torch.zeros(m, _pitch(k), dtype=torch.float8_e4m3fn, device=x.device)[:, :k]
    q.copy_(x)
    return q


def _gauss(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _scaled_rows(g, m, k):
    """Activations: rows of different sizes and a few outlying columns."""
    x = _gauss(g, m, k)
    x *= torch.exp(_gauss(g, m, 1))
    x *= torch.where(torch.rand(1, k, device="cuda", generator=g) < 0.01, 20.0, 1.0)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    if case["op"] == "quantize":
        m, k = case["m"], case["k"]
        x = _scaled_rows(g, m, k) if case["block_rows"] == 1 else _gauss(g, m, k) * (2.0 / k) ** 0.5
        s["x"] = x.to(DTYPES[case["dtype"]])
    elif case["op"] in ("linear", "matmul"):
        m, n, k = case["m"], case["n"], case["k"]
        if case["op"] == "linear":
            s["x"] = _scaled_rows(g, m, k).to(DTYPES[case["dtype"]])
        else:
            s["xq"] = _to_e4m3(_gauss(g, m, k) * 100)
            s["xs"] = torch.exp2(torch.randint(-9, -5, (m, _blocks(k)), device="cuda", generator=g).float())
        s["wq"] = _to_e4m3(_gauss(g, n, k) * 100)
        s["ws"] = (torch.rand(_blocks(n), _blocks(k), device="cuda", generator=g) + 0.5) * (0.01 / k ** 0.5)
        s["b"] = _gauss(g, n) * 0.1 if case["bias"] else None
    else:
        rows, vocab = case["rows"], case["vocab"]
        x = _gauss(g, rows, vocab)
        x *= torch.rand(rows, 1, device="cuda", generator=g) * 4 + 0.5
        if case["masked"]:
            x[torch.rand(rows, vocab, device="cuda", generator=g) < case["masked"]] = -math.inf
        s["logits"] = x.to(DTYPES[case["dtype"]])
        del x
        ids = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        ids[torch.rand(rows, device="cuda", generator=g) < 1 / 32] = -1    # rows without a given token
        s["ids"] = ids
        if case["op"] == "grad":
            s["g_logprob"], s["g_entropy"] = _gauss(g, rows), _gauss(g, rows) * 0.1
            s["lse"], s["entropy"] = _lse_entropy(s["logits"].float())[:2]
    return s


# ---------------------------------------------------------------- the plain forms

def _quantize(x, block_rows):
    """(e4m3 values, scales): the scale of a block is the least power of two that brings its values to at most 448."""
    m, k = x.shape
    br, kb = block_rows, _blocks(k)
    mb = (m + br - 1) // br
    p = torch.zeros(mb * br, kb * BLOCK, device=x.device)
    p[:m, :k] = x.float()
    p = p.view(mb, br, kb, BLOCK)
    fine = torch.isfinite(p)
    amax = torch.where(fine, p.abs(), 0.0).amax(dim=(1, 3))
    mantissa, exponent = torch.frexp(amax)                # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    exponent = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp(min=-126)
    scale = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), exponent), 1.0)
    q = torch.where(fine, p / scale[:, None, :, None], math.nan)
    return _to_e4m3(q.view(mb * br, kb * BLOCK)[:m, :k]), scale


def _dequantize(q, scale, block_rows):
    m, k = q.shape
    wide = scale.repeat_interleave(block_rows, 0)[:m] if block_rows > 1 else scale
    return q.float() * wide.repeat_interleave(BLOCK, 1)[:, :k]


def _product(s, xq, xs):
    y = _dequantize(xq, xs, 1) @ _dequantize(s["wq"], s["ws"], BLOCK).t()
    if s["b"] is not None:
        y = y + s["b"]
    if s["relu"]:
        y = torch.where(y < 0, 0.0, y)
    return y.to(DTYPES[s["out"]])


def _lse_entropy(x):
    """(log normaliser, entropy, rows to mark): of 32-bit logits."""
    bad = ~(x < math.inf).all(dim=1)                      # a NaN or +inf in the row
    top = x.amax(dim=1)
    empty = top == -math.inf
    t = x - torch.where(empty, 0.0, top)[:, None]
    e = torch.exp(t)
    z = e.sum(dim=1)
    mean = torch.where(e > 0, e * t, 0.0).sum(dim=1) / z
    lse = top + torch.log(z)
    entropy = torch.where(empty, 0.0, torch.log(z) - mean)
    lse = torch.where(empty, -math.inf, lse)
    return torch.where(bad, math.nan, lse), torch.where(bad, math.nan, entropy), bad


def _top(x, lse, bad, k):
    """The k largest of each row, the lower index first among equals; slots without a token hold -1 and -inf."""
    bits = x.view(torch.int32).to(torch.int64)
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    column = torch.arange(x.shape[1], device=x.device)
    key = order * (1 << 32) + ((1 << 31) - column)
    k_have = min(k, x.shape[1])
    key = torch.topk(key, k_have, dim=1).values
    ids = torch.full((x.shape[0], k), -1, dtype=torch.int64, device=x.device)
    ids[:, :k_have] = (1 << 31) - (key & 0xFFFFFFFF)
    lp = torch.full((x.shape[0], k), -math.inf, device=x.device)
    value = torch.gather(x, 1, ids[:, :k_have])
    none = value == -math.inf
    lp[:, :k_have] = torch.where(none, -math.inf, value - lse[:, None])
    ids[:, :k_have] = torch.where(none, -1, ids[:, :k_have])
    lp[bad], ids[bad] = math.nan, -1
    return lp, ids


def _logprobs(s):
    x = s["logits"].float()
    lse, entropy, bad = _lse_entropy(x)
    ids = s["ids"]
    given = torch.gather(x, 1, ids.clamp(min=0)[:, None])[:, 0]
    lp = torch.where(given == -math.inf, -math.inf, given - lse)
    lp = torch.where(bad, math.nan, torch.where(ids < 0, 0.0, lp))
    top_lp, top_ids = _top(x, lse, bad, s["top_k"]) if s["top_k"] else (x.new_empty(x.shape[0], 0), ids.new_empty(x.shape[0], 0))
    return lp, entropy, lse, top_lp, top_ids


def _grad(s):
    x = s["logits"].float()
    lp = x - s["lse"][:, None]
    p = torch.where(x == -math.inf, 0.0, torch.exp(lp))
    none = s["ids"] < 0
    g = torch.where(none, 0.0, s["g_logprob"])[:, None]
    d = torch.where(p == 0, 0.0, -p * (g + s["g_entropy"][:, None] * (lp + s["entropy"][:, None])))
    d.scatter_add_(1, s["ids"].clamp(min=0)[:, None], g)
    return d.to(s["logits"].dtype)


def run(s):
    op = s["op"]
    if own:
        import paper_2609_16742_gb300 as ct
        if op == "quantize":
            return ct.ct_fp8_quantize(s["x"], s["block_rows"])
        if op == "linear":
            return ct.ct_fp8_linear(s["x"], s["wq"], s["ws"], bias=s["b"], relu=s["relu"], out_dtype=DTYPES[s["out"]])
        if op == "matmul":
            return ct.ct_fp8_matmul(s["xq"], s["xs"], s["wq"], s["ws"], bias=s["b"], relu=s["relu"], out_dtype=DTYPES[s["out"]])
        if op == "logprobs":
            return ct.ct_logprobs(s["logits"], s["ids"], s["top_k"])
        return ct.ct_logprobs_grad(s["logits"], s["ids"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"])
    if op == "quantize":
        return _quantize(s["x"], s["block_rows"])
    if op == "linear":
        return _product(s, *_quantize(s["x"], 1))
    if op == "matmul":
        return _product(s, s["xq"], s["xs"])
    if op == "logprobs":
        return _logprobs(s)
    return _grad(s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "quantize":
        m, k, br = case["m"], case["k"], case["block_rows"]
        scales = (m + br - 1) // br * _blocks(k)
        return {"bytes": m * k * (SIZE[case["dtype"]] + 1) + 4 * scales, "flops": 3 * m * k}
    if op in ("linear", "matmul"):
        m, n, k = case["m"], case["n"], case["k"]
        x = m * k * SIZE[case["dtype"]] if op == "linear" else m * k + 4 * m * _blocks(k)
        return {"bytes": x + n * k + 4 * _blocks(n) * _blocks(k) + (4 * n if case["bias"] else 0) + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    rows, vocab, size = case["rows"], case["vocab"], SIZE[case["dtype"]]
    if op == "logprobs":
        return {"bytes": rows * (vocab * size + 8 + 12 + 12 * case["top_k"]), "flops": 6 * rows * vocab}
    return {"bytes": rows * (2 * vocab * size + 8 + 16), "flops": 7 * rows * vocab}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_quantize(x, block_rows):
    """By columns of blocks: amax, the exponent by log2 set right by comparison, and rounding by hand to 4 significant bits."""
    x = x.double()
    m, k = x.shape
    q = torch.empty_like(x)
    scale = torch.ones((m + block_rows - 1) // block_rows, _blocks(k), dtype=torch.float64, device=x.device)
    row = torch.arange(m, device=x.device) // block_rows
    for j in range(_blocks(k)):
        part = x[:, j * BLOCK:(j + 1) * BLOCK]
        amax = torch.zeros(scale.shape[0], dtype=torch.float64, device=x.device)
        amax.scatter_reduce_(0, row, part.abs().amax(dim=1), "amax")
        e = torch.floor(torch.log2(amax.clamp(min=1e-300) / E4M3_MAX)) - 1
        for _ in range(3):
            e = torch.where(amax > E4M3_MAX * torch.exp2(e), e + 1, e)
        step = torch.where(amax > 0, torch.exp2(e.clamp(min=-126)), 1.0)
        scale[:, j] = step
        v = part / step[row][:, None]
        unit = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        q[:, j * BLOCK:(j + 1) * BLOCK] = torch.round(v / unit) * unit
    return q, scale


def _exact_scaled(q, scale, block_rows):
    m, k = q.shape
    row = torch.arange(m, device=q.device) // block_rows
    column = torch.arange(k, device=q.device) // BLOCK
    return q.double() * scale.double()[row][:, column]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_quantize(s["x"], case["block_rows"])
    if op in ("linear", "matmul"):
        xq, xs = _exact_quantize(s["x"], 1) if op == "linear" else (s["xq"], s["xs"])
        x, w = _exact_scaled(xq, xs, 1), _exact_scaled(s["wq"], s["ws"], BLOCK)
        y = torch.zeros(case["m"], case["n"], dtype=torch.float64, device=x.device)
        if s["b"] is not None:
            y += s["b"].double()
        y.addmm_(x, w.t())
        return y.clamp_(min=0) if case["relu"] else y
    found = [[], [], [], [], []]
    for at in range(0, case["rows"], 128):                 # a few rows at a time: 64 bits of all of them would not be small
        x = s["logits"][at:at + 128].double()
        ids = s["ids"][at:at + 128]
        logp = torch.log_softmax(x, dim=1)
        logp = torch.where(x == -math.inf, -math.inf, logp)
        p = torch.exp(logp)
        plogp = torch.where(p > 0, p * logp, 0.0)
        h = -plogp.sum(dim=1)
        pick = torch.zeros_like(x)
        has = torch.nonzero(ids >= 0)[:, 0]
        pick[has, ids[has]] = 1.0
        if op == "grad":
            g, gh = s["g_logprob"][at:at + 128, None].double(), s["g_entropy"][at:at + 128, None].double()
            g = g * pick.sum(dim=1, keepdim=True)
            found[0].append(g * (pick - p) - gh * (plogp + p * h[:, None]))
            continue
        lp = torch.zeros_like(h)
        lp[has] = logp[has, ids[has]]
        found[0].append(lp)
        found[1].append(h)
        found[2].append(torch.logsumexp(x, dim=1))
        if case["top_k"]:
            value, order = torch.sort(x, dim=1, descending=True, stable=True)
            value, order = value[:, :case["top_k"]], order[:, :case["top_k"]]
            short = case["top_k"] - value.shape[1]
            best = torch.where(value == -math.inf, -math.inf, torch.gather(logp, 1, order))
            order = torch.where(value == -math.inf, -1, order)
            found[3].append(torch.nn.functional.pad(best, (0, short), value=-math.inf))
            found[4].append(torch.nn.functional.pad(order, (0, short), value=-1))
        else:
            found[3].append(x.new_empty(x.shape[0], 0))
            found[4].append(ids.new_empty(x.shape[0], 0))
    if op == "grad":
        d = torch.cat(found[0])
        return d
    return tuple(torch.cat(f) for f in found)
