"""What adapts the 8-bit answer head and lets it answer in earnest, measured one call at a time.

The head's weights are frozen in 8 bits.  What is trained beside them, and how
its rows of logits become tokens:

  adapters   y[t] += s[i] B[i] (A[i] x[t]), i = ids[t]: low-rank adapters of many
             requests at once, added to what the shared projection gave
  grad       the gradients of A, B and x of that
  clip       the norm of the gradients of many tensors, the norm of each, and
             the gradients scaled down to a given norm
  verify     drafted tokens held against the target's probabilities with given
             random numbers: how many stand, and the token that follows them

Where ``own`` is false, ``run`` computes them from elementary tensor
operations in 32 bits (in 64 where sums are long or a comparison decides);
where it is true it calls the framework.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one token of one request through a square layer: latency
        {"name": "adapters_token", "op": "adapters", "t": 1, "k": 4096, "n": 4096, "rank": 16, "adapters": 8, "order": "runs",
         "bare": False, "relu": False, "dtype": "bf16", "out": "bf16"},
        # the features of 64 images before VGG-16's first fully-connected layer, an adapter of its own for each
        {"name": "adapters_requests", "op": "adapters", "t": 64, "k": 25088, "n": 4096, "rank": 16, "adapters": 64, "order": "shuffled",
         "bare": False, "relu": True, "dtype": "f16", "out": "f16"},
        # the prompts of a few requests through a wide layer
        {"name": "adapters_prompt", "op": "adapters", "t": 8192, "k": 4096, "n": 8192, "rank": 64, "adapters": 4, "order": "runs",
         "bare": False, "relu": False, "dtype": "bf16", "out": "bf16"},
        # training one adapter of the 1000-class ResNet's classifier on its usual batch
        {"name": "grad_classes", "op": "grad", "t": 256, "k": 512, "n": 1000, "rank": 8, "adapters": 1, "order": "all",
         "bare": False, "dtype": "f32", "out": "f32"},
        # three adapters of an odd layer trained at once, rows of theirs and of none in any order
        {"name": "grad_ragged", "op": "grad", "t": 1777, "k": 5003, "n": 2999, "rank": 20, "adapters": 3, "order": "shuffled",
         "bare": True, "dtype": "f16", "out": "f32"},
        # training one adapter on a prompt's rows
        {"name": "grad_prompt", "op": "grad", "t": 8192, "k": 4096, "n": 8192, "rank": 64, "adapters": 1, "order": "all",
         "bare": False, "dtype": "bf16", "out": "bf16"},
        # one answer, four drafted tokens: latency
        {"name": "verify_one", "op": "verify", "batch": 1, "drafts": 4, "vocab": 131072, "lengths": "full", "point": False,
         "heat": "one", "masked": 0.0, "dtype": "f16"},
        # many answers at once over a large vocabulary, some tokens forbidden
        {"name": "verify_batch", "op": "verify", "batch": 64, "drafts": 5, "vocab": 131072, "lengths": "full", "point": False,
         "heat": "one", "masked": 0.02, "dtype": "bf16"},
        # drafts looked up, not drawn (no probabilities of their own), of different lengths, greedy rows among them
        {"name": "verify_ragged", "op": "verify", "batch": 37, "drafts": 7, "vocab": 32003, "lengths": "ragged", "point": True,
         "heat": "mixed", "masked": 0.0, "dtype": "f32"},
        # the gradients of twenty adapters of odd sizes, under the limit: only their norm is wanted
        {"name": "clip_adapters", "op": "clip", "tensors": 40, "values": 2000003, "spread": "even", "limit": "over", "kind": 2.0,
         "dtype": "bf16"},
        # ResNet-18's parameters (weights and biases), many of them small
        {"name": "clip_resnet", "op": "clip", "tensors": 42, "values": 11684712, "spread": "wide", "limit": "under", "kind": 2.0,
         "dtype": "f32"},
        # as many values as VGG-16 has, most of them in one tensor
        {"name": "clip_vgg", "op": "clip", "tensors": 32, "values": 138357544, "spread": "wide", "limit": "under", "kind": 2.0,
         "dtype": "f32"},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["adapters", "adapters", "grad", "verify", "verify", "clip"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op in ("adapters", "grad"):
        k, n = _log(rng, 16, 25088), _log(rng, 10, 16384)
        rank = rng.choice([1, 4, 5, 8, 16, 20, 32, 64, 128])
        adapters = _log(rng, 1, max(1, min(64, int(6e7 / (rank * (k + n))))))
        # the plain form multiplies every row with every adapter; its time bounds the rows too
        most = min(8192.0, 1.6e8 / (k + n), 2.5e10 / (adapters * rank * (k + n)))
        case = {"op": op, "t": _log(rng, 1, max(1, int(most))), "k": k, "n": n, "rank": rank, "adapters": adapters,
                "order": rng.choice(["runs", "shuffled"]), "bare": rng.random() < 0.3, "dtype": dtype, "out": rng.choice([dtype, "f32"])}
        return dict(case, relu=rng.random() < 0.3) if op == "adapters" else case
    if op == "verify":
        vocab, drafts = _log(rng, 10, 200000), rng.randint(1, 8)
        rows = min(1024, int(4.8e7 / vocab))                # target rows, then as many draft rows
        return {"op": op, "batch": _log(rng, 1, max(1, rows // (drafts + 1))), "drafts": drafts, "vocab": vocab,
                "lengths": rng.choice(["full", "ragged"]), "point": rng.random() < 0.3, "heat": rng.choice(["one", "mixed"]),
                "masked": rng.choice([0.0, 0.02, 0.5]), "dtype": dtype}
    tensors = _log(rng, 1, 60)
    return {"op": op, "tensors": tensors, "values": tensors + _log(rng, 100, 100000000), "spread": rng.choice(["even", "wide"]),
            "limit": rng.choice(["over", "under", "under"]), "kind": rng.choice([2.0, 2.0, math.inf]), "dtype": dtype}


def _lengths(case):
    """Drafted tokens of each sequence."""
    if case["lengths"] == "full":
        return [case["drafts"]] * case["batch"]
    return [(5 * b + 3) % (case["drafts"] + 1) for b in range(case["batch"])]


def _sizes(case):
    """Values of each tensor: about the same, or over a range of 2000."""
    count, total = case["tensors"], case["values"]
    weight = [1.0 + i % 3 if case["spread"] == "even" else 2000.0 ** (((7 * i + 5) % count) / max(1, count - 1)) for i in range(count)]
    size = [max(1, int(w * (total - count) / sum(weight))) for w in weight]
    size[0] += max(0, total - sum(size))
    return size


# ---------------------------------------------------------------- inputs

def _gauss(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _ids(case, g):
    t, n = case["t"], case["adapters"]
    if case["order"] == "all":
        return None
    i = torch.arange(t, device="cuda")
    names = torch.randperm(n, device="cuda", generator=g)
    ids = names[i * n // t] if case["order"] == "runs" else names[i % n][torch.randperm(t, device="cuda", generator=g)]
    if case["bare"]:
        ids[torch.rand(t, device="cuda", generator=g) < 1 / 16] = -1
    return ids


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op in ("adapters", "grad"):
        t, k, n, r, count = (case[c] for c in ("t", "k", "n", "rank", "adapters"))
        out = DTYPES[case["out"]]
        s["x"] = (_gauss(g, t, k) * torch.exp(0.5 * _gauss(g, t, 1))).to(dt)
        s["a"] = (_gauss(g, count, r, k) * k ** -0.5).to(dt)
        s["b"] = (_gauss(g, count, n, r) * r ** -0.5).to(dt)
        s["ids"] = _ids(case, g)
        s["scale"] = torch.rand(count, device="cuda", generator=g) + 0.5
        if op == "adapters":
            s["y"] = _gauss(g, t, n).to(out)                # what the shared projection gave
        else:
            s["dy"] = (_gauss(g, t, n) * 0.1).to(out)
            s["dx"] = (_gauss(g, t, k) * 0.1).to(out)       # the shared projection's part
    elif op == "verify":
        lengths, vocab, batch = _lengths(case), case["vocab"], case["batch"]
        count = sum(lengths)
        s["offsets"] = torch.tensor([sum(lengths[:b]) for b in range(batch + 1)], device="cuda")
        seq = torch.repeat_interleave(torch.arange(batch, device="cuda"), torch.tensor(lengths, device="cuda"))
        rows = torch.arange(count, device="cuda") + seq     # the target rows that have a draft
        x = _gauss(g, count + batch, vocab) * 4.0
        q = x[rows] + 0.7 * _gauss(g, count, vocab)         # a drafting head is near the target, not equal
        if case["masked"]:
            x[torch.rand(x.shape, device="cuda", generator=g) < case["masked"]] = -math.inf
        s["logits"] = x.to(dt)
        q = q.to(dt)
        s["temperature"] = None
        if case["heat"] == "mixed":
            s["temperature"] = torch.tensor([0.0, 0.7, 1.0, 1.3], device="cuda")[torch.randint(0, 4, (batch,), device="cuda", generator=g)]
        e = torch.empty(count, vocab, device="cuda").exponential_(generator=g).clamp_(min=1e-20)
        s["drafts"] = ((x[rows] if case["point"] else q.float()) - torch.log(e)).argmax(dim=1)
        if case["point"]:                                   # what is looked up is often what the target likes best
            often = torch.rand(count, device="cuda", generator=g) < 0.7
            s["drafts"] = torch.where(often, x[rows].argmax(dim=1), s["drafts"])
        s["q"] = None if case["point"] else q
        s["max"] = case["drafts"]
        s["uniform"] = torch.rand(count, device="cuda", generator=g)
        s["noise"] = torch.empty(batch, vocab, device="cuda").exponential_(generator=g).clamp_(min=1e-20)
    else:
        s["grads"] = [(_gauss(g, n) * (0.01 * 3.0 ** (i % 5))).to(dt) for i, n in enumerate(_sizes(case))]
        s["out"], s["max_norm"] = None, 1e6                 # the norm is under the limit: the gradients stay
        if case["limit"] == "under":                        # the limit is under the norm: scaled copies, the gradients are kept
            s["out"], s["max_norm"] = [torch.empty_like(t) for t in s["grads"]], 0.02
    return s


# ---------------------------------------------------------------- the plain forms

def _spread(v, ids, count):
    """[t, rank] -> [t, count * rank], each row in the place of its adapter."""
    t, r = v.shape
    wide = torch.zeros(t, count, r, device=v.device)
    has = torch.nonzero(ids >= 0)[:, 0]
    wide[has, ids[has]] = v[has]
    return wide.view(t, count * r)


def _gather(wide, ids, count):
    """The part of its adapter of each row; 0 for rows without one."""
    t = wide.shape[0]
    part = wide.view(t, count, -1)[torch.arange(t, device=wide.device), ids.clamp(min=0)]
    return torch.where((ids >= 0)[:, None], part, 0.0)


def _adapter_parts(s):
    count, r, k = s["a"].shape
    n = s["b"].shape[1]
    ids = s["ids"] if s["ids"] is not None else torch.zeros(s["x"].shape[0], dtype=torch.int64, device=s["x"].device)
    a = s["a"].float().view(count * r, k)
    b = (s["b"].float() * s["scale"][:, None, None]).transpose(1, 2).reshape(count * r, n)
    return ids, a, b, _gather(s["x"].float() @ a.t(), ids, count)


def _adapters(s):
    ids, a, b, v = _adapter_parts(s)
    y = s["y"].float() + _spread(v, ids, s["a"].shape[0]) @ b
    if s["relu"]:
        y = torch.where(y < 0, 0.0, y)
    return s["y"].copy_(y)


def _grad(s):
    ids, a, b, v = _adapter_parts(s)
    count, r, k = s["a"].shape
    dy = s["dy"].float()
    u = _spread(_gather(dy @ b.t(), ids, count), ids, count)
    da = (u.t() @ s["x"].float()).view(count, r, k)
    db = (dy.t() @ _spread(v, ids, count)).view(-1, count, r).transpose(0, 1) * s["scale"][:, None, None]
    dx = s["dx"].copy_(s["dx"].float() + u @ a)
    return dx, da.to(s["a"].dtype), db.to(s["b"].dtype)


def _softmax(x, heat):
    """(the probabilities' logarithms in 64 bits but for their normaliser's terms, which are 32 bits wide)"""
    top = x.amax(dim=1, keepdim=True)
    z = ((x - top) / heat).double()
    return z - torch.log(torch.exp(z.float()).sum(dim=1, keepdim=True, dtype=torch.float64))


def _first_best(value):
    """(the largest of each row, the lowest index that has it)"""
    top = value.amax(dim=1, keepdim=True)
    column = torch.arange(value.shape[1], device=value.device)
    return top[:, 0], torch.where(value == top, column, value.shape[1]).amin(dim=1)


def _verify(s):
    x, off, drafts, wide = s["logits"].float(), s["offsets"], s["drafts"], s["max"]
    batch, count, dev = off.shape[0] - 1, drafts.shape[0], x.device
    seq = torch.searchsorted(off, torch.arange(count, device=dev), right=True) - 1
    rows = torch.arange(count, device=dev) + seq
    own_seq = torch.searchsorted(off + torch.arange(batch + 1, device=dev), torch.arange(count + batch, device=dev), right=True) - 1
    heat = torch.ones(batch, device=dev) if s["temperature"] is None else s["temperature"]
    greedy, heat = heat == 0, torch.where(heat == 0, 1.0, heat)
    logp = _softmax(x, heat[own_seq][:, None])
    best = _first_best(x)[1]
    # which drafts stand
    lp = logp[rows, drafts]
    if s["q"] is None:
        fine = torch.log(s["uniform"].double()) < lp
    else:
        logq = _softmax(s["q"].float(), heat[seq][:, None])
        fine = torch.log(s["uniform"].double()) + logq[torch.arange(count, device=dev), drafts] < lp
    fine = torch.where(greedy[seq], drafts == best[rows], fine)
    at = torch.arange(wide, device=dev)
    there = off[:-1, None] + at
    within = there < off[1:, None]
    there = there.clamp(max=max(0, count - 1))
    stands = (fine[there] & within if count else within).long().cumprod(dim=1)
    accepted = stands.sum(dim=1)
    # the token that follows them
    last = off[:-1] + torch.arange(batch, device=dev) + accepted
    p = torch.exp(logp[last]).float()
    more = accepted < off[1:] - off[:-1]                     # a draft fell: the rest of the target without the draft's part
    if count:
        fell = (off[:-1] + accepted).clamp(max=count - 1)
        if s["q"] is None:
            q = torch.zeros_like(p)
            q[torch.arange(batch, device=dev), drafts[fell]] = 1.0
        else:
            q = torch.exp(logq[fell]).float()
        rest = torch.where(p > q, p - q, 0.0)
        use = more & (rest.amax(dim=1) > 0)
        p = torch.where(use[:, None], rest, p)
    score = torch.where(p > 0, p / s["noise"], -1.0)
    token = torch.where(greedy, best[last], _first_best(score)[1])
    tokens = torch.full((batch, wide + 1), -1, dtype=torch.int64, device=dev)
    logprob = torch.zeros(batch, wide + 1, device=dev)
    if count:
        tokens[:, :wide] = torch.where(stands > 0, drafts[there], -1)
        logprob[:, :wide] = torch.where(stands > 0, lp[there], 0.0).float()
    every = torch.arange(batch, device=dev)
    tokens[every, accepted] = token
    logprob[every, accepted] = logp[last, token].float()
    return accepted, tokens, logprob


def _clip(s):
    grads, out = s["grads"], s["out"]
    if s["kind"] == 2.0:
        norms = torch.sqrt(torch.stack([t.float().square().sum(dtype=torch.float64) for t in grads]))
        norm = torch.sqrt(norms.square().sum())
    else:
        norms = torch.stack([t.float().abs().amax() for t in grads]).double()
        norm = norms.amax()
    c = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    done = [t.copy_(f.float() * c) for t, f in zip(grads if out is None else out, grads)]
    return norm.float(), norms.float(), done


def run(s):
    op = s["op"]
    if own:
        import paper_2609_16742_gb300 as ct
        if op == "adapters":
            return ct.ct_adapters(s["y"], s["x"], s["a"], s["b"], s["ids"], s["scale"], relu=s["relu"])
        if op == "grad":
            return ct.ct_adapters_grad(s["dy"], s["x"], s["a"], s["b"], s["ids"], s["scale"], dx=s["dx"])
        if op == "verify":
            return ct.ct_verify_drafts(s["logits"], s["drafts"], s["offsets"], s["max"], s["uniform"], s["noise"],
                                       draft_logits=s["q"], temperature=s["temperature"])
        norm, norms = ct.ct_clip_grads(s["grads"], s["max_norm"], s["kind"], out=s["out"])
        return norm, norms, s["grads"] if s["out"] is None else s["out"]
    if op == "adapters":
        return _adapters(s)
    if op == "grad":
        return _grad(s)
    return _verify(s) if op == "verify" else _clip(s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op in ("adapters", "grad"):
        t, k, n, r = (case[c] for c in ("t", "k", "n", "rank"))
        wide = SIZE[case["out"]]
        used = min(case["adapters"], t)
        weights = used * r * (k + n) * size
        if op == "adapters":
            return {"bytes": t * k * size + weights + 2 * t * n * wide + 8 * t, "flops": 2 * t * r * (k + n)}
        return {"bytes": t * k * size + t * n * wide + 2 * t * k * wide + weights + case["adapters"] * r * (k + n) * size + 8 * t,
                "flops": 6 * t * r * (k + n)}
    if op == "verify":
        count, batch = sum(_lengths(case)), case["batch"]
        rows = count + batch + (0 if case["point"] else count)
        return {"bytes": rows * case["vocab"] * size + batch * case["vocab"] * 4 + 12 * count + 12 * batch * (case["drafts"] + 1),
                "flops": 4 * rows * case["vocab"]}
    return {"bytes": case["values"] * size * (2 if case["limit"] == "under" else 1), "flops": 3 * case["values"]}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_adapters(s):
    count, t = s["a"].shape[0], s["x"].shape[0]
    grad = s["op"] == "grad"
    y = (s["dx"] if grad else s["y"]).double()
    da, db = torch.zeros_like(s["a"], dtype=torch.float64), torch.zeros_like(s["b"], dtype=torch.float64)
    for i in range(count):
        mine = torch.arange(t, device=y.device) if s["ids"] is None else torch.nonzero(s["ids"] == i)[:, 0]
        x, a, b, scale = s["x"][mine].double(), s["a"][i].double(), s["b"][i].double(), s["scale"][i].double()
        if grad:
            dy = s["dy"][mine].double() * scale
            u = dy @ b
            da[i], db[i] = u.t() @ x, dy.t() @ (x @ a.t())
            y[mine] += u @ a
        else:
            y[mine] += scale * ((x @ a.t()) @ b.t())
    if grad:
        return y, da, db
    return y.clamp(min=0) if s["relu"] else y


def _exact_verify(s):
    off, wide = s["offsets"].tolist(), s["max"]
    batch = len(off) - 1
    heat = [1.0] * batch if s["temperature"] is None else s["temperature"].tolist()
    found = [0] * batch
    tokens, logprob = torch.full((batch, wide + 1), -1), torch.zeros(batch, wide + 1, dtype=torch.float64)
    for b in range(batch):
        x = s["logits"][off[b] + b:off[b + 1] + b + 1].double()
        logp = torch.log_softmax(x / (heat[b] or 1.0), dim=1)
        ids, u = s["drafts"][off[b]:off[b + 1]].tolist(), s["uniform"][off[b]:off[b + 1]].tolist()
        q = torch.zeros_like(logp[:-1])
        if s["q"] is not None:
            q = torch.softmax(s["q"][off[b]:off[b + 1]].double() / (heat[b] or 1.0), dim=1)
        elif ids:
            q[torch.arange(len(ids)), torch.tensor(ids)] = 1.0
        best = torch.nonzero(x == x.amax(dim=1, keepdim=True))
        first = {}
        for row, column in best.tolist():
            first.setdefault(row, column)
        j = 0
        while j < len(ids) and (ids[j] == first[j] if heat[b] == 0 else u[j] * float(q[j, ids[j]]) < math.exp(float(logp[j, ids[j]]))):
            tokens[b, j], logprob[b, j] = ids[j], float(logp[j, ids[j]])
            j += 1
        p = logp[j].exp()
        if j < len(ids):
            rest = (p - q[j]).clamp(min=0)
            p = rest if float(rest.max()) > 0 else p
        token = first[j] if heat[b] == 0 else int((p / s["noise"][b].double()).argmax())
        found[b], tokens[b, j], logprob[b, j] = j, token, float(logp[j, token])
    return torch.tensor(found), tokens, logprob


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] in ("adapters", "grad"):
        return _exact_adapters(s)
    if s["op"] == "verify":
        return _exact_verify(s)
    grads = [t.double() for t in s["grads"]]
    norms = torch.stack([torch.linalg.vector_norm(t, s["kind"]) for t in grads])
    norm = torch.linalg.vector_norm(norms, s["kind"])
    c = min(1.0, s["max_norm"] / float(norm))
    return norm, norms, [t * c for t in grads]
