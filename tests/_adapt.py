"""Plain 64-bit implementations of the adapters, clipping and verification of drafts, and the bounds their tests use."""
import math

import numpy as np

# half a step of each type, and its smallest step
HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}      # torch.finfo(t).eps / 2
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}


def name(dtype):
    return str(dtype).replace("torch.", "")


def steps(k):
    """Additions in 32 bits on the way of one sum of k products: at most 512 values (32 steps of 16) are added into one sum,
    those sums into another; 16 more for joins between lanes, splits and what is added at the end."""
    return 32 + k / 512 + 16


# A sum may lose a whole unit of its last place (2^-23) at each addition, as a sum that is cut off does.
UNIT = 2.0 ** -23
# The short vectors between the two products go on as two 16-bit parts for results of 16 bits (8 bits each at least: 2^-16), as three
# for results of 32 (or two of 11 bits relative to a row's largest: 2^-21).
PARTS = {"float32": 2.0 ** -21, "float16": 2.0 ** -15, "bfloat16": 2.0 ** -15}


def adapters(y, x, a, b, ids, scale, relu):
    """(result, its magnitude: |y| + scale |B| |A| |x|, the adapters' part of that)"""
    out, mag, part = y.copy(), np.abs(y), np.zeros_like(y)
    for t in range(x.shape[0]):
        i = 0 if ids is None else ids[t]
        if i == -1:
            continue
        if not 0 <= i < a.shape[0]:
            out[t] = np.nan
            continue
        s = 1.0 if scale is None else scale[i]
        out[t] += s * (b[i] @ (a[i] @ x[t]))
        part[t] = abs(s) * (np.abs(b[i]) @ (np.abs(a[i]) @ np.abs(x[t])))
    if relu:
        out = np.where(out < 0, 0.0, out)
    return out, mag + part, part


def adapters_bound(want, mag, part, k, rank, dtype):
    d = name(dtype)
    return HALF[d] * np.abs(want) * (1 + 2.0 ** -7) + UNIT * (steps(k) + steps(rank)) * mag + PARTS[d] * part + TINY[d]


def adapters_grad(dy, x, a, b, ids, scale, dx):
    """((dx, da, db), their magnitudes)"""
    t_, count = x.shape[0], a.shape[0]
    dx, mx = dx.copy(), np.abs(dx)
    da, db = np.zeros(a.shape), np.zeros(b.shape)
    ma, mb = np.zeros(a.shape), np.zeros(b.shape)
    for t in range(t_):
        i = 0 if ids is None else ids[t]
        if i == -1:
            continue
        if not 0 <= i < count:
            dx[t] = np.nan
            continue
        s = 1.0 if scale is None else scale[i]
        u, v = s * (dy[t] @ b[i]), s * (a[i] @ x[t])
        mu, mv = abs(s) * (np.abs(dy[t]) @ np.abs(b[i])), abs(s) * (np.abs(a[i]) @ np.abs(x[t]))
        dx[t] += u @ a[i]
        mx[t] += mu @ np.abs(a[i])
        da[i] += np.outer(u, x[t])
        ma[i] += np.outer(mu, np.abs(x[t]))
        db[i] += np.outer(dy[t], v)
        mb[i] += np.outer(np.abs(dy[t]), mv)
    return (dx, da, db), (mx, ma, mb)


def grad_bound(want, mag, lengths, dtype):
    d = name(dtype)
    return HALF[d] * np.abs(want) * (1 + 2.0 ** -7) + (UNIT * sum(steps(n) for n in lengths) + PARTS[d]) * mag + TINY[d]


def clip(grads, max_norm, kind):
    """(norm, norms, factor) of float64 arrays; the factor is 1 where the norm is not finite."""
    if kind == 2:
        # scaled: squares of large or small values would leave the range
        norms = []
        for g in grads:
            top = np.abs(g).max(initial=0.0)
            norms.append(top if top == 0 or not np.isfinite(top) else top * math.sqrt(((g / top) ** 2).sum()))
        norms = np.array(norms)
        top = norms.max(initial=0.0)
        norm = top if top == 0 or not np.isfinite(top) else top * math.sqrt(((norms / top) ** 2).sum())
    else:
        norms = np.array([np.abs(g).max(initial=0.0) for g in grads])
        norm = norms.max(initial=0.0)
    return norm, norms, max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0


# A probability's relative error: the exponent (x - m) / T, at most 64 where the probability counts, is rounded twice in 32 bits
# (2 x 64 x 2^-24 x log2(e)) next to the functions' few units of 2^-23; the normaliser's part is smaller.
PROB = 2.0 ** -15


def softmax(x, heat):
    m = x.max(initial=-math.inf)
    if m == -math.inf:
        return np.zeros(x.shape), -math.inf
    with np.errstate(over="ignore"):
        e = np.exp((x - m) * heat)
    return e / e.sum(), m * heat + math.log(e.sum())


def first_best(x):
    return int(np.flatnonzero(x == x.max())[0]) if x.size and x.max() > -math.inf else -1


def check_verify(got, x, q, drafts, offsets, most, uniform, noise, temperature):
    """Asserts that (accepted, token, logprob) are what the definition gives, up to PROB where a comparison is that close."""
    accepted, token, logprob = got
    count = drafts.shape[0]
    for b in range(offsets.shape[0] - 1):
        lo = min(max(int(offsets[b]), 0), count)
        d = min(min(max(int(offsets[b + 1]), lo), count) - lo, most)
        t = 1.0 if temperature is None else float(temperature[b])
        greedy, bad_t = t < 1e-30, not (0 <= t < math.inf)
        heat = 1.0 if greedy or bad_t else 1.0 / t
        n = int(accepted[b])
        assert 0 <= n <= d, (b, n, d)
        assert (token[b, n + 1:] == -1).all() and (logprob[b, n + 1:] == 0).all(), b
        ended = bad_t
        for j in range(n + 1):
            row = x[lo + b + j]
            needs_q = q is not None and not greedy and j < d
            ended = bad_t or not (row < math.inf).all() or (needs_q and not (q[lo + j] < math.inf).all())
            if ended:
                break
            p, lse = softmax(row, heat)
            qj = np.zeros_like(p)
            if j < d:
                i = int(drafts[lo + j])
                there = 0 <= i < p.size
                if needs_q:
                    qj = softmax(q[lo + j], heat)[0]
                elif there:
                    qj[i] = 1.0
                # u q < p in logarithms: at a small T both leave the range of 64 bits, their ratio does not
                lp = row[i] * heat - lse if there and row[i] > -math.inf else -math.inf
                lq = 0.0
                if needs_q and there:
                    lq = q[lo + j][i] * heat - softmax(q[lo + j], heat)[1] if q[lo + j][i] > -math.inf else -math.inf
                side = (math.log(uniform[lo + j]) if uniform[lo + j] > 0 else -math.inf) + lq
                near = 2 * PROB + 2.0 ** -22 * sum(abs(v) for v in (lp, lq) if v > -math.inf)
                if j < n:
                    assert there and token[b, j] == i, (b, j)
                    if greedy:
                        assert i == first_best(row), (b, j)
                    else:
                        assert lp > -math.inf and side <= lp + near, (b, j, side, lp)
                    want = row[i] * heat - lse
                    assert abs(logprob[b, j] - want) <= 2.0 ** -22 * (abs(want) + abs(row[i] * heat) + abs(lse)) + PROB / 16, (b, j)
                elif greedy:
                    assert i != first_best(row), (b, j)
                else:
                    assert lp == -math.inf or side >= lp - near, (b, j, side, lp)
        if ended:
            assert j == n and token[b, n] == -1 and math.isnan(logprob[b, n]), (b, n, token[b], logprob[b])
            continue
        got_token = int(token[b, n])
        if lse == -math.inf:
            assert got_token == -1 and logprob[b, n] == -math.inf, (b, n, got_token)
            continue
        assert 0 <= got_token < p.size, (b, got_token)
        want = row[got_token] * heat - lse
        assert abs(logprob[b, n] - want) <= 2.0 ** -22 * (abs(want) + abs(row[got_token] * heat) + abs(lse)) + PROB / 16, (b, n)
        if greedy:
            assert got_token == first_best(row), (b, got_token, first_best(row))
            continue
        w = np.maximum(p - qj, 0.0) if n < d else p
        slack = PROB * (p + qj) if n < d else PROB * p
        if n < d and w.max() <= 0:
            w, slack = p, PROB * p
        e = noise[b]
        best = ((w - slack) / e).max()
        assert (w[got_token] + slack[got_token]) / e[got_token] >= best, (b, n, got_token)


def same_as_defined(got, x, q, drafts, offsets, most, uniform, noise, temperature):
    check_verify(tuple(g.cpu().numpy() for g in got), x.double().cpu().numpy(), None if q is None else q.double().cpu().numpy(),
                 drafts.cpu().numpy(), offsets.cpu().numpy(), most, uniform.double().cpu().numpy(), noise.double().cpu().numpy(),
                 None if temperature is None else temperature.double().cpu().numpy())
