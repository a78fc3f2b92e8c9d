"""Plain 64-bit implementations of the 8-bit answer head, for its tests."""
import math

import numpy as np

E4M3_MAX = 448.0


def round_e4m3(v):
    """Nearest e4m3 value (ties to even) of finite v with |v| <= 448."""
    a = np.abs(v)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    unit = 2.0 ** (e - 3)
    return np.copysign(np.rint(a / unit) * unit, v)


def quantize(x, block_rows):
    """(values the 8-bit words stand for, scales) of a float64 matrix."""
    m, k = x.shape
    mb, kb = -(-m // block_rows), -(-k // 128)
    q = np.full((m, k), np.nan)
    s = np.ones((mb, kb))
    for i in range(mb):
        for b in range(kb):
            part = x[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128]
            fine = np.isfinite(part)
            amax = np.abs(part[fine]).max(initial=0.0)
            if amax > 0:
                e = -126
                while amax > E4M3_MAX * 2.0 ** e:
                    e += 1
                s[i, b] = 2.0 ** e
            q[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128][fine] = round_e4m3(part[fine] / s[i, b])
    return q, s


def widen(s, block_rows, m, k):
    return np.repeat(np.repeat(s, block_rows, 0)[:m], 128, 1)[:, :k]


def product(xv, wv, bias=None, relu=False):
    y = xv @ wv.T
    if bias is not None:
        y = y + bias
    return np.where(y < 0, 0.0, y) if relu else y


def logprobs(x, ids, k):
    """Definitions of ct_logprobs in 64 bits, one row at a time; what exceeds
    FP32's range is -inf, as in its FP32 outputs."""
    rows, vocab = x.shape
    lp, h, lse = np.zeros(rows), np.zeros(rows), np.full(rows, -math.inf)
    top_lp, top_id = np.full((rows, k), -math.inf), np.full((rows, k), -1, np.int64)
    for r in range(rows):
        row = x[r]
        if np.isnan(row).any() or (row == math.inf).any():
            lp[r] = h[r] = lse[r] = math.nan
            top_lp[r] = math.nan
            continue
        live = np.nonzero(row > -math.inf)[0]
        if len(live):
            v = row[live]
            m = v.max()
            z = np.exp(v - m).sum()
            lse[r] = m + math.log(z)
            p = np.exp(v - m) / z
            with np.errstate(divide="ignore", invalid="ignore"):
                h[r] = -np.where(p > 0, p * (v - m - math.log(z)), 0.0).sum()
            order = live[np.lexsort((live, -v))][:k]
            top_id[r, :len(order)] = order
            top_lp[r, :len(order)] = row[order] - lse[r]
        if ids[r] != -1:
            lp[r] = math.nan if not 0 <= ids[r] < vocab else row[ids[r]] - lse[r] if row[ids[r]] > -math.inf else -math.inf
    for a in (lp, h, lse, top_lp):
        with np.errstate(over="ignore", invalid="ignore"):
            far = np.isinf(a.astype(np.float32))
        a[far] = np.copysign(math.inf, a[far])
    return lp, h, lse, top_lp, top_id


def grad(x, ids, lse, h, g, gh):
    """Gradient of sum(g * logprob + gh * entropy), from given lse and entropy."""
    with np.errstate(invalid="ignore", over="ignore"):
        lp = x - lse[:, None]
        p = np.where(x == -math.inf, 0.0, np.exp(lp))
        has = (ids >= 0) & (ids < x.shape[1])
        ge = np.where(ids == -1, 0.0, np.where(has, g, np.nan))[:, None]
        d = np.where(p == 0, 0.0, -p * (ge + gh[:, None] * (lp + h[:, None])))
    for r in np.nonzero(has)[0]:
        d[r, ids[r]] += g[r]
    d[np.isnan(lse) | np.isnan(ge[:, 0])] = np.nan
    return d
