"""Plain implementation of the operators on rows of class logits in 64 bits (numpy, row by row, from the formulas of
include/isr.h), and how far results in 32 bits may lie from it."""
import numpy as np

U = 2.0 ** -24   # half a step of fp32, relative

# A row's sum is taken by threads in runs of at most 128 terms and joined in at most 40 levels of 4 roundings each; an
# exponential is off by 2 units of the last place and by its argument's rounding.  In all SUM half steps of the sum.
SUM = 128 + 160 + 8


def logp_tol(logp):
    """Of a log-probability: difference, product with the scale, its share in the exponentials' arguments, the sum's."""
    with np.errstate(invalid="ignore"):
        return U * (4 * np.where(np.isfinite(logp), np.abs(logp), 0.0) + SUM)


def row_logp(x, scale):
    """(log p, empty, bad) of a row of float64 or int64 logits."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or (x == np.inf).any():
        return np.full(x.shape, np.nan), False, True
    m = x.max()
    if m == -np.inf:
        return np.full(x.shape, -np.inf), True, False
    with np.errstate(over="ignore"):
        d = scale * (x - m)
    return d - np.log(np.exp(d).sum()), False, False


def _weighted(p, v):
    out = np.zeros_like(p)
    np.multiply(p, v, out=out, where=p > 0)
    return out


def logprobs(x, scale, given=None, top=0):
    """Lists over rows: log-probabilities of the given, entropies, top classes, their log-probabilities."""
    lp, h, tc, tl = [], [], [], []
    for r, row in enumerate(x):
        logp, empty, bad = row_logp(row, scale)
        n = len(logp)
        if given is not None:
            lp.append([0.0 if c < 0 else np.nan if c >= n or bad else logp[c] for c in given[r]])
        h.append(np.nan if bad else 0.0 if empty else -_weighted(np.exp(logp), logp).sum())
        if bad:
            tc.append([-1] * top)
            tl.append([np.nan] * top)
        else:
            order = np.argsort(-np.asarray(row, dtype=np.float64), kind="stable")[:top]
            some = np.asarray(row, dtype=np.float64)[order] > -np.inf
            tc.append(np.where(some, order, -1))
            tl.append(np.where(some, logp[order], -np.inf))
    return (np.array(lp, dtype=np.float64).reshape(len(x), -1), np.array(h), np.array(tc, dtype=np.int64).reshape(len(x), top),
            np.array(tl, dtype=np.float64).reshape(len(x), top))


def logprobs_grad(x, scale, given, up, up_h):
    """(gradient, tolerance before its rounding to the logits' type)"""
    g, tol = np.zeros(x.shape), np.zeros(x.shape)
    for r, row in enumerate(x):
        logp, empty, bad = row_logp(row, scale)
        u_h = 0.0 if up_h is None else up_h[r]
        counted = [i for i in range(given.shape[1]) if given[r, i] >= 0] if given is not None else []
        if empty or (not counted and u_h == 0):
            continue
        if bad or any(given[r, i] >= len(logp) for i in counted):
            g[r] = np.nan
            continue
        p = np.exp(logp)
        plogp = _weighted(p, logp)
        h = -plogp.sum()
        total = sum(up[r, i] for i in counted)
        g[r] = -p * total - u_h * (plogp + p * h)
        size = p * sum(abs(up[r, i]) for i in counted) + abs(u_h) * (p * (h + 1) - plogp)
        # the entropy's own error: a sum like the row's, of terms |log p|
        tol[r] = size * U * (SUM + 4 * np.where(p > 0, np.abs(np.where(p > 0, logp, 0)), 0)) + p * abs(u_h) * U * SUM * (2 + h)
        for i in counted:
            g[r, given[r, i]] += up[r, i]
            tol[r, given[r, i]] += 8 * U * abs(up[r, i])
        g[r] *= scale
        tol[r] = scale * (tol[r] + 4 * U * np.abs(g[r]) / scale)
    return g, tol


def distill(x, scale, entry, value, value_scale, rest, weight=None):
    """(loss, its tolerance, gradient, its tolerance before the rounding to the logits' type)"""
    rows, n = x.shape
    loss, ltol, g, gtol = np.zeros(rows), np.zeros(rows), np.zeros(x.shape), np.zeros(x.shape)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        there = np.flatnonzero(entry[r] >= 0)
        c, v = entry[r][there], np.asarray(value[r], dtype=np.float64)[there] * value_scale
        if len(there) == 0 or (not rest and v.max() == -np.inf):
            continue
        logp, empty, bad = row_logp(x[r], scale)
        if bad or (c >= n).any() or np.isnan(v).any() or (v == np.inf).any():
            loss[r] = np.nan
            g[r] = np.nan if w != 0 else 0
            continue
        logq = v if rest else v - v.max() - np.log(np.exp(v - v.max()).sum())
        q = np.exp(logq)
        member = np.zeros(n, dtype=bool)
        member[c] = True
        parts = [(q[i], logq[i], logp[c[i]]) for i in range(len(c)) if q[i] > 0]
        total, left = q.sum(), 0.0
        if rest:
            left = max(0.0, 1.0 - total)
            total += left
            others = logp[~member]
            top = others.max() if len(others) else -np.inf
            logr = top + np.log(np.exp(others - top).sum()) if top > -np.inf else -np.inf
            if left > 0:
                parts.append((left, np.log(left), logr))
        with np.errstate(invalid="ignore"):
            loss[r] = sum(a * (b - d) for a, b, d in parts)
            ltol[r] = sum(a * (2 * logp_tol(d) + U * (8 * abs(b) + 8)) for a, b, d in parts) + 4 * U * abs(loss[r])
        if empty or w == 0:
            continue
        p = np.exp(logp)
        g[r] = total * p
        rel = U * (SUM + 4 * np.where(p > 0, np.abs(np.where(p > 0, logp, 0)), 0))
        gtol[r] = total * p * rel
        if rest:
            inside = np.exp(logp[~member] - logr) if logr > -np.inf else np.zeros((~member).sum())
            pr = np.exp(logr)
            g[r, ~member] = inside * (total * pr - left)
            gtol[r, ~member] = inside * (total * pr * U * (2 * SUM + 8 * (abs(logr) if logr > -np.inf else 0)) + left * 4 * U) + np.abs(g[r, ~member]) * rel[~member]
        for i in range(len(c)):
            g[r, c[i]] -= q[i]
            gtol[r, c[i]] += q[i] * U * (16 + 4 * abs(logq[i]) if q[i] > 0 else 0)
        gtol[r] = (gtol[r] + 4 * U * np.abs(g[r])) * scale * abs(w)
        g[r] *= scale * w
    return loss, ltol, g, gtol
