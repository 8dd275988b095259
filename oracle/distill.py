"""Top logits, the divergence from them and cross entropy from hidden states, in float64.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

top_logits   the k largest entries of a row, best first, equal ones by ascending index, and
             tau log sum exp(x_j / tau) over the others.
distill      KL between softmax over (listed logits, rest) / tau and the student's shares of the same
             buckets, with its gradient by the buckets' own derivatives: d p_b / d s_j =
             p_j ([j in b] - p_b) / tau.
linear_ce    -w_r log softmax(X W^T)[r, y_r] and its gradients.
"""
import numpy as np


def _lse(x):
    m = np.max(x)
    return m + np.log(np.sum(np.exp(x - m))) if np.isfinite(m) else m


def top_logits(x, k, tau=1.0):
    """(logit [n, k], token [n, k], rest [n]) of x [n, V]."""
    x = np.asarray(x, dtype=np.float64) + 0.0  # (-0 becomes 0)
    order = np.argsort(-x, axis=1, kind="stable")
    tok = order[:, :k]
    rest = np.array([tau * _lse(row[o[k:]] / tau) if k < x.shape[1] else -np.inf for row, o in zip(x, order)])
    return np.take_along_axis(x, tok, 1), tok.astype(np.int32), rest


def distill_row(s, token, logit, rest, tau=1.0, reverse=False):
    """(loss, gradient [V]) of one row; rest None: -infinity.  None: the row's divergence is not defined."""
    s = np.asarray(s, dtype=np.float64)
    V = len(s)
    if np.any(token < -1):
        return None
    keep = token >= 0
    token, logit = token[keep], np.asarray(logit, dtype=np.float64)[keep]
    rest = -np.inf if rest is None else float(rest)
    if len(set(token.tolist())) < len(token) or np.any(token >= V) or np.any(np.isnan(logit)) or np.any(logit == np.inf):
        return None
    if np.isnan(rest) or rest == np.inf:
        return None
    n = len(token)
    teach = np.append(logit, rest) / tau
    if not np.any(teach > -np.inf):
        return 0.0, np.zeros(V)
    logt = teach - _lse(teach)
    z = s / tau
    logp = z - _lse(z)
    bucket = np.full(V, n)
    bucket[token] = np.arange(n)
    others = n < V
    logpb = np.append(logp[token], _lse(logp[bucket == n]) if others else -np.inf)
    p, t, pb = np.exp(logp), np.exp(logt), np.exp(logpb)
    if reverse:
        if np.any(logt[:n] == -np.inf) or (others and logt[n] == -np.inf):
            return None
        each = np.where(pb > 0, logpb - np.where(pb > 0, logt, 0.0), 0.0)
        loss = np.sum(np.where(pb > 0, pb * each, 0.0))
        slope = np.where(pb > 0, each + 1.0, 0.0)
    else:
        if rest > -np.inf and not others:
            return None
        part = t > 0
        loss = np.sum(np.where(part, t * (np.where(part, logt, 0.0) - np.where(part, logpb, 0.0)), 0.0))
        # d loss / d p_b = -t_b / p_b, in logarithms: p_b may be far below the least number
        grad = p * np.sum(t) - np.exp(logp - np.where(bucket < n, logp, logpb[n])) * t[bucket]
        return loss, grad / tau
    mean = np.sum(slope * pb)
    return loss, p * (slope[bucket] - mean) / tau


def linear_ce(x, w, token, weight=None, valid=None, scale=1.0):
    """(loss [n], logp [n], dx, dw) for float64 arrays."""
    n, V = len(x), len(w)
    weight = np.ones(n) if weight is None else np.asarray(weight, dtype=np.float64)
    valid = np.ones(n, dtype=bool) if valid is None else np.asarray(valid) != 0
    bad = valid & ((token < 0) | (token >= V) | ~np.isfinite(weight))
    take = np.where(valid & ~bad)[0]
    loss, logp = np.zeros(n), np.zeros(n)
    dx, dw = np.zeros_like(x), np.zeros_like(w)
    logits = x[take] @ w.T
    lp = logits - np.array([_lse(l) for l in logits]).reshape(-1, 1)
    logp[take] = lp[np.arange(len(take)), token[take]]
    loss[take] = -weight[take] * logp[take]
    d = np.exp(lp)
    d[np.arange(len(take)), token[take]] -= 1.0
    d *= scale * weight[take][:, None]
    dx[take] = d @ w
    dw += d.T @ x[take]
    for a in (loss, logp, dx):
        a[bad] = np.nan
    return loss, logp, dx, dw
