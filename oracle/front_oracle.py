"""Plain fp64 definitions of what stands in front of the experts: routing with softmax or sigmoid scores, a bias, groups, and the norm.  NumPy on the
CPU, a token at a time where a choice is made; no code of the HIP path."""
import numpy as np

MASKED = -1e30


def _scores(logits, scores):
    """(fp64 logits, masked, s) of one token or many; an infinite logit is the largest finite one."""
    l = np.asarray(logits, dtype=np.float32)
    masked = ~(l > MASKED)
    l = np.minimum(np.where(masked, 0.0, l.astype(np.float64)), float(np.finfo(np.float32).max))
    if scores == "sigmoid":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-l))
    else:
        top = np.where(masked, -np.inf, l).max(-1, keepdims=True)
        e = np.exp(np.where(masked, -np.inf, l) - np.where(np.isfinite(top), top, 0.0))
        z = e.sum(-1, keepdims=True)
        s = e / np.where(z > 0, z, 1.0)
    return l, masked, np.where(masked, 0.0, s)


def _weights(l, masked, s, chosen, scores, renorm, scale):
    """Weights of one token's chosen experts; the ratio of scores that are far below zero is that of their exponentials."""
    if not renorm:
        return scale * s[chosen]
    live = chosen[~masked[chosen]]
    w = np.zeros(len(chosen))
    if len(live):
        top = l[live].max()
        if scores == "softmax":
            e = np.where(masked[chosen], 0.0, np.exp(np.minimum(l[chosen] - top, 0.0)))
        else:
            top = min(top, 0.0)
            with np.errstate(over="ignore"):
                e = np.where(masked[chosen], 0.0, 1.0 / (np.exp(top - l[chosen]) + np.exp(top)))
        w = e / e.sum()
    return scale * w


def gate_fwd(logits, bias, k, scores, groups=1, kept=1, best=1, renorm=True, scale=1.0, n_shared=0):
    """logits [T, E] fp32, bias [E] fp32 or None -> topk_idx [T, k + n_shared] int32, topk_w fp64."""
    T, E = logits.shape
    size = E // groups
    idx = np.empty((T, k + n_shared), np.int32)
    w = np.ones((T, k + n_shared))
    for t in range(T):
        l, masked, s = _scores(logits[t], scores)
        with np.errstate(invalid="ignore"):
            c = l if bias is None else s + bias.astype(np.float64)
        c = np.where(masked | ~(c > np.float32(MASKED)), -np.inf, c)
        of = s if bias is None and best == 2 else c
        rating = []
        for g in range(groups):
            part = [of[e] for e in range(g * size, (g + 1) * size) if c[e] != -np.inf]
            rating.append(sum(sorted(part, reverse=True)[:best]) if part else -np.inf)
        stay = sorted(range(groups), key=lambda g: (-rating[g], g))[:kept]
        pool = [e for g in stay for e in range(g * size, (g + 1) * size)]
        chosen = np.array(sorted(pool, key=lambda e: (-c[e], e))[:k])
        idx[t, :k], w[t, :k] = chosen, _weights(l, masked, s, chosen, scores, renorm, scale)
    idx[:, k:] = np.arange(E, E + n_shared)
    return idx, w


def gate_weights(logits, idx, scores, renorm, scale):
    """Weights of given choices [T, k] (what gate_bwd differentiates), fp64 logits allowed."""
    out = np.empty(idx.shape)
    for t in range(len(idx)):
        l = np.asarray(logits[t], np.float64)
        s = 1.0 / (1.0 + np.exp(-l)) if scores == "sigmoid" else np.exp(l - l.max()) / np.exp(l - l.max()).sum()
        out[t] = s[idx[t]] / (s[idx[t]].sum() if renorm else 1.0) * scale
    return out


def balance_loss(logits, counts, k, scores, balance):
    l = np.asarray(logits, np.float64)
    s = 1.0 / (1.0 + np.exp(-l)) if scores == "sigmoid" else np.exp(l - l.max(1, keepdims=True))
    q = s / s.sum(1, keepdims=True)
    T, E = l.shape
    return balance * E / (k * T * T) * float((q.sum(0) * counts[:E]).sum())


def gate_bwd(dtopk_w, logits, idx, w, k, scores, renorm=True, scale=1.0, counts=None, balance=0.0):
    """(dlogits, loss, magnitude of dlogits' terms), all fp64; idx, w [T, >= k] as the forward call gave them."""
    T, E = logits.shape
    l, masked, s = _scores(logits, scores)
    slope = np.where(masked, 0.0, 1.0 - s) if scores == "sigmoid" else np.ones_like(s)
    if scores == "sigmoid":   # (1 - s without cancellation)
        with np.errstate(over="ignore"):
            slope = np.where(masked, 0.0, 1.0 / (1.0 + np.exp(l)))
    w, dw = w[:, :k].astype(np.float64), dtopk_w[:, :k].astype(np.float64)
    inner = (w * dw).sum(1, keepdims=True)
    size_inner = np.abs(w * dw).sum(1, keepdims=True)
    d = w * (dw - inner / scale) if renorm else w * dw
    size_d = np.abs(w) * (np.abs(dw) + size_inner / scale) if renorm else np.abs(w * dw)
    out, size = np.zeros((T, E)), np.zeros((T, E))
    for j in range(k):
        np.add.at(out, (np.arange(T), idx[:, j]), d[:, j])
        np.add.at(size, (np.arange(T), idx[:, j]), size_d[:, j])
    if scores == "softmax" and not renorm:
        out -= s * inner
        size += s * size_inner
    loss = 0.0
    if counts is not None:
        cost = counts[:E].astype(np.float64) * (balance * E / (k * max(T, 1) ** 2))
        if scores == "sigmoid":   # (over the largest one: scores far below zero keep their ratios)
            top = np.minimum(np.where(masked, -np.inf, l).max(1, keepdims=True), 0.0)
            top = np.where(np.isfinite(top), top, 0.0)
            with np.errstate(over="ignore"):
                e = np.where(masked, 0.0, 1.0 / (np.exp(top - l) + np.exp(top)))
        else:
            e = s
        z = e.sum(1, keepdims=True)
        q = e / np.where(z > 0, z, 1.0)
        mean = (q * cost).sum(1, keepdims=True)
        out += q * (cost - mean)
        size += q * (np.abs(cost) + np.abs(mean))
        loss = float(mean.sum())
    return out * slope, loss, size * slope


def norm_fwd(h, gamma, beta, centre, eps):
    """h [rows, cols] fp64 -> y, mean, rstd."""
    mean = h.mean(1, keepdims=True) if centre else np.zeros((h.shape[0], 1))
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (h - mean) * rstd
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean[:, 0], rstd[:, 0]


def norm_bwd(dy, h, gamma, mean, rstd, centre, addend=None):
    """dx, dgamma, dbeta and the magnitudes of their terms."""
    xh = (h - (mean[:, None] if centre else 0.0)) * rstd[:, None]
    loose = (np.abs(h) + (np.abs(mean[:, None]) if centre else 0.0)) * rstd[:, None]
    g = dy * (1.0 if gamma is None else gamma)
    sgx = (g * xh).mean(1, keepdims=True)
    sg = g.mean(1, keepdims=True) if centre else 0.0
    dx = rstd[:, None] * (g - sg - xh * sgx)
    size = rstd[:, None] * (np.abs(g) + (np.abs(g).mean(1, keepdims=True) if centre else 0.0) + loose * (np.abs(g) * loose).mean(1, keepdims=True))
    if addend is not None:
        dx, size = dx + addend, size + np.abs(addend)
    return dx, (dy * xh).sum(0), dy.sum(0), size, (np.abs(dy) * loose).sum(0), np.abs(dy).sum(0)
