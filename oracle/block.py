"""Float64 definitions of the operators around a compressed layer: the norms of its
residual block, the router's balance loss and the distillation loss, each with its
gradient.  Plain numpy; nothing of the CUDA path is used.
"""
from __future__ import annotations

import numpy as np


def _gate(gate, T, H):
    """The gate as [T, H]: None, [H], [T, 1] or [T, H]."""
    return np.ones((T, H)) if gate is None else np.broadcast_to(gate, (T, H))


def residual_norm(r, y=None, w_post=None, gate=None, w_pre=None, a=1.0, off=0.0, eps=1e-6):
    """(r_out, h, parts): the block's output normalised, gated and added to a r, and
    the sum normalised (h None without w_pre)."""
    T, H = r.shape
    p = dict(s1=np.ones((T, 1)), s2=np.ones((T, 1)), n=None, u=None)
    out = a * r
    if y is not None:
        if w_post is not None:
            p["s1"] = 1.0 / np.sqrt((y * y).mean(1, keepdims=True) + eps)
        p["n"] = y * p["s1"]
        p["u"] = p["n"] * (off + w_post) if w_post is not None else y
        out = out + _gate(gate, T, H) * p["u"]
    h = None
    if w_pre is not None:
        p["s2"] = 1.0 / np.sqrt((out * out).mean(1, keepdims=True) + eps)
        h = out * p["s2"] * (off + w_pre)
    return out, h, p


def residual_norm_grads(dr_out, dh, r, y=None, w_post=None, gate=None, w_pre=None, a=1.0, off=0.0,
                        eps=1e-6):
    """Gradients of sum(r_out dr_out) + sum(h dh) as a dict, each also as the sum of its
    terms' magnitudes ("|name|"), by which rounding errors go."""
    T, H = r.shape
    out, _, p = residual_norm(r, y, w_post, gate, w_pre, a, off, eps)
    D = np.zeros((T, H)) if dr_out is None else dr_out.astype(np.float64)
    M = np.abs(D)
    g = {}
    if w_pre is not None:
        x, d = out * p["s2"], np.zeros((T, H)) if dh is None else dh
        xm = np.abs(a * r) if y is None else np.abs(a * r) + np.abs(_gate(gate, T, H) * p["u"])
        xm = xm * p["s2"]                           # x is a sum, and its error goes by its terms
        e = d * (off + w_pre)
        D = D + p["s2"] * (e - x * (e * x).mean(1, keepdims=True))
        M = M + p["s2"] * (np.abs(e) + xm * (np.abs(e) * xm).mean(1, keepdims=True))
        g["dw_pre"], g["|dw_pre|"] = (d * x).sum(0), (np.abs(d) * xm).sum(0)
    g["dr"], g["|dr|"] = a * D, abs(a) * M
    if y is not None:
        if gate is not None:
            axis = 0 if gate.ndim == 1 else 1 if gate.shape == (T, 1) and H > 1 else None
            total = lambda v: v if axis is None else v.sum(axis, keepdims=axis == 1)  # noqa: E731
            g["dgate"], g["|dgate|"] = total(D * p["u"]), total(M * np.abs(p["u"]))
        G = _gate(gate, T, H)
        f, fm = D * G, M * np.abs(G)
        if w_post is None:
            g["dy"], g["|dy|"] = f, fm
        else:
            n, m = p["n"], np.abs(p["n"])
            g["dw_post"], g["|dw_post|"] = (f * n).sum(0), (fm * m).sum(0)
            f, fm = f * (off + w_post), fm * np.abs(off + w_post)
            g["dy"] = p["s1"] * (f - n * (f * n).mean(1, keepdims=True))
            g["|dy|"] = p["s1"] * (fm + m * (fm * m).mean(1, keepdims=True))
    return g


def _counted(logits, mask):
    """Rows that count: mask not 0 and some logit above -inf."""
    on = np.ones(len(logits), bool) if mask is None else np.asarray(mask) != 0
    return on & ~np.all(np.isneginf(logits), axis=1)


def router_balance(logits, ids, mask=None, alpha=0.01, beta=0.0):
    """(loss, balance, z), counts [E + 1] (the counted tokens last), prob [E], lse [T]."""
    T, E = logits.shape
    k = ids.shape[1]
    counts, prob, lse, z = np.zeros(E + 1, np.int64), np.zeros(E), np.full(T, -np.inf), 0.0
    for t in np.flatnonzero(_counted(logits, mask)):
        m = logits[t].max()
        ex = np.exp(logits[t] - m)
        lse[t] = m + np.log(ex.sum())
        prob += ex / ex.sum()
        z += lse[t] ** 2
        for e in set(int(i) for i in ids[t]):
            if 0 <= e < E:
                counts[e] += 1
        counts[E] += 1
    n = counts[E]
    if n == 0:
        return np.zeros(3), counts, prob, lse
    prob /= n
    bal = E * float((counts[:E] / (n * k) * prob).sum())
    return np.array([alpha * bal + beta * z / n, bal, z / n]), counts, prob, lse


def router_balance_grad(logits, ids, mask=None, alpha=0.01, beta=0.0, dloss=1.0):
    """Gradient of dloss times the loss with respect to the logits, counts fixed."""
    T, E = logits.shape
    _, counts, _, lse = router_balance(logits, ids, mask, alpha, beta)
    n, c = counts[E], counts[:E].astype(np.float64)
    d = np.zeros((T, E))
    for t in np.flatnonzero(_counted(logits, mask)):
        p = np.exp(logits[t] - lse[t])
        d[t] = dloss * p * (alpha * E / (float(n) ** 2 * ids.shape[1]) * (c - (c * p).sum())
                            + 2 * beta / n * lse[t])
    return d


def _log_softmax(z):
    m = z.max()
    return z - m - np.log(np.exp(z - m).sum())


def distill(logits, ids, top, tau=1.0, top_lse=None, a=1.0, labels=None, b=0.0, weight=None,
            magnitude=False):
    """(loss [T], gradient of its sum [T, V]) of distillation from the teacher's entries;
    with `magnitude` also the sums of the gradient's terms' magnitudes."""
    T, V = logits.shape
    loss, grad, mag = np.zeros(T), np.zeros((T, V)), np.zeros((T, V))
    for t in range(T):
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0 or np.all(np.isneginf(logits[t])):
            continue

        def term(at, v):
            grad[t, at] += v
            mag[t, at] += np.abs(v)

        lp = _log_softmax(logits[t] / tau)
        keep = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < V and not np.isneginf(top[t, j])]
        if keep:
            tj = np.array([top[t, j] for j in keep]) / tau
            lq = tj - top_lse[t] if top_lse is not None else _log_softmax(tj)
            for j, l in zip(keep, lq):
                q, v = np.exp(l), ids[t, j]
                if q > 0:
                    loss[t] += a * tau ** 2 * q * (l - lp[v])
                term(slice(None), a * tau * q * np.exp(lp))
                term(v, -a * tau * q)
        if labels is not None and 0 <= labels[t] < V:
            l1 = _log_softmax(logits[t])
            loss[t] -= b * l1[labels[t]]
            term(slice(None), b * np.exp(l1))
            term(labels[t], -b)
        loss[t] *= w
        grad[t] *= w
        mag[t] *= abs(w)
    return (loss, grad, mag) if magnitude else (loss, grad)
