"""Float64 definitions of the products around a compressed layer: the norm's output in
8 bits, a dense product with its epilogue, and the cross-entropy of the head's logits,
with their gradients.  Plain numpy; nothing of the CUDA path is used.
"""
from __future__ import annotations

import numpy as np
from scipy.special import erf

E4M3_MAX, TINY = 448.0, 2.0 ** -126


def q8_scale(h):
    """A token's scale: its largest magnitude over e4m3's."""
    return np.maximum(np.abs(h).max(1) / E4M3_MAX, TINY)


def e4m3_half_step(v):
    """Half the distance of e4m3's values around v (|v| <= 448)."""
    exp = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return 2.0 ** (exp - 4)


def activation(name, z):
    """(act(z), act'(z))."""
    if name == "relu":
        return np.maximum(z, 0.0), (z > 0) * 1.0
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        cdf = 0.5 * (1.0 + erf(z / np.sqrt(2.0)))
        return z * cdf, cdf + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    return z, np.ones_like(z)


def linear(x, w, act="none", bias=None, residual=None):
    """(y, z): act(x w^T + bias) + residual and what act is taken of."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    y = activation(act, z)[0]
    return (y if residual is None else y + residual), z


def linear_grads(dy, x, w, act, z):
    """(dx, dw, dbias, dz) of linear, z being what act was taken of."""
    dz = dy * activation(act, z)[1]
    return dz @ w, dz.T @ x, dz.sum(0), dz


def head_loss(h, w, labels, weight=None):
    """(loss [T], dh, dw, dz): weighted cross-entropy of h w^T, and the gradients of its sum; rows
    without a label in [0, V) or of weight 0 take no part."""
    T, V = h.shape[0], w.shape[0]
    weight = np.ones(T) if weight is None else np.asarray(weight, np.float64)
    loss, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        if not 0 <= labels[t] < V or weight[t] == 0:
            continue
        z = w @ h[t]
        top = z.max()
        e = np.exp(z - top)
        loss[t] = weight[t] * (top + np.log(e.sum()) - z[labels[t]])
        dz[t] = weight[t] * e / e.sum()
        dz[t, labels[t]] -= weight[t]
    used = np.where((dz != 0).any(1)[:, None], h, 0.0)
    return loss, dz @ w, dz.T @ used, dz
