"""Bounds shared by the GPU tests of the operators around a layer (not a test file).

fp32 arithmetic: a value formed by some tens of roundings of 2^-24 each, on terms as
large as the tensor's largest value, is within 1e-5 of that largest value; a sum over
tokens adds at most 150 values one after the other on each level, so it is within
1e-5 of the sum of its terms' magnitudes.  Rounding to bf16 adds 2^-8 of the value.
"""
import numpy as np
import torch

F32 = 1e-5


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def close(got, want, bf16, scale=None, what=""):
    """|got - want| within the bounds above; scale: magnitudes the fp32 part goes by
    (the tensor's largest value unless given)."""
    g, w = f64(got), np.asarray(want, np.float64)
    assert g.shape == w.shape, (what, g.shape, w.shape)
    assert np.array_equal(np.isfinite(g), np.isfinite(w)), what
    if not np.isfinite(w).all():
        assert np.array_equal(g[~np.isfinite(w)], w[~np.isfinite(w)], equal_nan=True), what
        g, w = np.where(np.isfinite(w), g, 0), np.where(np.isfinite(w), w, 0)
    if w.size == 0:
        return
    s = np.abs(w).max() if scale is None else scale
    bound = F32 * s + (2.0 ** -8 * np.abs(w) if bf16 else 0) + 1e-30
    over = np.abs(g - w) - bound
    assert (over <= 0).all(), f"{what}: {np.abs(g - w).max():.3g} off, {over.max():.3g} over the bound"


def gen(seed):
    return torch.Generator().manual_seed(seed)
