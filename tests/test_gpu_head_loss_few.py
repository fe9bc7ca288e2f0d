"""head_loss of up to 16 tokens: the gradients are rounded once.

Bounds as in test_gpu_head_loss, but for what is rounded on the way: row_weight dz is held as a value in bf16 and the
rest in bf16, 2^-16 of it off (2^-8 of what 2^-8 leaves) and 2^-24 for the product; the sum over the tokens has
64 terms."""
import numpy as np
import pytest
import torch

from block_checks import f64
from oracle import products as O
from paper_2608_07814_gb300 import lx
from test_gpu_head_loss import R, _case

pytestmark = pytest.mark.gpu


def _check(got, h, w, labels, weight=None):
    X, W = f64(h), f64(w)
    lab = labels.cpu().numpy()
    T, V, H = X.shape[0], W.shape[0], X.shape[1]
    wt = np.ones(T) if weight is None else f64(weight)
    loss, dh, dw, dz = O.head_loss(X, W, lab, wt)
    used = np.where(((lab >= 0) & (lab < V) & (wt != 0))[:, None], X, 0.0)
    mm = lambda n: (n / 16 + 16) * 2.0 ** -23  # noqa: E731
    e = mm(H) * (np.abs(used) @ np.abs(W).T).max(1)
    parts = np.abs(used @ W.T).max(1) + np.log(V)
    assert (np.abs(f64(got.loss) - loss) <= np.abs(wt) * (2 * e + 2.0 ** -20 * parts)).all()
    p = np.abs(dz)
    p[np.arange(T), np.clip(lab, 0, V - 1)] += 2 * np.abs(wt) * (used != 0).any(1)  # p - 1: what it is formed of
    term = p * (2 * e + 2.0 ** -19)[:, None] + 2.0 ** -15.9 * np.abs(dz)
    err = term @ np.abs(W) + 2 * mm(V) * (np.abs(dz) @ np.abs(W))
    assert (np.abs(f64(got.dh) - dh) <= err * 1.01 + R * np.abs(dh) + 1e-37).all()
    err = term.T @ np.abs(used) + mm(64) * (np.abs(dz).T @ np.abs(used))
    assert (np.abs(f64(got.dw) - dw) <= err * 1.01 + R * np.abs(dw) + 1e-37).all()


@pytest.mark.parametrize("T,V,H,masked", [(1, 1, 8, 0), (1, 1000, 64, 0), (1, 40003, 264, 0), (2, 257, 72, 0), (8, 5000, 2056, 0.3),
                                          (11, 3001, 520, 0.2), (15, 600, 136, 0.5), (16, 20011, 96, 0), (16, 256, 2048, 0.1)])
def test_gradients_are_rounded_once(T, V, H, masked):
    h, w, labels, weight = _case(T, V, H, masked)
    labels[0] = V // 2
    _check(lx.head_loss(h, w, labels, row_weight=weight), h, w, labels, weight)
    _check(lx.head_loss(h, w, labels), h, w, labels)
    _check(lx.head_loss(h, w, labels, row_weight=weight * -1e-6), h, w, labels, weight * -1e-6)


@pytest.mark.parametrize("T", [1, 7, 16])
def test_rows_that_take_no_part(T):
    """None at all, or some that hold what is no number, in a workspace of NaNs: nothing of it reaches the others."""
    h, w, labels, weight = _case(T, 900, 264)
    n = lx.head_loss_workspace_bytes(T, 900, 264)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    got = lx.head_loss(h, w, torch.full_like(labels, -1), row_weight=weight, workspace=ws)
    assert not got.loss.any() and not got.dh.any() and not got.dw.any()
    labels[T // 2] = 900
    h[T // 2] = float("nan")
    ws.fill_(255)
    got = lx.head_loss(h, w, labels, row_weight=weight, workspace=ws)
    h[T // 2] = 0
    _check(got, h, w, labels, weight)
    for a, b in ((True, False), (False, True), (False, False)):
        ws.fill_(255)
        part = lx.head_loss(h, w, labels, row_weight=weight, want_dh=a, want_dw=b, workspace=ws)
        assert all(p is None or torch.equal(p, q) for p, q in zip(part, got))


def test_what_is_no_number_stays_in_its_row():
    h, w, labels, _ = _case(12, 300, 64)
    h[7, 3] = float("nan")
    got = lx.head_loss(h, w, labels)
    assert torch.isnan(got.loss[7]) and torch.isnan(got.dh[7]).all()
    ok = torch.arange(12, device="cuda") != 7
    assert torch.isfinite(got.loss[ok]).all() and torch.isfinite(got.dh[ok]).all()
