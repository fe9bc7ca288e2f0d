"""The float64 definitions of the products around a layer, pinned against torch's autograd in
float64 and closed forms (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import products as O


def _rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_linear_and_its_gradients(act):
    g = _rng(1)
    x, w, b, r, dy = (g.standard_normal(s) for s in ((7, 5), (6, 5), (6,), (7, 6), (7, 6)))
    tx, tw, tb, tr = (torch.tensor(v, requires_grad=True) for v in (x, w, b, r))
    f = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act]
    ty = f(tx @ tw.T + tb) + tr
    ty.backward(torch.tensor(dy))
    y, z = O.linear(x, w, act, b, r)
    dx, dw, db, _ = O.linear_grads(dy, x, w, act, z)
    for got, want in ((y, ty), (dx, tx.grad), (dw, tw.grad), (db, tb.grad), (dy, tr.grad)):
        np.testing.assert_allclose(got, want.detach().numpy(), rtol=1e-12, atol=1e-13)


def test_head_loss_and_its_gradients():
    g = _rng(2)
    h, w = g.standard_normal((6, 4)), g.standard_normal((9, 4))
    labels, weight = np.array([3, -100, 0, 8, 9, 2]), np.array([0.5, 1.0, 2.0, 1.0, 1.0, 0.0])
    th, tw = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    use = [0, 2, 3]
    tl = torch.nn.functional.cross_entropy((th @ tw.T)[use], torch.tensor(labels[use]), reduction="none")
    tl = tl * torch.tensor(weight[use])
    tl.sum().backward()
    loss, dh, dw, dz = O.head_loss(h, w, labels, weight)
    np.testing.assert_allclose(loss[use], tl.detach().numpy(), rtol=1e-12)
    assert (loss[[1, 4, 5]] == 0).all() and (dh[[1, 4, 5]] == 0).all()
    np.testing.assert_allclose(dh, th.grad.numpy(), atol=1e-13)
    np.testing.assert_allclose(dw, tw.grad.numpy(), atol=1e-13)
    np.testing.assert_allclose(dz.sum(1), 0, atol=1e-13)


def test_a_row_that_takes_no_part_may_hold_anything():
    h, w = np.ones((2, 3)), np.eye(3)
    h[1] = np.nan
    loss, dh, dw, _ = O.head_loss(h, w, np.array([1, -1]))
    assert np.isfinite(loss).all() and np.isfinite(dh).all() and np.isfinite(dw).all()
    np.testing.assert_allclose(loss[0], np.log(3))


def test_e4m3_steps():
    """Every e4m3 value's neighbours are two half steps away (within its binade)."""
    v = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (v[1:] + v[:-1]) / 2
    np.testing.assert_allclose(O.e4m3_half_step(mid), (v[1:] - v[:-1]) / 2)
    np.testing.assert_allclose(O.q8_scale(np.array([[1.0, -896.0], [0.0, 0.0]])), [2.0, O.TINY])
