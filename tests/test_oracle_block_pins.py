"""Pins of oracle/block.py: gradients against central differences of the float64
losses, closed forms, and planted mistakes that must fail a pin (CPU)."""
import numpy as np
import pytest

from oracle import block


def _rng(seed):
    return np.random.default_rng(seed)


def _difference(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        g[i] = (up - f()) / (2 * step)
        x[i] = keep
    return g


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True)])
def test_norm_gradients_are_the_differences(gate, post, pre):
    g = _rng(3)
    T, H = 3, 5
    v = dict(r=g.normal(size=(T, H)), y=g.normal(size=(T, H)))
    if post:
        v["w_post"] = g.normal(size=H)
    if pre:
        v["w_pre"] = g.normal(size=H)
    if gate != "none":
        v["gate"] = g.normal(size={"channel": (H,), "token": (T, 1), "full": (T, H)}[gate])
    dr, dh = g.normal(size=(T, H)), g.normal(size=(T, H)) if pre else None

    def loss():
        out, h, _ = block.residual_norm(a=0.7, off=0.5, eps=1e-3, **v)
        return float((out * dr).sum() + (0 if h is None else (h * dh).sum()))

    got = block.residual_norm_grads(dr, dh, a=0.7, off=0.5, eps=1e-3, **v)
    for name in v:
        want = _difference(loss, v[name])
        assert np.allclose(got["d" + name], want, rtol=1e-6, atol=1e-7), name


def test_norm_closed_forms():
    r = np.array([[3.0, 4.0]])
    _, h, _ = block.residual_norm(r, w_pre=np.ones(2), eps=0.0)
    assert np.allclose(h, r / np.sqrt(12.5))
    out, h, _ = block.residual_norm(r, y=2 * r, w_post=np.zeros(2), w_pre=np.ones(2), off=1.0, eps=0.0, a=0.0)
    assert np.allclose(2 * out, h)            # a normalised row is its own norm (and h has weight 1 + 1)
    out, _, _ = block.residual_norm(r, y=r, gate=np.array([[0.5]]))
    assert np.allclose(out, 1.5 * r)


def test_balance_gradient_is_the_difference():
    g = _rng(5)
    l, ids = g.normal(size=(4, 5)), g.integers(-1, 6, size=(4, 3))
    mask = np.array([1, 0, 1, 1])
    l[3, 2] = -np.inf
    f = lambda: block.router_balance(l, ids, mask, 0.3, 0.2)[0][0]  # noqa: E731
    got = block.router_balance_grad(l, ids, mask, 0.3, 0.2)
    fin = np.isfinite(l)
    want = _difference(f, l)[fin]
    assert np.allclose(got[fin], want, rtol=1e-6, atol=1e-8)
    assert np.all(got[1] == 0) and got[3, 2] == 0


def test_balance_closed_forms():
    E, T = 8, 16
    ids = (np.arange(T)[:, None] * 2 + np.arange(2)) % E          # every expert equally often
    loss, counts, prob, lse = block.router_balance(np.zeros((T, E)), ids, None, 1.0, 1.0)
    assert np.allclose(loss, [1 + np.log(E) ** 2, 1, np.log(E) ** 2]) and np.allclose(prob, 1 / E)
    assert list(counts) == [4] * E + [T]
    one = np.zeros((T, E))
    one[:, 3] = 200.0                                             # all weight and choice on one expert
    assert np.allclose(block.router_balance(one, np.full((T, 1), 3))[0][1], E)
    assert np.allclose(block.router_balance(one, np.full((T, 2), 3))[1][3], T)   # repeats count once
    assert np.all(block.router_balance(one, ids, np.zeros(T))[0] == 0)


@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("lse", [False, True])
def test_distill_gradient_is_the_difference(tau, lse):
    g = _rng(7)
    T, V, K = 5, 9, 4
    z, top = g.normal(size=(T, V)), g.normal(size=(T, K))
    ids = np.stack([g.permutation(V)[:K] for _ in range(T)])
    ids[1, 2] = -1
    ids[2, 0] = ids[2, 1]
    labels, w = np.array([0, 8, -100, 3, 2]), np.array([1, 0.5, 1, 0, 2.0])
    L = np.log(np.exp(top / tau).sum(1)) + 0.5 if lse else None
    f = lambda: block.distill(z, ids, top, tau, L, 0.6, labels, 0.4, w)[0].sum()  # noqa: E731
    _, got = block.distill(z, ids, top, tau, L, 0.6, labels, 0.4, w)
    assert np.allclose(got, _difference(f, z), rtol=1e-6, atol=1e-8)
    assert np.all(got[3] == 0)


def test_distill_closed_forms():
    g = _rng(9)
    z = g.normal(size=(3, 6))
    ids = np.tile(np.arange(6), (3, 1))
    loss, grad = block.distill(z, ids, z + 5.0, tau=3.0)           # the teacher is the student
    assert np.allclose(loss, 0) and np.allclose(grad, 0)
    loss, grad = block.distill(z, ids[:, 2:3], z[:, :1])           # one entry: the cross-entropy
    assert np.allclose(loss, -(z[:, 2] - np.log(np.exp(z).sum(1))))
    assert np.allclose(loss, block.distill(z, ids[:, :1], z[:, :1], a=0.0, labels=np.full(3, 2), b=1.0)[0])
    none, gnone = block.distill(z, np.full((3, 2), -1), z[:, :2])
    assert np.all(none == 0) and np.all(gnone == 0)


@pytest.mark.parametrize("mistake", ["no mean", "gate dropped", "eps outside"])
def test_planted_norm_mistakes_show(mistake):
    g = _rng(11)
    r, y, w = g.normal(size=(2, 4)), g.normal(size=(2, 4)), g.normal(size=4)
    gate = g.normal(size=4)
    out, h, _ = block.residual_norm(r, y, w, gate, w, 0.5, 0.0, 0.1)
    rms = lambda v: v / np.sqrt((v * v).mean(1, keepdims=True) + 0.1)  # noqa: E731
    want = 0.5 * r + gate * rms(y) * w
    assert np.allclose(out, want) and np.allclose(h, rms(want) * w)
    bad = {"no mean": lambda v: v / np.sqrt((v * v).sum(1, keepdims=True) + 0.1),
           "eps outside": lambda v: v / (np.sqrt((v * v).mean(1, keepdims=True)) + 0.1),
           "gate dropped": rms}[mistake]
    wrong = 0.5 * r + (1 if mistake == "gate dropped" else gate) * bad(y) * w
    assert not np.allclose(out, wrong, rtol=1e-3)
