"""Products and the 8-bit norm on arrays of more than 2^31 elements: rows on both sides of that, and the last,
against the definition (bounds as in test_gpu_linear, test_gpu_head_loss and test_gpu_norm_q8)."""
import numpy as np
import pytest
import torch

from block_checks import F32, f64
from oracle import block as B
from oracle import products as O
from paper_2608_07814_gb300 import lx
from test_gpu_linear import BF, R, _check_y, _mm_err

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


@pytest.mark.parametrize("N", [32768, 32769])
def test_linear_and_its_gradients(N):
    """(N off a multiple of 8: rows that TMA does not take)"""
    T, K = 70000, 64
    randn = _gen(1)
    x, w = randn(T, K).to(BF), (randn(N, K) / 8).to(BF)
    res = torch.empty(T, N, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    pre = torch.empty(T, N, dtype=BF, device="cuda")
    y = lx.linear(x, w, act="silu", residual=res, pre=pre)
    rows = [0, 65532, 65533, 65535, 65536, 65537, T - 2, T - 1]
    X, W = f64(x[rows]), f64(w)
    _check_y(y[rows], X, W, "silu", None, res[rows])
    _, z = O.linear(X, W, "silu")
    err = _mm_err(K, np.abs(X) @ np.abs(W).T)
    assert (np.abs(f64(pre[rows]) - z) <= err * (1 + R) + R * np.abs(z)).all()
    d = lx.linear_backward(res, x, w, act="silu", pre=pre)
    D = f64(res[rows])
    want, _, _, dz = O.linear_grads(D, X, W, "silu", f64(pre[rows]))  # (of pre as it is stored)
    moved = 2.0 ** -20 * np.abs(D) * (1 + np.abs(z))
    term = moved * (1 + R) + R * np.abs(dz)
    err = term @ np.abs(W) + _mm_err(N, (np.abs(dz) + term) @ np.abs(W))
    assert (np.abs(f64(d.dx[rows]) - want) <= err * (1 + R) + R * np.abs(want)).all()
    cols = [0, 1, N // 2, N - 1]
    zc, Dc, Xc = pre[:, cols].double(), res[:, cols].double(), x.double()
    s = torch.sigmoid(zc)
    dz = Dc * s * (1 + zc * (1 - s))
    term = 2.0 ** -20 * Dc.abs() * (1 + zc.abs()) * (1 + R) + R * dz.abs()
    want = dz.t() @ Xc
    err = term.t() @ Xc.abs() + _mm_err(T, (dz.abs() + term).t() @ Xc.abs())
    assert bool(((d.dw[cols].double() - want).abs() <= err * (1 + R) + R * want.abs()).all())


def test_weights_of_a_few_tokens_product():
    T, N, K = 2, 600000, 4096
    x = _gen(3)(T, K).to(BF)
    w = torch.empty(N, K, dtype=BF, device="cuda").normal_(0, K ** -0.5, generator=torch.Generator(device="cuda").manual_seed(4))
    y = lx.linear(x, w)
    cols = list(range(0, N, 9973)) + [524287, 524288, N - 1]
    _check_y(y[:, cols], f64(x), f64(w[cols]), "none", None, None)


@pytest.mark.parametrize("V,H", [(600000, 4096), (2200000, 1024)])
def test_head_loss(V, H):
    """(the wider vocabulary's logits are not kept: its dz is worked on in five pieces)"""
    T = 3
    h = _gen(5)(T, H).to(BF)
    w = torch.empty(V, H, dtype=BF, device="cuda").normal_(0, 2 * H ** -0.5, generator=torch.Generator(device="cuda").manual_seed(6))
    labels = torch.tensor([V - 1, 524287, V - V // 20], dtype=torch.int32, device="cuda")
    got = lx.head_loss(h, w, labels)
    X = h.double()
    z = torch.cat([X @ p.double().t() for p in w.split(50000)], 1)
    e = (H / 16 + 16) * 2.0 ** -23 * max(float((X.abs() @ p.double().abs().t()).max()) for p in w.split(50000))
    at = labels.long()[:, None]
    loss = torch.logsumexp(z, 1) - z.gather(1, at)[:, 0]
    parts = float(z.abs().max()) + np.log(V)
    assert float((got.loss.double() - loss).abs().max()) <= 2 * e + 2.0 ** -20 * parts
    dz = torch.softmax(z, 1).scatter_add_(1, at, -torch.ones_like(loss)[:, None])
    p = dz.abs().scatter_add_(1, at, 2 * torch.ones_like(loss)[:, None])
    term = p * (2 * e + 2.0 ** -19) + R * dz.abs() * (1 + 1e-3)
    want, err = 0, 0
    mm = (V / 16 + 16) * 2.0 ** -23
    for v in range(0, V, 50000):
        s = slice(v, v + 50000)
        want = want + dz[:, s] @ w[s].double()
        err = err + (term[:, s] + mm * dz[:, s].abs()) @ w[s].double().abs()
    assert bool(((got.dh.double() - want).abs() <= err * 1.01 + R * want.abs()).all())
    rows = list(range(0, V, 9973)) + [524286, 524287, 524288, V - V // 20, V - 2, V - 1]
    want = dz[:, rows].t() @ X
    err = (term[:, rows] + 17 * 2.0 ** -23 * dz[:, rows].abs()).t() @ X.abs()
    assert bool(((got.dw[rows].double() - want).abs() <= err * 1.01 + R * want.abs() + 1e-37).all())


@pytest.mark.parametrize("T,H", [(600000, 4096), (1100000, 2047)])
def test_norm_q8(T, H):
    r = torch.empty(T, H, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(7))
    w_pre = 1 + 0.2 * _gen(8)(H)
    out = lx.residual_norm_q8(r, w_pre=w_pre)
    rows = [0, 2 ** 31 // H - 1, 2 ** 31 // H, 2 ** 31 // H + 1, T - 2, T - 1]
    _, h, _ = B.residual_norm(f64(r[rows]), None, None, None, f64(w_pre), a=1.0, off=0.0)
    scale = f64(out.scale[rows])
    np.testing.assert_allclose(scale, O.q8_scale(h), rtol=F32)
    v = h / scale[:, None]
    q = f64(out.q.view(torch.uint8)[rows].view(torch.float8_e4m3fn).float())
    assert (np.abs(q - np.clip(v, -448, 448)) <= O.e4m3_half_step(v) + F32 * 448).all()
