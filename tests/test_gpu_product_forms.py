"""linear, its gradients and head_loss in the forms that the other tests pass by, against their definitions in float64
(bounds as in test_gpu_linear and test_gpu_head_loss): few tokens in several tiles; residual and pre together in
the large product, by TMA; gradients whose long sums are cut into ranges, one of them or both; the head's logits formed
twice, of several blocks of K, the last ragged."""
import numpy as np
import pytest
import torch

from block_checks import f64
from oracle import products as O
from paper_2608_07814_gb300 import lx
from test_gpu_linear import BF, E4M3, R, _case, _check_grads, _check_y, _gen, _mm_err

pytestmark = pytest.mark.gpu


def _check_pre(pre, X, W, bias):
    _, z = O.linear(X, W, "none", f64(bias))
    err = _mm_err(X.shape[1], np.abs(X) @ np.abs(W).T + np.abs(f64(bias))) + 2.0 ** -23 * np.abs(z)
    assert (np.abs(f64(pre) - z) <= err * (1 + R) + R * np.abs(z)).all()


def _all_parts(T, N, K, dtype, act):
    x, w, kw, X, W = _case(T, N, K, dtype)
    g = _gen(9)
    bias, res = torch.randn(N, generator=g).to(BF).cuda(), torch.randn(T, N, generator=g).to(BF).cuda()
    pre = torch.full((T, N), float("nan"), dtype=BF, device="cuda")
    y = lx.linear(x, w, bias=bias, act=act, residual=res, pre=pre, **kw)
    _check_y(y, X, W, act, bias, res)
    _check_pre(pre, X, W, bias)
    pre.fill_(float("nan"))
    y = lx.linear(x, w, bias=bias, act=act, pre=pre, **kw)
    _check_y(y, X, W, act, bias, None)
    _check_pre(pre, X, W, bias)
    _check_y(lx.linear(x, w, act=act, residual=res, **kw), X, W, act, None, res)
    inplace = res.clone()
    pre.fill_(float("nan"))
    _check_y(lx.linear(x, w, bias=bias, act=act, residual=inplace, y=inplace, pre=pre, **kw), X, W, act, bias, res)
    _check_pre(pre, X, W, bias)


@pytest.mark.parametrize("dtype", [BF, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K,act", [(257, 300, 8192, "gelu"), (600, 130, 16384, "silu"), (700, 264, 8192, "relu"),
                                       (513, 129, 8208, "none"), (1024, 1024, 8192, "silu")])
def test_few_tokens_in_several_tiles(T, N, K, act, dtype):
    _all_parts(T, N, K, dtype, act)


@pytest.mark.parametrize("dtype", [BF, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K,act", [(1000, 2048, 256, "gelu"), (3000, 520, 144, "silu"), (513, 4096, 160, "relu"),
                                       (5000, 136, 80, "none"), (2049, 1928, 512, "gelu"), (20000, 264, 64, "silu")])
def test_residual_and_pre_in_the_large_product(T, N, K, act, dtype):
    _all_parts(T, N, K, dtype, act)


@pytest.mark.parametrize("T,N,K,act", [(4500, 264, 136, "silu"), (130, 8200, 72, "gelu"), (4100, 4104, 264, "none"),
                                       (4100, 4104, 264, "relu"), (5000, 100, 2056, "gelu"), (33, 12001, 520, "silu"),
                                       (9001, 33, 40, "gelu")])
def test_gradients_of_long_sums(T, N, K, act):
    _check_grads(T, N, K, act)
    _check_grads(T, N, K, act, lddy_pad=3, dbias=False, seed=2)


@pytest.mark.parametrize("T,V,H,masked", [(2100, 33003, 1096, 0.0), (2100, 33003, 1096, 0.3), (4300, 16100, 2120, 0.1),
                                          (2049, 66000, 200, 0.0)])
def test_logits_formed_twice(T, V, H, masked):
    """Losses of all rows, dh of a sample of rows and dw of a sample of columns."""
    g = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    h, w = randn(T, H).to(BF), (randn(V, H) * (2.5 / H ** 0.5)).to(BF)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(T, generator=g, device="cuda") < masked] = -100
    weight = torch.rand(T, generator=g, device="cuda") + 0.5
    got = lx.head_loss(h, w, labels, row_weight=weight)
    live = labels >= 0
    W, wt = w.double(), weight.double() * live
    mm = lambda n: (n / 16 + 16) * 2.0 ** -23  # noqa: E731
    cols = torch.arange(0, V, V // 61, device="cuda")
    cols[-1] = V - 1
    dw, err_w = torch.zeros(len(cols), H, dtype=torch.float64, device="cuda"), 0.0
    for t0 in range(0, T, 300):
        r = slice(t0, min(T, t0 + 300))
        X, wr = h[r].double(), wt[r]
        z = X @ W.t()
        e = mm(H) * (X.abs() @ W.abs().t()).amax(1)
        at = labels[r].clamp(min=0).long()[:, None]
        lse = torch.logsumexp(z, 1)
        loss = wr * (lse - z.gather(1, at)[:, 0])
        parts = z.abs().amax(1) + np.log(V)
        assert bool(((got.loss[r].double() - loss).abs() <= wr * (2 * e + 2.0 ** -20 * parts)).all())
        dz = torch.softmax(z, 1).scatter_add_(1, at, -torch.ones_like(at, dtype=torch.float64)) * wr[:, None]
        p = dz.abs().scatter_add_(1, at, 2 * wr[:, None])   # p - 1: what it is formed of
        term = p * (2 * e + 2.0 ** -19)[:, None] + R * dz.abs() * (1 + 1e-3)
        s = slice(0, None, 17)
        want = dz[s] @ W
        err = term[s] @ W.abs() + mm(V) * (dz[s].abs() @ W.abs())
        assert bool(((got.dh[r][s].double() - want).abs() <= err * 1.01 + R * want.abs() + 1e-37).all())
        d, X = dz[:, cols], X * live[r][:, None]
        dw += d.t() @ X
        err_w = err_w + term[:, cols].t() @ X.abs() + (R * (1 + R) + mm(T)) * (d.abs().t() @ X.abs())
    assert bool(((got.dw[cols].double() - dw).abs() <= err_w * 1.01 + R * dw.abs() + 1e-37).all())
    assert not got.loss[~live].any() and not got.dh[~live].any()
