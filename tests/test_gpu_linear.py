"""linear and linear_backward against their definitions in float64.

Bounds.  A product's sum of K terms is made 16 at a time (32 in 8 bits) by the tensor core, which
cuts the running sum off: at most 2^-23 of the terms' magnitudes a step, and a few roundings for
the terms of a step and the CTAs' parts: (K / 16 + 16) 2^-23 of the sum of magnitudes.  Activations
rise by at most 1.13, and are themselves right to 2^-20 of their value and argument.  y is rounded to bf16
once: 2^-8.  In the backward z (pre) is rounded to bf16, which moves act' by at most 0.8 of that
(the largest second derivative, gelu's), and dz to bf16: 2^-8 of each term."""
import numpy as np
import pytest
import torch

from block_checks import f64
from oracle import products as O
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn
R = 2.0 ** -8


def _mm_err(K, mag):
    return (K / 16 + 16) * 2.0 ** -23 * mag


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _case(T, N, K, dtype, seed=0, pad=0, padw=0):
    g = _gen(seed)
    x, w = torch.randn(T, K + pad, generator=g), torch.randn(N, K + padw, generator=g) / K ** 0.5
    if dtype == BF:
        x, w = x.to(BF).cuda()[:, :K], w.to(BF).cuda()[:, :K]
        return x, w, {}, f64(x), f64(w)
    xs, ws = (0.01 + torch.rand(T, generator=g)).cuda(), (0.01 + torch.rand(N, generator=g)).cuda()
    x, w = (x * 3).to(E4M3).cuda()[:, :K], (w * 30).to(E4M3).cuda()[:, :K]
    return x, w, dict(x_scale=xs, w_scale=ws), f64(x.float()) * f64(xs)[:, None], f64(w.float()) * f64(ws)[:, None]


def _check_y(y, X, W, act, bias, residual):
    want, z = O.linear(X, W, act, f64(bias), f64(residual))
    mag = np.abs(X) @ np.abs(W).T + (0 if bias is None else np.abs(f64(bias)))
    err = 1.13 * _mm_err(X.shape[1], mag) + 2.0 ** -20 * np.abs(z) + (0 if residual is None else 2.0 ** -23 * np.abs(f64(residual)))
    over = np.abs(f64(y) - want) - err * (1 + R) - R * np.abs(want)
    assert (over <= 0).all(), (over.max(), np.abs(want).max())


SIZES = [(1, 16, 16), (1, 1, 64), (1, 2048, 2048), (3, 100, 1040), (16, 8192, 128), (17, 129, 4096), (64, 2048, 8192),
         (65, 300, 272), (128, 1000, 512), (129, 257, 2064), (256, 512, 2048), (257, 2049, 144), (300, 40, 48),
         (1000, 2000, 256), (1031, 4100, 400), (2500, 4096, 128)]


@pytest.mark.parametrize("dtype", [BF, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", SIZES)
def test_sizes(T, N, K, dtype):
    x, w, kw, X, W = _case(T, N, K, dtype)
    g = _gen(9)
    bias, res = torch.randn(N, generator=g).to(BF).cuda(), torch.randn(T, N, generator=g).to(BF).cuda()
    _check_y(lx.linear(x, w, **kw), X, W, "none", None, None)
    act = ("relu", "silu", "gelu")[(T + N) % 3]
    _check_y(lx.linear(x, w, bias=bias, act=act, residual=res, **kw), X, W, act, bias, res)


@pytest.mark.parametrize("T,N", [(5, 200), (700, 3000)])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_activations_over_their_range(T, N, act):
    """z from -12 to 12, through one input of 1."""
    x = torch.zeros(T, 16, dtype=BF, device="cuda")
    x[:, 0] = 1
    w = torch.zeros(N, 16, dtype=BF, device="cuda")
    w[:, 0] = torch.linspace(-12, 12, N).to(BF).cuda()
    pre = torch.empty(T, N, dtype=BF, device="cuda")
    y = lx.linear(x, w, act=act, pre=pre)
    assert torch.equal(pre, w[:, 0].expand(T, N))
    _check_y(y, f64(x), f64(w), act, None, None)


@pytest.mark.parametrize("T,N", [(3, 77), (33, 264), (600, 2050), (513, 4096)])
def test_strides_in_place_and_what_lies_beside(T, N):
    K = 160
    x, w, _, X, W = _case(T, N, K, BF, pad=24, padw=8)
    g = _gen(5)
    wide = torch.randn(T + 2, N + 5, generator=g).to(BF).cuda()
    before = wide.clone()
    y = wide[1:-1, 3:3 + N]
    res = y.clone()
    out = lx.linear(x, w, residual=y, act="silu", y=y)
    assert out is y
    _check_y(y, X, W, "silu", None, res)
    wide[1:-1, 3:3 + N] = before[1:-1, 3:3 + N]
    assert torch.equal(wide, before)
    # the same bits, wherever the rows lie
    assert torch.equal(lx.linear(x, w, residual=res, act="silu"), lx.linear(x.contiguous(), w.contiguous(), residual=before[1:-1, 3:3 + N], act="silu"))


@pytest.mark.parametrize("T,N,ld", [(600, 2011, 2016), (1000, 1999, 2056), (5000, 130, 136), (513, 4095, 4096),
                                    (2000, 3001, 3008), (9000, 515, 520), (2500, 2052, 2056)])
def test_rows_on_16_byte_boundaries_that_end_elsewhere(T, N, ld):
    """Columns behind the last and rows below it are left as they were; the residual's are not read."""
    x, w, _, X, W = _case(T, N, 72, BF)
    out = torch.full((T + 40, ld), 7.0, dtype=BF, device="cuda")
    res = torch.full((T, ld), float("nan"), dtype=BF, device="cuda")
    res[:, :N] = torch.randn(T, N, generator=_gen(2)).to(BF).cuda()
    pre = torch.empty(T, N, dtype=BF, device="cuda")
    y = lx.linear(x, w, act="silu", residual=res[:, :N], y=out[:T, :N])
    _check_y(y, X, W, "silu", None, res[:, :N].contiguous())
    assert (out[:, N:] == 7).all() and (out[T:] == 7).all()
    assert torch.equal(lx.linear(x, w, act="silu", residual=res[:, :N], pre=pre), y)


def test_what_is_no_number_stays_in_its_row():
    for T, N in ((9, 100), (600, 4000)):
        x, w, _, X, W = _case(T, N, 64, BF)
        x[4, 7] = float("nan")
        for act in ("none", "relu", "silu", "gelu"):
            y = lx.linear(x, w, act=act)
            assert torch.isnan(y[4]).all()
            y[4] = 0
            assert torch.isfinite(y).all()


def _check_grads(T, N, K, act, lddy_pad=0, dbias=True, seed=0):
    x, w, _, X, W = _case(T, N, K, BF, seed=seed)
    g = _gen(seed + 100)
    bias = torch.randn(N, generator=g).to(BF).cuda()
    dy = (torch.randn(T, N + lddy_pad, generator=g) * 0.1).to(BF).cuda()[:, :N]
    pre = torch.empty(T, N, dtype=BF, device="cuda") if act != "none" else None
    lx.linear(x, w, bias=bias, act=act, pre=pre)
    got = lx.linear_backward(dy, x, w, act=act, pre=pre, want_dbias=dbias)
    _, z = O.linear(X, W, act, f64(bias))
    D = f64(dy)
    dx, dw, db, dz = O.linear_grads(D, X, W, act, z)
    if pre is not None:
        err = _mm_err(K, np.abs(X) @ np.abs(W).T + np.abs(f64(bias)))
        assert (np.abs(f64(pre) - z) <= err * (1 + R) + R * np.abs(z)).all()
        if act == "relu":   # a sum that is 0 but for its error may have either sign
            sure = np.abs(z) > err
            dz = np.where(sure, dz, D * (f64(pre) > 0))
            dx, dw, db = dz @ W, dz.T @ X, dz.sum(0)
        moved = np.abs(D) * 0.8 * (R * np.abs(z) + err * (1 + R)) if act != "relu" else 0 * np.abs(D)
    else:
        moved = 0 * np.abs(D)
    moved = moved + 2.0 ** -20 * np.abs(D) * (1 + (np.abs(z) if act != "none" else 0))
    A = np.abs(dz)
    term = moved * (1 + R) + R * A
    for name, g_, want, err in (("dx", got.dx, dx, term @ np.abs(W) + _mm_err(N, (A + term) @ np.abs(W))),
                                ("dw", got.dw, dw, term.T @ np.abs(X) + _mm_err(T, (A + term).T @ np.abs(X))),
                                ("dbias", got.dbias, db, (moved + 1e-5 * A).sum(0))):
        if name == "dbias" and not dbias:
            assert g_ is None
            continue
        over = np.abs(f64(g_) - want) - err * (1 + R) - R * np.abs(want)
        assert (over <= 0).all(), (name, over.max(), np.abs(want).max())


@pytest.mark.parametrize("T,N,K,act,pad", [
    (1, 8, 8, "none", 0), (1, 1, 16, "silu", 0), (2, 100, 264, "gelu", 0), (64, 64, 64, "none", 0), (65, 130, 72, "relu", 3),
    (257, 1003, 1032, "silu", 0), (300, 256, 512, "none", 8), (300, 256, 512, "none", 4), (511, 777, 80, "gelu", 0),
    (1100, 520, 2048, "silu", 0), (2048, 2050, 136, "relu", 0)])
def test_gradients(T, N, K, act, pad):
    _check_grads(T, N, K, act, lddy_pad=pad)
    _check_grads(T, N, K, act, lddy_pad=pad, dbias=False, seed=3)


def test_gradients_against_differences():
    """dx, dw and dbias along random directions against differences of the float64 loss."""
    T, N, K, act = 70, 90, 64, "gelu"
    x, w, _, X, W = _case(T, N, K, BF)
    g = _gen(4)
    bias, dy = torch.randn(N, generator=g).to(BF).cuda(), torch.randn(T, N, generator=g).to(BF).cuda()
    pre = torch.empty(T, N, dtype=BF, device="cuda")
    lx.linear(x, w, bias=bias, act=act, pre=pre)
    got = lx.linear_backward(dy, x, w, act=act, pre=pre, want_dbias=True)
    rng = np.random.default_rng(0)
    f = lambda a, b, c: (O.linear(a, b, act, c)[0] * f64(dy)).sum()  # noqa: E731
    Bi = f64(bias)
    for i, (grad, v) in enumerate(((got.dx, X), (got.dw, W), (got.dbias, Bi))):
        u, e = rng.standard_normal(v.shape), 1e-5
        args = [X, W, Bi]
        hi, lo = list(args), list(args)
        hi[i], lo[i] = v + e * u, v - e * u
        want = (f(*hi) - f(*lo)) / (2 * e)
        # independent roundings of 2^-8 each: their sum along u is within 6 of its spread
        spread = 2 * R * np.sqrt(((f64(grad) * u) ** 2).sum()) + 2 * R * np.sqrt((f64(grad) ** 2).mean() * (u ** 2).sum())
        assert abs((f64(grad) * u).sum() - want) < 6 * spread


def test_parts_of_the_gradients_and_no_tokens():
    x, w, _, _, _ = _case(100, 72, 64, BF)
    dy = torch.randn(100, 72, generator=_gen(1)).to(BF).cuda()
    full = lx.linear_backward(dy, x, w, want_dbias=True)
    for kw in (dict(want_dx=False), dict(want_dw=False), dict(want_dx=False, want_dw=False, want_dbias=True)):
        part = lx.linear_backward(dy, x, w, **kw)
        for a, b in zip(part, full):
            assert a is None or torch.equal(a, b)
        assert (part.dx is None) == (not kw.get("want_dx", True)) and (part.dw is None) == (not kw.get("want_dw", True))
    e = torch.empty(0, 64, dtype=BF, device="cuda")
    assert lx.linear(e, w).shape == (0, 72)
    none = lx.linear_backward(torch.empty(0, 72, dtype=BF, device="cuda"), e, w, want_dbias=True)
    assert none.dx.shape == (0, 64) and not none.dw.any() and not none.dbias.any()


def test_the_same_bits_again():
    for T, N, K in ((64, 2048, 8192), (257, 1003, 1032), (1500, 4096, 1024)):
        x, w, _, _, _ = _case(T, N, K, BF)
        dy = torch.randn(T, N, generator=_gen(1)).to(BF).cuda()
        a, ga = lx.linear(x, w), lx.linear_backward(dy, x, w, want_dbias=True)
        for _ in range(3):
            assert torch.equal(lx.linear(x, w), a)
            assert all(torch.equal(p, q) for p, q in zip(lx.linear_backward(dy, x, w, want_dbias=True), ga))


@pytest.mark.parametrize("T,N", [(8, 512), (600, 4096)])
def test_a_wait_that_runs_out_gives_nan(T, N):
    x, w, _, _, _ = _case(T, N, 256, BF)
    dy = torch.randn(T, N, generator=_gen(1)).to(BF).cuda()
    want, grads = lx.linear(x, w), lx.linear_backward(dy, x, w)
    lx.inject_unmet_wait_call(lx.LX_WAIT_CALL_PRODUCT, 2_000_000)
    bad = lx.linear(x, w, act="relu", residual=dy)
    torch.cuda.synchronize()
    assert torch.isnan(bad).all()
    lx.inject_unmet_wait_call(lx.LX_WAIT_CALL_PRODUCT, 2_000_000)
    bad = lx.linear_backward(dy, x, w)
    torch.cuda.synchronize()
    assert torch.isnan(bad.dx).all() and torch.isnan(bad.dw).all()
    assert torch.equal(lx.linear(x, w), want)
    assert all(torch.equal(a, b) for a, b in zip(lx.linear_backward(dy, x, w)[:2], grads[:2]))
