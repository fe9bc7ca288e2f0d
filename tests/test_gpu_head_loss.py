"""head_loss against its definition in float64.

Bounds.  A logit of H terms is off by (H / 16 + 16) 2^-23 of its terms' magnitudes (the tensor
core's sums, see test_gpu_linear), e at most over the rows; a loss by 2 e and 2^-20 of its parts;
a softmax by 2 e + 2^-19 of itself; dz is rounded to bf16 (2^-8 of each term of the gradients'
sums), and so are, for dw, the hidden states times the weights (as much again), dh and dw."""
import math

import numpy as np
import pytest
import torch

from block_checks import f64
from oracle import products as O
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
R = 2.0 ** -8


def _case(T, V, H, masked=0.0, seed=0, pad=0, std=2.5):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn(T, H + pad, generator=g).to(BF).cuda()[:, :H]
    w = (torch.randn(V, H + pad, generator=g) * (std / H ** 0.5)).to(BF).cuda()[:, :H]
    labels = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    labels[torch.rand(T, generator=g) < masked] = -100
    return h, w, labels.cuda(), (torch.rand(T, generator=g) + 0.5).cuda()


def _check(got, h, w, labels, weight=None):
    X, W = f64(h), f64(w)
    lab = labels.cpu().numpy()
    T, V, H = X.shape[0], W.shape[0], X.shape[1]
    wt = np.ones(T) if weight is None else f64(weight)
    loss, dh, dw, dz = O.head_loss(X, W, lab, wt)
    used = np.where(((lab >= 0) & (lab < V) & (wt != 0))[:, None], X, 0.0)
    mm = lambda n: (n / 16 + 16) * 2.0 ** -23  # noqa: E731
    z = used @ W.T
    e = mm(H) * (np.abs(used) @ np.abs(W).T).max(1)
    parts = np.abs(z).max(1) + np.log(V)
    assert (np.abs(f64(got.loss) - loss) <= np.abs(wt) * (2 * e + 2.0 ** -20 * parts)).all()
    p = np.abs(dz)
    p[np.arange(T), np.clip(lab, 0, V - 1)] += 2 * np.abs(wt) * (used != 0).any(1)  # p - 1: what it is formed of
    term = p * (2 * e + 2.0 ** -19)[:, None] + R * np.abs(dz) * (1 + 1e-3)
    if got.dh is not None:
        err = term @ np.abs(W) + mm(V) * (np.abs(dz) @ np.abs(W))
        assert (np.abs(f64(got.dh) - dh) <= err * 1.01 + R * np.abs(dh) + 1e-37).all()
    if got.dw is not None:
        weighted = 0 if weight is None else R * (1 + R) * (np.abs(dz).T @ np.abs(used))
        err = term.T @ np.abs(used) + weighted + mm(T) * (np.abs(dz).T @ np.abs(used))
        assert (np.abs(f64(got.dw) - dw) <= err * 1.01 + R * np.abs(dw) + 1e-37).all()


@pytest.mark.parametrize("T,V,H,masked", [
    (1, 1, 8, 0), (1, 7, 8, 0), (1, 1000, 64, 0), (2, 256, 64, 0), (3, 257, 72, 0.5), (64, 1152, 200, 0.3), (65, 129, 136, 0),
    (255, 4003, 256, 0.1), (256, 640, 264, 0), (257, 5003, 512, 0.6), (300, 300, 2048, 0.9), (700, 2000, 96, 0.5)])
def test_against_the_definition(T, V, H, masked):
    h, w, labels, weight = _case(T, V, H, masked)
    _check(lx.head_loss(h, w, labels, row_weight=weight), h, w, labels, weight)
    _check(lx.head_loss(h, w, labels), h, w, labels)


def test_wide_vocabulary_in_several_pieces():
    """Rows enough that a piece of the vocabulary (256 MiB of dz) is 16384 columns: three pieces, the last ragged; a
    sample of rows and of columns against the definition."""
    T, V, H = 8192, 40003, 64
    h, w, labels, weight = _case(T, V, H, 0.2, std=1.0)
    got = lx.head_loss(h, w, labels, row_weight=weight)
    z = h.double() @ w.double().t()
    live = ((labels >= 0) & (labels < V)).double()
    dz = torch.softmax(z, 1)
    lse = torch.logsumexp(z, 1)
    at = labels.clamp(min=0).long()[:, None]
    loss = weight * live * (lse - z.gather(1, at)[:, 0])
    dz.scatter_add_(1, at, -torch.ones_like(dz[:, :1])).mul_((weight * live)[:, None])
    dh, dw = dz @ w.double(), dz.t() @ h.double()
    assert float((got.loss - loss).abs().max()) < 1e-4
    # norms: roundings of 2^-8 of each term and of the result, each by itself
    for a, b in ((got.dh, dh), (got.dw, dw)):
        assert float((a.double() - b).norm() / b.norm()) < R
    dead = live == 0
    assert not got.loss[dead].any() and not got.dh[dead].any()


@pytest.mark.parametrize("T,V,H", [(2048, 300, 64), (2049, 300, 64), (9000, 130, 72), (70001, 33, 16)])
def test_many_rows(T, V, H):
    h, w, labels, weight = _case(T, V, H, 0.3, seed=4)
    labels[T // 3: T // 3 + 2100] = -100  # a whole run of rows takes no part
    _check(lx.head_loss(h, w, labels, row_weight=weight), h, w, labels, weight)


@pytest.mark.parametrize("T,V,H", [(40, 700, 2056), (300, 600, 4104)])
def test_long_sums(T, V, H):
    h, w, labels, weight = _case(T, V, H, 0.1, seed=6)
    _check(lx.head_loss(h, w, labels, row_weight=weight), h, w, labels, weight)


@pytest.mark.parametrize("T", [5, 300])
def test_rows_that_take_no_part_are_not_used(T):
    h, w, labels, weight = _case(T, 500, 128, 0.4, seed=2)
    labels[0], labels[1], labels[2] = 500, -1, 2 ** 31 - 1
    weight[3] = 0
    dead = (labels < 0) | (labels >= 500) | (weight == 0)
    want = lx.head_loss(h, w, labels, row_weight=weight)
    _check(want, h, w, labels, weight)
    h2 = h.clone()
    h2[dead] = float("nan")
    weight[labels < 0] = float("nan")
    got = lx.head_loss(h2, w, labels, row_weight=weight)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not got.loss[dead].any() and not got.dh[dead].any()


def test_no_row_takes_part_and_no_rows():
    h, w, labels, _ = _case(70, 300, 64)
    labels.fill_(-100)
    got = lx.head_loss(h, w, labels)
    assert not got.loss.any() and not got.dh.any() and not got.dw.any()
    got = lx.head_loss(h[:0], w, labels[:0])
    assert got.loss.shape == (0,) and got.dh.shape == (0, 64) and not got.dw.any()


def test_what_is_no_number_stays_in_its_row():
    h, w, labels, _ = _case(40, 300, 64)
    h[7, 3] = float("nan")
    got = lx.head_loss(h, w, labels)
    assert torch.isnan(got.loss[7]) and torch.isnan(got.dh[7]).all()
    ok = torch.arange(40, device="cuda") != 7
    assert torch.isfinite(got.loss[ok]).all() and torch.isfinite(got.dh[ok]).all()


def test_logits_far_from_zero():
    """A shared part of 1000 in every logit, and one logit far above the others."""
    h, w, labels, weight = _case(33, 600, 64, std=1.0)
    h[:, 0], w[:, 0] = 32, 32
    _check(lx.head_loss(h, w, labels), h, w, labels)
    h, w, labels, weight = _case(33, 600, 64, std=1.0)
    w[77] *= 100
    _check(lx.head_loss(h, w, labels), h, w, labels)


@pytest.mark.parametrize("T,V", [(40, 600), (300, 9000), (2100, 40000)])
def test_sure_rows(T, V):
    """Labels far above the rest: the loss, log(1 + sum of the others), is below 0.1 and never below 0, and the
    label's dz is 1 - exp(-loss), seen in dh along a direction that only the label's row of w has.
    Relative: the others' logits of 64 terms are off by less than 1e-4, 2e-3 covers it (and 2^-8 twice for dz and
    dh in bf16).  Absolute: the sum is at least the label's 1 and below 2, so each addition after it rounds by at most
    2^-24: 64 of them in the chain of its half tile, and with V <= 40000 at most 16 and 32 more where the
    half tiles' sums are joined: 120 2^-24 < 2^-17."""
    g = torch.Generator().manual_seed(1)
    h = torch.zeros(T, 64)
    h[:, :32] = torch.randn(T, 32, generator=g)
    h[:, 32] = 1
    w = torch.randn(V, 64, generator=g) * 0.1
    w[:, 32:] = 0
    w[7, :32] = 0
    w[7, 32] = 5 + math.log(V)
    scale = torch.linspace(1, 2, T)
    h[:, 32] = scale
    w[7, 40] = 1   # h is 0 there: dh's entry 40 is the label's dz
    h, w = h.to(BF).cuda(), w.to(BF).cuda()
    labels = torch.full((T,), 7, dtype=torch.int32, device="cuda")
    got = lx.head_loss(h, w, labels)
    z = h.double() @ w.double().t()
    rest = torch.logsumexp(torch.cat([z[:, :7], z[:, 8:]], 1), 1) - z[:, 7]
    want = torch.log1p(torch.exp(rest))
    assert float(want.max()) < 0.1 and float(got.loss.min()) >= 0
    assert float(((got.loss - want).abs() - 2e-3 * want).max()) <= 2.0 ** -17
    p = -torch.expm1(-want)
    assert float(((got.dh[:, 40].double() + p).abs() - (2e-3 + 2 * R) * p).max()) <= 2.0 ** -17


def test_slices_of_wider_arrays_parts_and_the_same_bits():
    h, w, labels, weight = _case(130, 900, 264, 0.1, pad=16)
    full = lx.head_loss(h, w, labels, row_weight=weight)
    _check(full, h, w, labels, weight)
    for a, b in ((True, True), (True, False), (False, True), (False, False)):
        got = lx.head_loss(h.contiguous(), w.contiguous(), labels, row_weight=weight, want_dh=a, want_dw=b)
        assert (got.dh is not None) == a and (got.dw is not None) == b
        assert all(p is None or torch.equal(p, q) for p, q in zip(got, full))


def test_gradient_against_differences():
    h, w, labels, weight = _case(50, 200, 64)
    got = lx.head_loss(h, w, labels, row_weight=weight)
    lab, rng = labels.cpu().numpy(), np.random.default_rng(0)
    f = lambda a, b: O.head_loss(a, b, lab, f64(weight))[0].sum()  # noqa: E731
    X, W = f64(h), f64(w)
    for i, (grad, v) in enumerate(((got.dh, X), (got.dw, W))):
        u, e = rng.standard_normal(v.shape), 1e-5
        hi, lo = (v + e * u, W) if i == 0 else (X, v + e * u), (v - e * u, W) if i == 0 else (X, v - e * u)
        want = (f(*hi) - f(*lo)) / (2 * e)
        # independent roundings of 2^-8 each: their sum along u is within 6 of its spread
        spread = 2 * R * np.sqrt(((f64(grad) * u) ** 2).sum()) + 2 * R * np.sqrt((f64(grad) ** 2).mean() * (u ** 2).sum())
        assert abs((f64(grad) * u).sum() - want) < 6 * spread


def test_a_wait_that_runs_out_gives_nan():
    h, w, labels, _ = _case(300, 1000, 128, 0.2)
    want = lx.head_loss(h, w, labels)
    live = labels >= 0
    lx.inject_unmet_wait_call(lx.LX_WAIT_CALL_PRODUCT, 2_000_000)
    bad = lx.head_loss(h, w, labels)
    torch.cuda.synchronize()
    assert torch.isnan(bad.loss[live]).all() and torch.isnan(bad.dh[live]).all() and torch.isnan(bad.dw).all()
    assert all(torch.equal(a, b) for a, b in zip(lx.head_loss(h, w, labels), want))
