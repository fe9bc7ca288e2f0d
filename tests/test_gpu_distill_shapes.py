"""lx_distill_loss at the sizes where its shape changes: rows that just fit one, two, four
or eight CTAs' shared memory and rows that do not, few and many rows, negative and zero
weights.  Bounds as in test_gpu_distill.py; the oracle skips rows of weight 0, so most
rows of the large cases have it."""
import numpy as np
import pytest
import torch

from block_checks import close, f64, gen
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu


def _case(T, V, K, dtype, tau=1.0, labels=True, on=3, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(T, V, generator=g, device="cuda").mul_(2.5).to(dtype)
    ids = torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32)
    top = torch.randn(T, K, generator=g, device="cuda")
    w = torch.zeros(T, device="cuda")
    rows = torch.unique(torch.cat([torch.tensor([0, T - 1], device="cuda"),
                                   torch.randint(0, T, (on,), generator=g, device="cuda")]))
    w[rows] = torch.rand(len(rows), generator=g, device="cuda") + 0.5
    lab = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32) if labels else None
    return z, ids, top, lab, w, rows


def _check(z, ids, top, lab, w, rows, tau=1.0, a=0.7, b=0.3):
    b = b if lab is not None else 0.0
    loss, d = lx.distill_loss(z, ids, top, temperature=tau, kd_weight=a, labels=lab, ce_weight=b, row_weight=w)
    pick = lambda t: f64(t[rows])  # noqa: E731
    wl, wd, mag = block.distill(pick(z), ids[rows].cpu().numpy(), pick(top), tau, None, a,
                                None if lab is None else lab[rows].cpu().numpy(), b, pick(w), True)
    close(loss[rows], wl, False, (float(z.float().abs().max()) + 10) * max(1.0, tau) * float(w.abs().max()), "loss")
    close(d[rows], wd, z.dtype == torch.bfloat16,
          mag + 1e-3 * np.abs(pick(w))[:, None] * (abs(a) * tau + b), "dlogits")
    off = w == 0
    assert (loss[off] == 0).all() and (d[off] == 0).all()


# 64 entries leave 18 pieces of 512 threads, 8192 bytes each, to a CTA's part of a row, and
# 9 or so of 256 and 128 threads; on both sides of one, two, four and eight CTAs
@pytest.mark.parametrize("V", [9000, 20000, 20480, 36000, 40961, 73728, 73729, 147456, 147464, 294912, 294920,
                               589824, 589832])
def test_rows_at_the_edge_of_what_is_held(V):
    _check(*_case(160, V, 64, torch.bfloat16, seed=V))


@pytest.mark.parametrize("V", [36863, 36864, 147455, 147457, 294912, 294913, 300001])
def test_fp32_rows_at_the_edge(V):
    _check(*_case(155, V, 64, torch.float32, seed=V), tau=2.0)


@pytest.mark.parametrize("K", [1, 31, 33, 64, 127, 200, 513, 1024])
@pytest.mark.parametrize("V", [1500, 70001])
def test_entries(K, V):
    _check(*_case(170, V, K, torch.bfloat16, seed=K), tau=0.7)


@pytest.mark.parametrize("T", [1, 2, 18, 19, 20, 38, 76, 77, 152, 153, 305, 1000])
def test_rows_spread_over_ctas(T):
    _check(*_case(T, 33000, 16, torch.bfloat16, seed=T), tau=2.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("a,b", [(0.0, 0.3), (0.7, 0.0), (0.0, 0.0), (-0.5, 0.3), (0.7, -0.2)])
def test_zero_and_negative_factors(a, b, dtype):
    for tau in (1.0, 2.0):
        z, ids, top, lab, w, rows = _case(40, 5000, 16, dtype, seed=3)
        w[rows[0]] *= -1
        loss, d = lx.distill_loss(z, ids, top, temperature=tau, kd_weight=a, labels=lab, ce_weight=b, row_weight=w)
        pick = lambda t: f64(t[rows])  # noqa: E731
        wl, wd, mag = block.distill(pick(z), ids[rows].cpu().numpy(), pick(top), tau, None, a, lab[rows].cpu().numpy(), b,
                                    pick(w), True)
        close(loss[rows], wl, False, 60.0, "loss")
        close(d[rows], wd, dtype == torch.bfloat16, mag + 2e-3, "dlogits")


def test_logits_far_apart_and_large():
    """Values that rise by hundreds along a row (the reference is raised many times), and a
    row of large ones."""
    z, ids, top, lab, w, rows = _case(30, 9000, 8, torch.float32, on=30, seed=9)
    z[0] = torch.linspace(-300, 300, 9000, device="cuda")
    z[29] = z[29] + 3000.0
    r = torch.tensor([0, 29], device="cuda")
    w[r] = 1.0
    loss, d = lx.distill_loss(z, ids, top, labels=lab, kd_weight=0.5, ce_weight=0.5, row_weight=w)
    wl, wd, mag = block.distill(f64(z[r]), ids[r].cpu().numpy(), f64(top[r]), 1.0, None, 0.5, lab[r].cpu().numpy(), 0.5,
                                f64(w[r]), True)
    # the exponent of a value of size x is rounded to 2^-24 x: 1e-6 of x in the exponent
    close(loss[r], wl, False, np.array([60.0, 400.0]), "loss")
    close(d[r], wd, False, mag * np.array([[40.0], [40.0]]) + 1e-3, "dlogits")


@pytest.mark.parametrize("V", [4099, 100003])
def test_in_place_over_many_rows(V):
    z, ids, top, lab, w, rows = _case(700 if V < 10000 else 200, V, 20, torch.bfloat16, on=40, seed=V)
    want, dw = lx.distill_loss(z, ids, top, temperature=2.0, labels=lab, kd_weight=0.6, ce_weight=0.4, row_weight=w)
    loss, d = lx.distill_loss(z, ids, top, temperature=2.0, labels=lab, kd_weight=0.6, ce_weight=0.4, row_weight=w,
                              dlogits=z)
    assert d is z and torch.equal(loss, want) and torch.equal(d, dw)
