"""residual_norm_q8 against its definition in float64.

q is within half a step of e4m3 of h / scale, which the kernel forms by some tens of fp32
roundings on terms as large as the row's largest (1e-5 of 448, as in block_checks); the scale is
one of h's values over 448, the same 1e-5 off.  Everything else is residual_norm's, bit for bit."""
import numpy as np
import pytest
import torch

from block_checks import F32, close, f64
from oracle import block as B
from oracle import products as O
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def _inputs(T, H, dtype, gate, seed=0, pad=0, y=True):
    g = torch.Generator().manual_seed(seed)
    rows = lambda std: (torch.randn(T, H + pad, generator=g) * std).to(dtype).cuda()[:, :H]  # noqa: E731
    ch = lambda: (1 + 0.2 * torch.randn(H, generator=g)).cuda()  # noqa: E731
    kw = dict(w_pre=ch())
    if y:
        kw["w_post"] = ch()
        if gate == "channel":
            kw["gate"] = ch()
        elif gate == "token":
            kw["gate"] = torch.rand(T, 1, generator=g).cuda()
        elif gate == "full":
            kw["gate"] = rows(0.7)
    return rows(1.5), (rows(0.3) if y else None), kw


def _check(r, y, kw, a=0.75, off=0.0):
    h_out = torch.empty(r.shape, dtype=r.dtype, device="cuda")
    out = lx.residual_norm_q8(r, y, res_scale=a, weight_offset=off, h_out=h_out, **kw)
    r_want, h_want = lx.residual_norm(r, y, res_scale=a, weight_offset=off, **kw)
    assert torch.equal(out.r_out, r_want) and torch.equal(h_out, h_want)
    _, h, _ = B.residual_norm(f64(r), f64(y), f64(kw.get("w_post")), f64(kw.get("gate")), f64(kw["w_pre"]), a=a, off=off)
    scale = O.q8_scale(h)
    assert out.q.dtype == E4M3 and out.q.shape == r.shape and out.scale.shape == (r.shape[0],)
    np.testing.assert_allclose(f64(out.scale), scale, rtol=F32)
    v = h / f64(out.scale)[:, None]
    q = f64(out.q.float())
    over = np.abs(q - np.clip(v, -448, 448)) - O.e4m3_half_step(v) - F32 * 448
    assert (over <= 0).all(), over.max()
    # nothing but the row's largest reaches the end of e4m3
    assert (np.abs(q).max(1) == 448).all()


@pytest.mark.parametrize("T,H,dtype,gate,pad", [
    (1, 2048, torch.bfloat16, "channel", 0), (1, 1, torch.float32, "none", 0), (3, 17, torch.bfloat16, "full", 1),
    (37, 100, torch.float32, "token", 4), (200, 512, torch.bfloat16, "token", 8), (65, 513, torch.bfloat16, "none", 0),
    (130, 2047, torch.float32, "token", 1), (64, 2560, torch.bfloat16, "full", 2560), (9, 4104, torch.bfloat16, "channel", 0),
    (5, 9001, torch.float32, "full", 3), (2, 40000, torch.bfloat16, "channel", 0), (2, 65536, torch.float32, "none", 0)])
def test_against_the_definition(T, H, dtype, gate, pad):
    _check(*_inputs(T, H, dtype, gate, pad=pad))
    if T > 30:
        _check(*_inputs(T, H, dtype, "none", seed=1, pad=pad), a=1.0, off=1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_without_a_block_before(dtype):
    r, _, kw = _inputs(20, 256, dtype, "none", y=False)
    out = lx.residual_norm_q8(r, **kw)
    assert out.r_out is r
    _check(r, None, kw)


@pytest.mark.parametrize("H", [256, 2048, 2047, 10000, 40000])
def test_rows_of_zeros_and_of_what_is_no_number(H):
    r, _, kw = _inputs(4, H, torch.float32, "none", y=False)
    r[0] = 0
    r[1, H // 2] = float("nan")
    r[2, 3] = float("inf")
    out = lx.residual_norm_q8(r, **kw)
    q, s = out.q.float(), out.scale
    assert (q[0] == 0).all() and float(s[0]) == 2.0 ** -126
    assert torch.isnan(q[1]).all() and torch.isnan(s[1])
    assert torch.isnan(q[2, 3]) and not torch.isfinite(s[2])     # inf / inf
    assert torch.isfinite(q[3]).all() and torch.isfinite(s[3])


def test_values_far_below_one():
    """Rows whose norm's eps keeps h small: the scale goes with them."""
    r, _, kw = _inputs(6, 512, torch.float32, "none", y=False)
    _check(r * 1e-20, None, kw, a=1.0)


def test_unaligned_outputs_in_place_and_stats():
    r, y, kw = _inputs(33, 264, torch.bfloat16, "channel")
    want = lx.residual_norm_q8(r, y, **kw)
    buf = torch.full((33 * 264 + 8,), 7, dtype=torch.uint8, device="cuda")
    q = buf[3:3 + 33 * 264].view(33, 264).view(E4M3)
    scale, stats, stats2 = torch.empty(33, device="cuda"), torch.empty(2, 33, device="cuda"), torch.empty(2, 33, device="cuda")
    lx.residual_norm(r, y, stats=stats2, **kw)
    r2 = r.clone()
    out = lx.residual_norm_q8(r2, y, r_out=r2, q_out=q, scale_out=scale, stats=stats, **kw)
    assert out.r_out is r2 and out.scale is scale
    # (rows are summed in another order where they are written by single elements)
    _, h, _ = B.residual_norm(f64(r), f64(y), f64(kw["w_post"]), f64(kw["gate"]), f64(kw["w_pre"]))
    close(r2, f64(want.r_out), True)
    close(stats, f64(stats2), False)
    np.testing.assert_allclose(f64(scale), O.q8_scale(h), rtol=F32)
    v = h / f64(scale)[:, None]
    assert (np.abs(f64(q.float()) - np.clip(v, -448, 448)) <= O.e4m3_half_step(v) + F32 * 448).all()
    assert (buf[:3] == 7).all() and (buf[3 + 33 * 264:] == 7).all()


def test_no_tokens():
    r, y, kw = _inputs(0, 64, torch.bfloat16, "none")
    out = lx.residual_norm_q8(r, y, **kw)
    assert out.q.shape == (0, 64) and out.scale.shape == (0,)
