"""residual_norm_q8 of rows so small that 448 over the largest of them is beyond fp32's range.

With eps = 1e-6 a row far below it is multiplied by 1000: h is a normal number down to rows of 1e-38, and below
that the scale stays at 2^-126.  Bounds as in test_gpu_norm_q8: the scale 1e-5 off, q half a step of e4m3 and
1e-5 of 448.  What fp32 cannot hold below 2^-126 it rounds by at most 2^-150, and (r' w) is at least 5e-40
where a row's largest is, so that adds 2^-150 / 5e-40 = 1.4e-6 of the largest, which 1e-5 covers."""
import numpy as np
import pytest
import torch

from block_checks import F32, f64
from oracle import block as B
from oracle import products as O
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu


def _check(r, y, kw, a):
    out = lx.residual_norm_q8(r, y, res_scale=a, **kw)
    r_want, _ = lx.residual_norm(r, y, res_scale=a, **kw)
    assert torch.equal(out.r_out, r_want)
    _, h, _ = B.residual_norm(f64(r), f64(y), f64(kw.get("w_post")), f64(kw.get("gate")), f64(kw["w_pre"]), a=a, off=0.0)
    np.testing.assert_allclose(f64(out.scale), O.q8_scale(h), rtol=F32)
    v = h / f64(out.scale)[:, None]
    q = f64(out.q.float())
    assert np.isfinite(q).all()
    assert (np.abs(q - np.clip(v, -448, 448)) <= O.e4m3_half_step(v) + F32 * 448).all()
    assert (q[h == 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [48, 512, 2047, 40000])
@pytest.mark.parametrize("size", [1e-30, 1e-33, 1e-35, 3e-37, 1e-38, 1e-39])
def test_rows_far_below_eps(size, H, dtype):
    g = torch.Generator().manual_seed(7)
    r = torch.randn(5, H, generator=g, dtype=torch.float64) * size
    r[:, ::3] = 0
    r[3] = 0
    kw = dict(w_pre=(1 + 0.2 * torch.randn(H, generator=g)).cuda())
    _check(r.to(dtype).cuda(), None, kw, 1.0)
    # the same rows through the residual, with a block's output of nothing
    kw["w_post"] = (1 + 0.2 * torch.randn(H, generator=g)).cuda()
    _check(r.to(dtype).cuda(), torch.zeros(5, H, dtype=dtype, device="cuda"), kw, 0.5)


@pytest.mark.parametrize("size", [1e-35, 1e-37, 1e-38])
def test_weights_far_below_one(size):
    """h small by its weights instead: r' is of the usual size or far above it."""
    g = torch.Generator().manual_seed(8)
    for rows in (1.0, 1e-4):
        r = (torch.randn(4, 256, generator=g) * rows).cuda()
        r[:, 5] = 0
        _check(r, None, dict(w_pre=(torch.randn(256, generator=g, dtype=torch.float64) * size).float().cuda()), 1.0)
