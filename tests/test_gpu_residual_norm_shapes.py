"""lx_residual_norm where its shape changes: rows held by parts of warps, by CTAs and by
clusters, on and off 16-byte boundaries, in place, first and last rows of a buffer that
has nothing around them.  Bounds as in test_gpu_residual_norm.py."""
import pytest
import torch

import test_gpu_residual_norm as base
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [2, 15, 16, 17, 63, 65, 127, 128, 129, 255, 256, 511, 512, 513, 520, 1023, 1040, 4095,
                               4096, 4097, 4104])
def test_widths(H, dtype):
    base._check(*base._inputs(41, H, dtype, "full", seed=H), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,pad", [(32767, 0), (32768, 0), (32769, 0), (40001, 1), (65535, 0)])
def test_widest(H, pad, dtype):
    base._check(*base._inputs(2, H, dtype, "channel", pad=pad, seed=H), dtype)


@pytest.mark.parametrize("T", [1, 2, 3, 151, 152, 153, 609, 2500])
@pytest.mark.parametrize("H", [24, 768, 769])
def test_rows(T, H):
    base._check(*base._inputs(T, H, "bf16", "channel", seed=T + H), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [7, 130, 2047, 9001])
def test_in_place_off_the_grid(H, dtype):
    v, _, _ = base._inputs(333, H, dtype, "token", seed=H)
    kw = {k: v[k] for k in ("w_post", "gate", "w_pre")}
    want = lx.residual_norm(v["r"], v["y"], **kw)
    r = v["r"].clone()
    got = lx.residual_norm(r, v["y"], r_out=r, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", range(8))
def test_garbage_around_a_slice_is_not_used(off, dtype):
    """Every element around the slice is NaN."""
    T, H = 9, 70
    v, dr, dh = base._inputs(T, H, dtype, "full", seed=off)

    def wrap(t):
        wide = torch.full((T + 2, H + 19), float("nan"), dtype=t.dtype, device="cuda")
        s = wide[1:T + 1, off:off + H]
        s.copy_(t)
        return s

    v = {k: wrap(t) if k in ("r", "y", "gate") else t for k, t in v.items()}
    base._check(v, wrap(dr), wrap(dh), dtype)


def test_large_offsets():
    """Rows past 2^31 elements, close together and far apart."""
    H, ld, T = 64, 1 << 20, 2060
    buf = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    y = buf.view(T, ld)[:, :H]
    v, _, _ = base._inputs(T, H, "bf16", "none", seed=1)
    y.copy_(v["y"])
    want = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], w_pre=v["w_pre"])
    got = lx.residual_norm(v["r"], y, w_post=v["w_post"], w_pre=v["w_pre"])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_too_far_apart_is_refused():
    d = lx.ResnormDesc(lx.LX_BF16, 2, 64, 0, 1 << 30, 0, 0, 4096, None, None, None, 4096, 1.0, 0.0, 1e-6)
    assert lx.lib().lx_residual_norm(d, None, 1 << 23, None, None) == lx.LX_ERR_SHAPE
