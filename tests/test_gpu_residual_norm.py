"""lx_residual_norm and its backward against the float64 definition (oracle/block.py):
widths held by a warp, a CTA and a cluster, odd widths and row distances, every gate,
absent parts, in-place and side-stream calls, refusals."""
import numpy as np
import pytest
import torch

from block_checks import close, f64, gen
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(T, H, dtype, gate, post=True, pre=True, y=True, pad=0, seed=0):
    g = gen(seed)
    dt = DT[dtype]

    def rows(std=1.0, pad=0):
        wide = (torch.randn(T, H + pad, generator=g) * std).to(dt).cuda()
        return wide[:, :H]

    v = dict(r=rows(1.5, pad), y=rows(0.4, pad) if y else None,
             w_post=(torch.randn(H, generator=g) * 0.3 + 1).cuda() if post and y else None,
             w_pre=(torch.randn(H, generator=g) * 0.3 + 1).cuda() if pre else None)
    v["gate"] = {"none": None, "channel": torch.randn(H, generator=g).cuda(),
                 "token": torch.rand(T, 1, generator=g).cuda(), "full": rows(0.7, pad)}[gate if y else "none"]
    return v, rows(0.1, pad), rows(0.1, pad) if pre else None


def _check(v, dr, dh, dtype, a=0.75, off=0.5, eps=1e-6, stream=None):
    bf = dtype == "bf16"
    T, H = v["r"].shape
    kw = {k: v[k] for k in ("w_post", "gate", "w_pre")}
    stats = torch.empty(2, T, device="cuda")
    out, h = lx.residual_norm(v["r"], v["y"], res_scale=a, weight_offset=off, eps=eps, stats=stats, **kw)
    g = lx.residual_norm_backward(dr, dh, v["r"], v["y"], stats, res_scale=a, weight_offset=off, **kw)
    torch.cuda.synchronize()
    n = {k: f64(t) for k, t in v.items()}
    w_out, w_h, _ = block.residual_norm(a=a, off=off, eps=eps, **n)
    close(out, w_out, bf, what="r_out")
    if h is not None:
        close(h, w_h, bf, what="h")
    want = block.residual_norm_grads(f64(dr), f64(dh), a=a, off=off, eps=eps, **n)
    for name in ("dr", "dy", "dw_post", "dgate", "dw_pre"):
        got = getattr(g, name)
        assert (got is None) == (name not in want), name
        if got is not None:
            close(got, want[name], got.dtype == torch.bfloat16, want["|" + name + "|"], name)
    return out, h, g


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(1, 2048), (37, 64), (300, 2048), (5, 1), (700, 7), (33, 257), (19, 2047)])
def test_against_the_definition(T, H, dtype, gate):
    _check(*_inputs(T, H, dtype, gate, seed=T + H), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,pad", [(3, 8192, 0), (2, 8200, 0), (5, 16384, 8), (2, 20001, 0), (1, 65536, 0),
                                     (40, 8193, 3)])
def test_wide_rows(T, H, pad, dtype):
    _check(*_inputs(T, H, dtype, "channel", pad=pad, seed=H), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [1, 3, 8, 2048])
def test_slices_of_wider_rows(pad, dtype):
    _check(*_inputs(50, 512, dtype, "full", pad=pad, seed=pad), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [1, 3])
def test_rows_from_an_odd_address(off, dtype):
    """Contiguous rows whose first element is not on a 16-byte boundary."""
    T, H = 20, 256
    v, dr, dh = _inputs(T, H, dtype, "none", seed=off)
    flat = torch.zeros(T * H + 8, dtype=DT[dtype], device="cuda")
    flat[off:off + T * H] = v["y"].reshape(-1)
    v["y"] = flat[off:off + T * H].view(T, H)
    _check(v, dr, dh, dtype)


@pytest.mark.parametrize("post,pre,y", [(False, True, True), (True, False, True), (False, False, True),
                                        (False, True, False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [96, 1000, 9000])
def test_absent_parts(H, dtype, post, pre, y):
    v, dr, dh = _inputs(23, H, dtype, "token" if y else "none", post, pre, y, seed=H)
    _check(v, dr, dh, dtype)


@pytest.mark.parametrize("dr,dh", [(True, False), (False, True)])
def test_one_gradient_alone(dr, dh):
    v, g1, g2 = _inputs(77, 640, "f32", "channel", seed=2)
    _check(v, g1 if dr else None, g2 if dh else None, "f32")


def test_many_tokens_of_one_width():
    """More rows than the resident grid holds: the parameter sums run over many rounds."""
    _check(*_inputs(5000, 320, "f32", "channel", seed=4), "f32")


def test_against_differences():
    """Directional derivatives of the kernel's own fp32 forward's definition: the change
    of the float64 loss along a direction against the gradient's product with it.  The
    gradient is within 1e-5 of its terms and the difference within 1e-8 of the loss, so
    1e-4 of the summed magnitudes holds both."""
    v, dr, dh = _inputs(6, 200, "f32", "channel", seed=8)
    stats = torch.empty(2, 6, device="cuda")
    kw = {k: v[k] for k in ("w_post", "gate", "w_pre")}
    lx.residual_norm(v["r"], v["y"], res_scale=0.5, stats=stats, **kw)
    g = lx.residual_norm_backward(dr, dh, v["r"], v["y"], stats, res_scale=0.5, **kw)
    n = {k: f64(t) for k, t in v.items()}
    rng = np.random.default_rng(0)

    def loss():
        out, h, _ = block.residual_norm(a=0.5, **n)
        return (out * f64(dr)).sum() + (h * f64(dh)).sum()

    for name in n:
        d, x, step = rng.normal(size=n[name].shape), n[name], 1e-5
        n[name] = x + step * d
        up = loss()
        n[name] = x - step * d
        slope = (up - loss()) / (2 * step)
        n[name] = x
        terms = f64(getattr(g, "d" + name)) * d
        assert abs(slope - terms.sum()) <= 1e-4 * np.abs(terms).sum(), name


def test_in_place_and_given_buffers():
    v, _, _ = _inputs(130, 2048, "bf16", "channel", seed=5)
    want = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], gate=v["gate"], w_pre=v["w_pre"])
    r, h = v["r"].clone(), torch.empty_like(v["r"])
    got = lx.residual_norm(r, v["y"], w_post=v["w_post"], gate=v["gate"], w_pre=v["w_pre"], r_out=r, h_out=h)
    assert got[0] is r and got[1] is h
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_repeats_give_the_same_bits():
    v, dr, dh = _inputs(900, 1024, "bf16", "channel", seed=6)
    one, two = (_check(v, dr, dh, "bf16") for _ in range(2))
    for a, b in zip(one[2], two[2]):
        assert torch.equal(a, b)


def test_side_stream():
    """Inputs of the current stream used on another: made there before, read there
    after a wait, and the results the same."""
    v, dr, dh = _inputs(64, 2048, "bf16", "channel", seed=9)
    want = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], w_pre=v["w_pre"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], w_pre=v["w_pre"], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_infinities_and_nan_stay_in_their_rows():
    v, _, _ = _inputs(8, 512, "f32", "none", seed=10)
    clean = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], w_pre=v["w_pre"])
    v["y"][2, 7], v["r"][5, 3] = float("nan"), float("inf")
    got = lx.residual_norm(v["r"], v["y"], w_post=v["w_post"], w_pre=v["w_pre"])
    for t in range(8):
        if t not in (2, 5):
            assert torch.equal(got[0][t], clean[0][t]) and torch.equal(got[1][t], clean[1][t])
    assert torch.isnan(got[1][2]).all()
    assert torch.isnan(got[1][5, 3]) and (got[1][5, :3] == 0).all()


def test_no_tokens():
    r = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    out, h = lx.residual_norm(r, r, w_post=w, w_pre=w)
    assert out.shape == (0, 64) and h.shape == (0, 64)
    g = lx.residual_norm_backward(out, h, r, r, torch.empty(2, 0, device="cuda"), w_post=w, w_pre=w)
    torch.cuda.synchronize()
    assert (g.dw_post == 0).all() and (g.dw_pre == 0).all()


def test_refusals():
    r = torch.zeros(4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    bad = [
        lambda: lx.residual_norm(r.cpu(), w_pre=w),
        lambda: lx.residual_norm(r.double(), w_pre=w),
        lambda: lx.residual_norm(r, r[:3], w_pre=w),
        lambda: lx.residual_norm(r, r.bfloat16(), w_pre=w),
        lambda: lx.residual_norm(r, w_pre=w[:63]),
        lambda: lx.residual_norm(r, w_pre=w.bfloat16()),
        lambda: lx.residual_norm(r.t(), w_pre=w[:4]),
        lambda: lx.residual_norm(r, r, gate=torch.zeros(4, 2, device="cuda"), w_pre=w),
        lambda: lx.residual_norm(r, r, w_pre=w, stats=torch.zeros(4, device="cuda")),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: lx.residual_norm(r), lambda: lx.residual_norm(r, gate=w, w_pre=w),
              lambda: lx.residual_norm(r, w_pre=w, eps=-1.0),
              lambda: lx.residual_norm(r, r, w_pre=w, h_out=r),
              lambda: lx.residual_norm_backward(None, None, r, r, torch.zeros(2, 4, device="cuda"), w_pre=w),
              lambda: lx.residual_norm_backward(r, r, r, None, torch.zeros(2, 4, device="cuda"), w_pre=w,
                                                workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(lx.LxError) as e:
            f()
        assert e.value.status == lx.LX_ERR_ARG
    with pytest.raises(lx.LxError) as e:
        lx.residual_norm(r[:1].expand(4, 64), w_pre=w)
    assert e.value.status == lx.LX_ERR_SHAPE
