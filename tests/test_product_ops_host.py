"""Argument checks of the products around a layer (no GPU): a refused call returns its status
before any CUDA call, and the binding refuses tensors of other types, shapes and devices."""
import ctypes

import pytest
import torch

from paper_2608_07814_gb300 import lx
from test_block_devices_host import _on

X, W, Y, FAR = 1 << 20, 1 << 24, 1 << 26, 1 << 28  # addresses that no refused call reads
ARG, SHAPE, UNSUPPORTED, OK = lx.LX_ERR_ARG, lx.LX_ERR_SHAPE, lx.LX_ERR_UNSUPPORTED, lx.LX_OK


def _desc(**kw):
    d = dict(dtype=lx.LX_BF16, T=4, N=32, K=64, act=0, ldx=64, ldw=64, ldr=0, x=X, w=W, x_scale=None, w_scale=None,
             bias=None, residual=None)
    d.update(kw)
    return lx.LinearDesc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=lx.LX_F32), ARG), (dict(dtype=9), ARG), (dict(act=4), ARG), (dict(act=-1), ARG), (dict(T=-1), ARG),
    (dict(T=(1 << 30) + 1), SHAPE), (dict(N=0), SHAPE), (dict(N=(1 << 24) + 1), SHAPE), (dict(K=0), SHAPE),
    (dict(K=60), SHAPE), (dict(ldx=63), SHAPE), (dict(ldx=68), SHAPE), (dict(ldw=56), SHAPE), (dict(ldw=65), SHAPE),
    (dict(x=None), ARG), (dict(w=None), ARG), (dict(x=X + 8), ARG), (dict(w=W + 2), ARG),
    (dict(T=1 << 30, N=1 << 24), SHAPE), (dict(dtype=lx.LX_E4M3, K=72, ldx=80, ldw=80), SHAPE),
    (dict(dtype=lx.LX_E4M3, ldx=72), SHAPE)])
def test_linear_descriptors(kw, status):
    L, d = lx.lib(), _desc(**kw)
    assert L.lx_linear(d, Y, 32, None, None) == status
    assert L.lx_linear_backward(d, Y, 32, None, FAR, None, None, FAR * 2, 1 << 40, None) == status
    assert L.lx_last_error()


def test_linear_outputs():
    L = lx.lib()
    f = lambda d, y=Y, ldy=32, pre=None: L.lx_linear(d, y, ldy, pre, None)  # noqa: E731
    assert L.lx_linear(None, Y, 32, None, None) == ARG
    assert f(_desc(), y=None) == ARG and f(_desc(), y=Y + 1) == ARG and f(_desc(), ldy=31) == SHAPE
    assert f(_desc(), pre=Y) == ARG                      # each other
    assert f(_desc(), y=X + 64) == ARG and f(_desc(), y=W) == ARG and f(_desc(), pre=X) == ARG
    assert f(_desc(bias=Y)) == ARG and f(_desc(bias=FAR + 1)) == ARG
    assert f(_desc(residual=FAR, ldr=16)) == SHAPE
    assert f(_desc(residual=Y + 64, ldr=32)) == ARG      # shifted in place
    assert f(_desc(residual=Y, ldr=40)) == ARG           # in place, with other rows
    assert f(_desc(residual=FAR, ldr=32), pre=FAR) == ARG
    assert f(_desc(x_scale=FAR)) == ARG                  # scales are e4m3's
    assert f(_desc(dtype=lx.LX_E4M3)) == ARG and f(_desc(dtype=lx.LX_E4M3, x_scale=FAR)) == ARG
    assert f(_desc(dtype=lx.LX_E4M3, x_scale=FAR, w_scale=FAR + 2)) == ARG
    assert f(_desc(T=0, x=None), y=None) == OK


def test_linear_gradients():
    L, ws = lx.lib(), 1 << 32
    b = lambda d, dy=Y, lddy=32, pre=None, dx=FAR, dw=None, db=None, w=ws, n=1 << 20: (  # noqa: E731
        L.lx_linear_backward(d, dy, lddy, pre, dx, dw, db, w, n, None))
    need = ctypes.c_uint64()
    assert L.lx_linear_workspace(4, 32, 64, need) == OK and 0 < need.value < 1 << 20
    assert L.lx_linear_workspace(4, 32, 64, None) == ARG and L.lx_linear_workspace(-1, 32, 64, need) == ARG
    assert L.lx_linear_workspace(4, 32, 60, need) == SHAPE
    assert b(_desc(dtype=lx.LX_E4M3, x_scale=FAR, w_scale=FAR)) == UNSUPPORTED
    bad = [b(_desc(), dy=None), b(_desc(), dx=None), b(_desc(), pre=FAR * 4), b(_desc(act=2)), b(_desc(), dx=FAR + 2),
           b(_desc(), dx=X), b(_desc(), dx=W), b(_desc(), dx=Y), b(_desc(), dw=FAR), b(_desc(), db=FAR),
           b(_desc(), w=None), b(_desc(), w=ws + 16), b(_desc(), n=need.value - 1), b(_desc(), w=X), b(_desc(), dy=Y + 1)]
    assert bad == [ARG] * len(bad)
    assert b(_desc(), lddy=31) == SHAPE


def test_head_loss_arguments():
    L, ws = lx.lib(), 1 << 34
    need = ctypes.c_uint64()
    assert L.lx_head_loss_workspace(4, 100, 64, 1, 1, need) == OK and need.value > 0
    assert L.lx_head_loss_workspace(4, 100, 64, 1, 1, None) == ARG
    assert L.lx_head_loss_workspace(0, 100, 64, 1, 1, need) == OK and need.value == 0
    some = ctypes.c_uint64()
    assert L.lx_head_loss_workspace(4, 100, 64, 1, 1, need) == OK
    assert L.lx_head_loss_workspace(4, 100, 64, 0, 0, some) == OK and some.value < need.value
    for T, V, H in ((-1, 100, 64), (4, 0, 64), (4, 100, 0), (4, 100, 63), ((1 << 24) + 1, 100, 64), (4, (1 << 24) + 1, 64)):
        assert L.lx_head_loss_workspace(T, V, H, 1, 1, some) in (ARG, SHAPE)
    lab, loss = 1 << 21, 1 << 22

    def f(h=X, ldh=64, w=W, ldw=64, labels=lab, rw=None, T=4, V=100, H=64, loss=loss, dh=Y, dw=FAR, ws=ws, n=need.value):
        return L.lx_head_loss(h, ldh, w, ldw, labels, rw, T, V, H, loss, dh, dw, ws, n, None)

    assert [f(ldh=63), f(ldh=68), f(ldw=56), f(ldw=65), f(H=60), f(V=0)] == [SHAPE] * 6
    bad = [f(h=None), f(w=None), f(labels=None), f(loss=None), f(h=X + 8), f(w=W + 8), f(dh=Y + 2), f(dw=FAR + 4),
           f(labels=lab + 2), f(rw=lab + 1), f(loss=loss + 1), f(ws=None), f(ws=ws + 16), f(n=need.value - 1), f(dh=X),
           f(dh=W), f(dw=W), f(dw=X), f(loss=lab), f(dh=FAR), f(dh=ws), f(loss=ws + 64), f(T=-1)]
    assert bad == [ARG] * len(bad)


def test_norm_q8_arguments():
    L = lx.lib()
    r, y, q, s, far = 1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24

    def f(q=q, s=s, r_out=far, h=None, stats=None, **kw):
        d = dict(dtype=lx.LX_BF16, T=4, H=64, gate_kind=0, ldr=64, ldy=64, ldg=0, r=r, y=y, gate=None, w_post=None,
                 w_pre=4096, res_scale=1.0, weight_offset=0.0, eps=1e-6)
        d.update(kw)
        return L.lx_residual_norm_q8(lx.ResnormDesc(**d), r_out, q, s, h, stats, None)

    assert L.lx_residual_norm_q8(None, far, q, s, None, None, None) == ARG
    bad = [f(q=None), f(s=None), f(s=s + 2), f(w_pre=None), f(q=r), f(q=y), f(q=far), f(s=r), f(s=q), f(h=q), f(h=far),
           f(s=far), f(stats=s), f(stats=q), f(q=4096), f(r_out=y), f(dtype=lx.LX_E4M3)]
    assert bad == [ARG] * len(bad)
    assert f(H=0) == SHAPE and f(ldr=63) == SHAPE
    assert f(T=0, q=None, s=None) == OK


def test_the_other_calls_do_not_take_e4m3():
    L = lx.lib()
    assert L.lx_distill_loss(lx.LX_E4M3, X, 64, W, W, None, None, None, 4, 64, 2, 1.0, 1.0, 0.0, Y, None, 64, None) == ARG
    assert L.lx_router_balance_backward(lx.LX_E4M3, X, 64, W, W, None, 4, 64, 2, 0.1, 0.0, Y, None) == ARG


# ---- the binding, with tensors that tell of a device; the library only gives sizes of workspaces
@pytest.fixture
def no_library(monkeypatch):
    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError("the library was reached: " + name)
            return call

    monkeypatch.setattr(lx, "_current_device", lambda: 0)
    monkeypatch.setattr(lx, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(lx, "lib", Library)
    for name in ("linear_workspace_bytes", "head_loss_workspace_bytes"):
        monkeypatch.setattr(lx, name, lambda *a: 1 << 16)


BF = torch.bfloat16


def _t(*shape, dtype=BF, dev=0):
    return _on(torch.empty(*shape, dtype=dtype), dev)


def _calls():
    """(call, its tensor arguments by name)."""
    q8 = dict(r=_t(4, 8), y=_t(4, 8), w_pre=_t(8, dtype=torch.float32), r_out=_t(4, 8), h_out=_t(4, 8),
              q_out=_t(4, 8, dtype=torch.float8_e4m3fn), scale_out=_t(4, dtype=torch.float32),
              stats=_t(2, 4, dtype=torch.float32))
    lin = dict(x=_t(4, 16), w=_t(8, 16), bias=_t(8), residual=_t(4, 8), y=_t(4, 8), pre=_t(4, 8))
    e = torch.float8_e4m3fn
    lin8 = dict(x=_t(4, 16, dtype=e), w=_t(8, 16, dtype=e), x_scale=_t(4, dtype=torch.float32),
                w_scale=_t(8, dtype=torch.float32))
    bwd = dict(dy=_t(4, 8), x=_t(4, 16), w=_t(8, 16), pre=_t(4, 8), workspace=_t(1 << 16, dtype=torch.uint8))
    head = dict(h=_t(4, 8), w=_t(9, 8), labels=_t(4, dtype=torch.int32), row_weight=_t(4, dtype=torch.float32),
                workspace=_t(1 << 16, dtype=torch.uint8))
    return [(lx.residual_norm_q8, q8), (lx.linear, lin), (lx.linear, lin8), (lx.linear_backward, bwd), (lx.head_loss, head)]


@pytest.mark.parametrize("i", range(5))
def test_tensors_elsewhere_or_of_another_kind_are_refused(no_library, i):
    f, kw = _calls()[i]
    for name, t in kw.items():
        for other in (_on(t.clone(), 1), _on(t.clone(), -1)):
            with pytest.raises(ValueError):
                f(**{**kw, name: other})
        if name == "workspace":
            continue
        with pytest.raises(ValueError):      # another type
            f(**{**kw, name: _on(torch.empty(t.shape, dtype=torch.float64))})
        if name not in ("x", "w", "r", "h"):
            with pytest.raises(ValueError):  # another size
                f(**{**kw, name: _on(torch.empty(tuple(s + 1 for s in t.shape), dtype=t.dtype))})


def test_shapes_that_do_not_go_together(no_library):
    f = torch.float32
    for call in (lambda: lx.linear(_t(4, 16), _t(8, 24)), lambda: lx.linear(_t(4, 16), _t(8, 16), act="tanh"),
                 lambda: lx.linear(_t(4, 16, dtype=f), _t(8, 16, dtype=f)),
                 lambda: lx.linear(_t(4, 16), _t(8, 16), x_scale=_t(4, dtype=f)),
                 lambda: lx.linear(_t(4, 16, dtype=torch.float8_e4m3fn), _t(8, 16, dtype=torch.float8_e4m3fn)),
                 lambda: lx.linear(_t(16, 4).t(), _t(8, 16)), lambda: lx.linear(_t(4), _t(8, 16)),
                 lambda: lx.head_loss(_t(4, 8), _t(9, 16), _t(4, dtype=torch.int32)),
                 lambda: lx.head_loss(_t(4, 8), _t(9, 8), _t(4, dtype=torch.int64)),
                 lambda: lx.head_loss(_t(4, 8, dtype=f), _t(9, 8, dtype=f), _t(4, dtype=torch.int32)),
                 lambda: lx.residual_norm_q8(_t(4, 8), w_pre=_t(8, dtype=f), q_out=_t(4, 8, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
