"""Argument checks of the operators around a layer, through the C ABI (no GPU): a
refused call returns its status before any CUDA call."""
import ctypes

import pytest

from paper_2608_07814_gb300 import lx

BUF = 4096  # an address that no refused call reads


def _desc(**kw):
    d = dict(dtype=lx.LX_BF16, T=4, H=64, gate_kind=0, ldr=64, ldy=64, ldg=0, r=BUF, y=1 << 20, gate=None,
             w_post=BUF, w_pre=BUF, res_scale=1.0, weight_offset=0.0, eps=1e-6)
    d.update(kw)
    return lx.ResnormDesc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), lx.LX_ERR_ARG), (dict(T=-1), lx.LX_ERR_ARG), (dict(H=0), lx.LX_ERR_SHAPE),
    (dict(H=65537), lx.LX_ERR_SHAPE), (dict(ldr=63), lx.LX_ERR_SHAPE), (dict(ldy=63), lx.LX_ERR_SHAPE),
    (dict(r=None), lx.LX_ERR_ARG), (dict(r=BUF + 1), lx.LX_ERR_ARG), (dict(w_pre=BUF + 2), lx.LX_ERR_ARG),
    (dict(gate_kind=4, gate=BUF), lx.LX_ERR_ARG), (dict(gate_kind=1), lx.LX_ERR_ARG), (dict(gate=BUF), lx.LX_ERR_ARG),
    (dict(gate_kind=3, gate=BUF, ldg=10), lx.LX_ERR_SHAPE), (dict(gate_kind=2, gate=BUF, ldg=-1), lx.LX_ERR_SHAPE),
    (dict(y=None), lx.LX_ERR_ARG), (dict(y=None, w_post=None, w_pre=None), lx.LX_ERR_ARG),
    (dict(eps=float("nan")), lx.LX_ERR_ARG), (dict(eps=-1e-6), lx.LX_ERR_ARG)])
def test_norm_descriptors(kw, status):
    L, d = lx.lib(), _desc(**kw)
    h = 1 << 22 if d.w_pre else None
    assert L.lx_residual_norm(d, 1 << 23, h, None, None) == status
    assert L.lx_residual_norm_backward(d, BUF, BUF, 64, None, 0, 1 << 24, None, None, None, None, None, 0,
                                       None) == status
    assert L.lx_last_error()


def test_norm_outputs():
    L, out, far = lx.lib(), 1 << 23, 1 << 22
    assert L.lx_residual_norm(None, out, far, None, None) == lx.LX_ERR_ARG
    assert L.lx_residual_norm(_desc(), out, None, None, None) == lx.LX_ERR_ARG             # no h_out
    assert L.lx_residual_norm(_desc(w_pre=None), out, far, None, None) == lx.LX_ERR_ARG    # no w_pre
    assert L.lx_residual_norm(_desc(w_pre=None), None, None, None, None) == lx.LX_ERR_ARG  # nothing to write
    assert L.lx_residual_norm(_desc(), BUF + 64, far, None, None) == lx.LX_ERR_ARG         # shifted in place
    assert L.lx_residual_norm(_desc(), 1 << 20, far, None, None) == lx.LX_ERR_ARG          # over y
    assert L.lx_residual_norm(_desc(), out, BUF, None, None) == lx.LX_ERR_ARG              # h over r
    assert L.lx_residual_norm(_desc(), out, out + 64, None, None) == lx.LX_ERR_ARG         # each other
    assert L.lx_residual_norm(_desc(T=0), None, None, None, None) == lx.LX_OK
    b = lambda d, stats=BUF, dr=BUF, dh=None, out=1 << 24, dy=None, w1=None, dg=None, w2=None, ws=None, n=0: (  # noqa: E731
        L.lx_residual_norm_backward(d, stats, dr, 64, dh, 64, out, dy, w1, dg, w2, ws, n, None))
    bad = [b(_desc(), stats=None), b(_desc(), dr=None), b(_desc(), dg=BUF), b(_desc(w_post=None), w1=BUF),
           b(_desc(w_pre=None), w2=BUF), b(_desc(w_pre=None), dh=BUF), b(_desc(y=None, w_post=None), dy=BUF),
           b(_desc(), out=BUF), b(_desc(), dy=1 << 24), b(_desc(), w1=BUF), b(_desc(), w1=BUF, ws=BUF, n=8),
           b(_desc(), w1=BUF, ws=BUF + 4, n=1 << 30)]
    assert bad == [lx.LX_ERR_ARG] * len(bad)


def test_workspace_sizes():
    n = ctypes.c_uint64()
    L = lx.lib()
    for f in (L.lx_residual_norm_workspace, L.lx_router_balance_workspace):
        assert f(4, 64, None) == lx.LX_ERR_ARG
        assert f(-1, 64, n) == lx.LX_ERR_ARG
        assert f(100000, 64, n) == lx.LX_OK and 0 < n.value < 1 << 24
    assert L.lx_residual_norm_workspace(4, 65537, n) == lx.LX_ERR_SHAPE
    assert L.lx_router_balance_workspace(4, 1025, n) == lx.LX_ERR_ARG


def test_balance_calls():
    L = lx.lib()
    ok = dict(dtype=0, logits=BUF, ld=16, ids=BUF, mask=None, T=4, E=16, k=2, counts=BUF, prob=BUF, lse=BUF, loss=BUF,
              ws=BUF, n=1 << 20)

    def call(**kw):
        v = dict(ok, **kw)
        return L.lx_router_balance(v["dtype"], v["logits"], v["ld"], v["ids"], v["mask"], v["T"], v["E"], v["k"], 0.1, 0.1,
                                   v["counts"], v["prob"], v["lse"], v["loss"], v["ws"], v["n"], None)

    for kw in (dict(dtype=3), dict(T=-1), dict(E=0), dict(E=1025), dict(k=0), dict(k=33), dict(logits=None), dict(ids=None),
               dict(counts=None), dict(prob=None), dict(lse=None), dict(loss=None), dict(ws=None), dict(n=7),
               dict(logits=BUF + 2), dict(ids=BUF + 1), dict(ws=BUF + 8)):
        assert call(**kw) == lx.LX_ERR_ARG, kw
    assert call(ld=15) == lx.LX_ERR_SHAPE
    back = lambda **kw: L.lx_router_balance_backward(*[dict(  # noqa: E731
        dtype=0, logits=BUF, ld=16, lse=BUF, counts=BUF, dloss=None, T=4, E=16, k=2, a=0.1, b=0.1, out=1 << 20, s=None,
        **{}) | kw][0].values())
    for kw in (dict(dtype=3), dict(T=-1), dict(E=0), dict(k=0), dict(logits=None), dict(lse=None), dict(counts=None),
               dict(out=None), dict(out=BUF + 64), dict(out=(1 << 20) + 2), dict(dloss=BUF + 1)):
        assert back(**kw) == lx.LX_ERR_ARG, kw
    assert back(ld=15) == lx.LX_ERR_SHAPE
    assert back(T=0) == lx.LX_OK


def test_distill_calls():
    L = lx.lib()

    def call(**kw):
        v = dict(dtype=0, logits=BUF, ld=50, ids=BUF, top=BUF, tl=None, labels=None, w=None, T=4, V=50, K=2, tau=1.0, a=1.0,
                 b=0.0, loss=BUF, d=1 << 20, ldd=50, s=None)
        v.update(kw)
        return L.lx_distill_loss(*v.values())

    for kw in (dict(dtype=2), dict(T=-1), dict(K=0), dict(K=1025), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("inf")),
               dict(tau=float("nan")), dict(b=0.5), dict(logits=None), dict(ids=None), dict(top=None), dict(loss=None),
               dict(logits=BUF + 2), dict(top=BUF + 2), dict(d=BUF + 4), dict(d=BUF, ldd=51), dict(labels=BUF + 1)):
        assert call(**kw) == lx.LX_ERR_ARG, kw
    for kw in (dict(V=0), dict(ld=49), dict(ldd=49)):
        assert call(**kw) == lx.LX_ERR_SHAPE, kw
    assert call(T=0) == lx.LX_OK
