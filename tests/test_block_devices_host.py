"""Every tensor of a call around a layer is on one device, the current one, and a caller's
workspace is a contiguous array there: anything else is refused before the library is
reached.  The tensors lie in host memory and tell of a device; the library is not called."""
import pytest
import torch

from paper_2608_07814_gb300 import lx


class On(torch.Tensor):
    """A tensor that says it is on device `dev`."""
    dev = 0

    is_cuda = property(lambda self: self.dev >= 0)

    def get_device(self):
        return self.dev


def _on(t, dev=0):
    t = t.as_subclass(On)
    t.dev = dev
    return t


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """Device 0 is current; the library only gives sizes of workspaces."""
    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError("the library was reached: " + name)
            return call

    monkeypatch.setattr(lx, "_current_device", lambda: 0)
    monkeypatch.setattr(lx, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(lx, "lib", Library)
    for name in ("residual_norm_workspace_bytes", "router_balance_workspace_bytes"):
        monkeypatch.setattr(lx, name, lambda *a: 1 << 16)


T, H, K = 4, 8, 2


def _calls():
    """name: (call, its tensors)."""
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ws = lambda: torch.zeros(1 << 16, dtype=torch.uint8)  # noqa: E731
    return {
        "norm": (lambda r, y, **k: lx.residual_norm(r, y, **k),
                 dict(r=f(T, H), y=f(T, H), w_post=f(H), gate=f(H), w_pre=f(H), r_out=f(T, H), h_out=f(T, H), stats=f(2, T))),
        "norm, token gate": (lambda r, y, **k: lx.residual_norm(r, y, **k),
                             dict(r=f(T, H), y=f(T, H), gate=f(T, 1), w_pre=f(H))),
        "norm, full gate": (lambda r, y, **k: lx.residual_norm(r, y, **k),
                            dict(r=f(T, H), y=f(T, H), gate=f(T, H), w_pre=f(H))),
        "norm backward": (lambda dr_out, dh, r, y, stats, **k: lx.residual_norm_backward(dr_out, dh, r, y, stats, **k),
                          dict(dr_out=f(T, H), dh=f(T, H), r=f(T, H), y=f(T, H), stats=f(2, T), w_post=f(H), gate=f(H),
                               w_pre=f(H), workspace=ws())),
        "balance": (lambda logits, ids, **k: lx.router_balance(logits, ids, **k),
                    dict(logits=f(T, H), ids=i(T, K), mask=torch.ones(T, dtype=torch.bool), workspace=ws())),
        "balance backward": (lambda logits, lse, counts, **k: lx.router_balance_backward(
            logits, lx.RouterBalance(None, counts, None, lse), K, **k),
            dict(logits=f(T, H), lse=f(T), counts=i(H + 1), dloss=f(1), out=f(T, H))),
        "distill": (lambda logits, ids, top, **k: lx.distill_loss(logits, ids, top, **k),
                    dict(logits=f(T, H), ids=i(T, K), top=f(T, K), teacher_lse=f(T), labels=i(T), row_weight=f(T),
                         dlogits=f(T, H))),
    }


CASES = [(c, a) for c, (_, kw) in _calls().items() for a in kw]


@pytest.mark.parametrize("call", list(_calls()))
def test_one_device_is_taken(call):
    fn, kw = _calls()[call]
    with pytest.raises(AssertionError, match="reached"):
        fn(**{k: _on(t) for k, t in kw.items()})


@pytest.mark.parametrize("elsewhere", [1, -1])
@pytest.mark.parametrize("call,arg", CASES)
def test_a_tensor_elsewhere_is_refused(call, arg, elsewhere):
    """On another device, or in host memory (-1)."""
    fn, kw = _calls()[call]
    with pytest.raises(ValueError):
        fn(**{k: _on(t, elsewhere if k == arg else 0) for k, t in kw.items()})


@pytest.mark.parametrize("call", list(_calls()))
def test_another_current_device_is_refused(call, monkeypatch):
    fn, kw = _calls()[call]
    monkeypatch.setattr(lx, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        fn(**{k: _on(t) for k, t in kw.items()})


@pytest.mark.parametrize("call", ["norm backward", "balance"])
def test_a_workspace_of_repeated_bytes_is_refused(call):
    fn, kw = _calls()[call]
    kw["workspace"] = torch.zeros(1, dtype=torch.uint8).expand(1 << 16)
    with pytest.raises(ValueError, match="workspace"):
        fn(**{k: _on(t) for k, t in kw.items()})
