"""examples/heal.py trains what it says: the reported total is the loss that the gradients belong
to, and a gradient is formed for the optimiser's parameters alone."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def heal():
    spec = importlib.util.spec_from_file_location("heal", os.path.join(ROOT, "examples", "heal.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_only_what_is_trained_counts(heal, monkeypatch):
    built, calls = {}, {"balance": 0, "backward": 0}
    build, forward, backward = heal.build, heal.lx.router_balance, heal.lx.router_balance_backward

    def kept(seed=0):
        built["all"] = build(seed)
        return built["all"]

    def counted(name, fn):
        def call(*a, **k):
            calls[name] += 1
            return fn(*a, **k)
        return call

    monkeypatch.setattr(heal, "build", kept)
    monkeypatch.setattr(heal.lx, "router_balance", counted("balance", forward))
    monkeypatch.setattr(heal.lx, "router_balance_backward", counted("backward", backward))
    (total, kd, bal), counts = heal.heal(steps=1)[0]
    assert calls["balance"] == calls["backward"] == heal.BLOCKS - 1
    student = built["all"][1]
    for b in student:
        assert b.w_post.grad is not None and b.gate.grad is not None
        assert (b.w_pre.grad is not None) == (b is student[-1])
    z = (total - kd - heal.BALANCE * bal) / heal.Z  # one router's: mean of lse^2, lse about log E
    assert bal >= 0.9 and 0 < z < 100
    assert counts[-1] == heal.TOKENS
