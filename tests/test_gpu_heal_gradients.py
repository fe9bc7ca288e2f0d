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


def _rms(v, eps):
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def test_gradients_of_a_step_are_those_of_its_loss(heal, monkeypatch):
    """One step's gradients against autograd through the step in fp64, the experts' outputs and
    the experts' counts held fixed as the example holds them.  The example's tensors between
    the operators are bf16 (2^-9 of a value): the logits, about 3 and 13 at most, are off by
    0.006 and 0.025, and so are the shares of the softmax; the other roundings are smaller.  A
    gradient adds over 384 tokens, so 5 % of its length holds it."""
    seen, built = [], {}
    build, forward = heal.build, heal.Block.forward

    def kept(seed=0):
        built["all"] = build(seed)
        built["start"] = [[p.clone() for p in (b.w_post, b.gate, b.w_pre)] for b in built["all"][1]]
        return built["all"]

    def watched(self, r, h, keep=False):
        out = forward(self, r, h, keep)
        if keep:
            seen.append((out[2][1], out[2][3]))
        return out

    monkeypatch.setattr(heal, "build", kept)
    monkeypatch.setattr(heal.Block, "forward", watched)
    temperature = 2.0
    (total, kd, _), _ = heal.heal(steps=1, temperature=temperature)[0]
    teacher, student, first, x, head = built["all"]
    ids, top, lse = heal.targets(teacher, first, x, head, temperature)
    d = lambda t: t.detach().double()  # noqa: E731
    params = [[d(p).requires_grad_(True) for p in ps] for ps in built["start"]]
    r = d(x)
    h = _rms(r, heal.EPS) * d(first)
    loss = 0.0
    for i, (b, (y, experts), (w_post, gate, w_pre)) in enumerate(zip(student, seen, params)):
        if i:
            rl = h @ d(b.router).t()
            load = torch.zeros_like(rl).scatter_(1, experts.long(), 1.0).sum(0)
            n = rl.shape[0]
            loss = loss + heal.BALANCE * heal.E * (load / (n * heal.K) * torch.softmax(rl, 1).mean(0)).sum()
            loss = loss + heal.Z * (torch.logsumexp(rl, 1) ** 2).mean()
        r = r + gate * (_rms(d(y), heal.EPS) * w_post)
        h = _rms(r, heal.EPS) * w_pre
    logits = h @ d(head).t()
    lq = d(top) / temperature - d(lse)[:, None]
    lp = torch.log_softmax(logits / temperature, 1).gather(1, ids.long())
    distilled = temperature ** 2 * (lq.exp() * (lq - lp)).sum(1).mean()
    assert abs(distilled.item() - kd) <= 0.02 and abs((loss + distilled).item() - total) <= 0.02
    (loss + distilled).backward()
    for b, (w_post, gate, w_pre) in zip(student, params):
        pairs = [(b.w_post.grad, w_post), (b.gate.grad, gate)] + ([(b.w_pre.grad, w_pre)] if b is student[-1] else [])
        for got, p in pairs:
            assert float((d(got) - p.grad).norm()) <= 0.05 * float(p.grad.norm())
