"""The products around a layer together, as examples/heal.py uses them, on several streams at once
and in CUDA graphs."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import products as O
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16


@pytest.fixture(scope="module")
def heal():
    spec = importlib.util.spec_from_file_location("heal", os.path.join(ROOT, "examples", "heal.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _rms(v, eps):
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def test_a_step_on_labels_has_its_loss_s_gradients(heal):
    """Gradients of the example's step against autograd through it in fp64, from the layers' own outputs.
    What passes between the operators is bf16, 2^-9 of a value each time: eight such roundings on
    the longest way from the loss to a gradient, and logits of size 3 off by 0.006, so 5 % of a
    gradient's length holds them."""
    _, student, first, x, head = heal.build()
    g = torch.Generator(device="cuda").manual_seed(5)
    expert = heal.Shared(g)
    labels = torch.randint(0, heal.VOCAB, (heal.TOKENS,), generator=g, device="cuda", dtype=torch.int32)
    labels[::5] = -100
    weight = torch.rand(heal.TOKENS, generator=g, device="cuda") / heal.TOKENS
    loss, grads = heal.labels_step(student, expert, first, x, head, labels, weight)
    r, h = lx.residual_norm(x, w_pre=first, eps=heal.EPS)
    for b in student[:-1]:
        r, h, _ = b.forward(r, h)
    b = student[-1]
    y = b.layer.moe_forward(h, heal.K).double()
    p = {n: t.detach().double().requires_grad_(True) for n, t in dict(
        head=head, up=expert.up, bias=expert.bias, down=expert.down, w_post=b.w_post, gate=b.gate, w_pre=b.w_pre).items()}
    a = torch.nn.functional.gelu(h.double() @ p["up"].t() + p["bias"])
    y = y + a @ p["down"].t()
    out = _rms(r.double() + p["gate"] * _rms(y, heal.EPS) * p["w_post"], heal.EPS) * p["w_pre"]
    live = labels >= 0
    want = (torch.nn.functional.cross_entropy((out @ p["head"].t())[live], labels[live].long(), reduction="none")
            * weight[live].double()).sum()
    assert abs(loss.item() - want.item()) <= 0.01 * want.item()
    want.backward()
    for n, t in p.items():
        assert float((grads[n].double() - t.grad).norm()) <= 0.05 * float(t.grad.norm()), n


def test_the_example_runs_and_its_expert_is_served_in_8_bits(heal):
    """The served expert against float64 of the stored values: q and the weights as they are in
    8 bits, one rounding to bf16 between the products (2^-8) and one behind them."""
    _, student, first, x, head = heal.build()
    losses, expert = heal.train_on_labels(student, first, x, head, steps=2)
    assert len(losses) == 2 and all(np.isfinite(losses))
    g = torch.Generator(device="cuda").manual_seed(3)
    y = torch.randn(heal.TOKENS, heal.H, generator=g, device="cuda").to(BF)
    r_out, got = heal.shared_8bit(expert, x, y, first)
    n = lx.residual_norm_q8(x, y, w_pre=first, eps=heal.EPS)
    assert torch.equal(r_out, n.r_out)
    up, s = heal.to_8bit(expert.up)
    d = lambda t: t.float().cpu().double().numpy()  # noqa: E731
    a, _ = O.linear(d(n.q) * d(n.scale)[:, None], d(up) * d(s)[:, None], "gelu", d(expert.bias))
    want = a @ d(expert.down).T
    err = (2.0 ** -8 + 1e-4) * (np.abs(a) @ np.abs(d(expert.down)).T) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(d(got) - want) <= err + 1e-6).all()
    # and the 8 bits themselves: each value within half a step of e4m3, at most 2^-4 of it or 2^-10 of the
    # scale's unit, on both sides of the product
    h = d(lx.residual_norm(x, y, w_pre=first, eps=heal.EPS)[1])
    qerr = np.maximum(2.0 ** -4 * np.abs(h), 2.0 ** -10 * d(n.scale)[:, None]) + 2.0 ** -8 * np.abs(h) + 1e-5
    assert (np.abs(d(n.q) * d(n.scale)[:, None] - h) <= qerr).all()


def _pass(seed, T, H, N, V):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(BF)  # noqa: E731
    t = dict(r=randn(T, H), y=randn(T, H), w=randn(N, H, std=H ** -0.5), b=randn(N), v=randn(V, H, std=H ** -0.5),
             dy=randn(T, N), wp=1 + randn(H, std=0.1).float(),
             labels=torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32))
    w8 = (t["w"].float() * 100).to(torch.float8_e4m3fn)
    ws = torch.full((N,), 0.01, device="cuda")

    def run():
        n = lx.residual_norm_q8(t["r"], t["y"], w_pre=t["wp"])
        a = lx.linear(n.q, w8, x_scale=n.scale, w_scale=ws, bias=t["b"], act="silu")
        pre = torch.empty(T, N, dtype=BF, device="cuda")
        y = lx.linear(n.r_out, t["w"], bias=t["b"], act="gelu", pre=pre, residual=a)
        d = lx.linear_backward(t["dy"], n.r_out, t["w"], act="gelu", pre=pre, want_dbias=True)
        return [n.r_out, n.q.view(torch.uint8), n.scale, a, pre, y, *d, *lx.head_loss(n.r_out, t["v"], t["labels"])]

    return t, run


SHAPES = [(1, 256, 512, 3001), (70, 272, 1003, 2000), (300, 512, 300, 5000), (1500, 256, 2048, 1000)]


def test_streams_at_the_same_time():
    runs = [_pass(i, *s)[1] for i, s in enumerate(SHAPES)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(5):
        got = []
        for run, s in zip(runs, streams):
            with torch.cuda.stream(s):
                got.append(run())
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_a_given_stream():
    t, _ = _pass(0, *SHAPES[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    n0, n1 = (lx.residual_norm_q8(t["r"], t["y"], w_pre=t["wp"], stream=st) for st in (None, s))
    y0, y1 = (lx.linear(t["r"], t["w"], bias=t["b"], stream=st) for st in (None, s))
    d0, d1 = (lx.linear_backward(t["dy"], t["r"], t["w"], stream=st) for st in (None, s))
    h0, h1 = (lx.head_loss(t["r"], t["v"], t["labels"], stream=st) for st in (None, s))
    torch.cuda.synchronize()
    for a, b in zip((n0.scale, y0, *d0[:2], *h0), (n1.scale, y1, *d1[:2], *h1)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", SHAPES)
def test_graphs_replayed_on_new_inputs(shape):
    """Two graphs captured with their own buffers, replayed in turn after the inputs changed in place."""
    t, run = _pass(1, *shape)
    run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    for turn in range(3):
        new, _ = _pass(10 + turn, *shape)
        for n in ("r", "y", "b", "dy", "labels"):
            t[n].copy_(new[n])
        want = run()
        torch.cuda.synchronize()
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_workspace_of_the_caller_s_is_used_again():
    T, H, N, V = SHAPES[2]
    (t, _), (u, _) = _pass(1, T, H, N, V), _pass(2, T, H, N, V)
    ws = torch.full((lx.head_loss_workspace_bytes(T, V, H),), 255, dtype=torch.uint8, device="cuda")
    wl = torch.full((lx.linear_workspace_bytes(T, N, H),), 255, dtype=torch.uint8, device="cuda")
    for v in (t, u, t):
        a, b = lx.head_loss(v["r"], v["v"], v["labels"], workspace=ws), lx.head_loss(v["r"], v["v"], v["labels"])
        c, d = lx.linear_backward(v["dy"], v["r"], v["w"], workspace=wl), lx.linear_backward(v["dy"], v["r"], v["w"])
        assert all(torch.equal(p, q) for p, q in zip((*a, *c[:2]), (*b, *d[:2])))
