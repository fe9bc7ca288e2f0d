"""The operators around a layer on several streams at the same time: the bits of the calls made
one after the other."""
import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu


def _pass(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r, y, dr, dh = (torch.randn(900, 1030, generator=g, device="cuda").bfloat16() for _ in range(4))
    w = torch.randn(1030, generator=g, device="cuda")
    rl = torch.randn(5000, 128, generator=g, device="cuda")
    ids = torch.topk(rl, 8, dim=1).indices.int()
    zs = [torch.randn(T, V, generator=g, device="cuda").bfloat16() for T, V in ((700, 4096), (300, 40000), (160, 100000))]
    tops = [torch.topk(z.float(), 24, dim=1) for z in zs]
    tops = [(t.indices.int(), t.values) for t in tops]

    def run():
        stats = torch.empty(2, 900, device="cuda")
        out = list(lx.residual_norm(r, y, w_post=w, gate=w, w_pre=w, stats=stats))
        out += lx.residual_norm_backward(dr, dh, r, y, stats, w_post=w, gate=w, w_pre=w)
        b = lx.router_balance(rl, ids, z_coef=0.1)
        out += [*b, lx.router_balance_backward(rl, b, 8, z_coef=0.1)]
        for z, (i, t) in zip(zs, tops):
            out += lx.distill_loss(z, i, t, temperature=2.0)
        return out

    return run


def test_streams_at_the_same_time():
    runs = [_pass(s) for s in range(4)]
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
