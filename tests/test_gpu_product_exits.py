"""Products whose waits give up anywhere, by bounds from next to nothing on: each value is NaN or what it is otherwise,
the call ends, and the calls after it are as they were."""
import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
BOUNDS = [1, 300, 1000, 3000, 10000, 30000]


def _bounded(cycles, call):
    lx.inject_unmet_wait_call(lx.LX_WAIT_NONE, cycles)
    out = call()
    torch.cuda.synchronize()
    return out


def _check(call):
    want = call()
    for cycles in BOUNDS:
        for _ in range(3):
            for g, w in zip(_bounded(cycles, call), want):
                assert bool((torch.isnan(g) | (g == w)).all()), cycles
    assert all(torch.equal(g, w) for g, w in zip(call(), want))


@pytest.mark.parametrize("T,N,K", [(8, 512, 2048), (300, 300, 8192), (600, 4096, 512), (3000, 4096, 2048)])
def test_linear(T, N, K):
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    x, w, r = randn(T, K), randn(N, K) * K ** -0.5, randn(T, N)
    pre = torch.empty(T, N, dtype=BF, device="cuda")
    _check(lambda: (lx.linear(x, w),))
    _check(lambda: (lx.linear(x, w, act="silu", residual=r, pre=pre), pre.clone()))
    dy = randn(T, N)
    _check(lambda: lx.linear_backward(dy, x, w, want_dbias=True))


@pytest.mark.parametrize("T,V,H", [(5, 3000, 512), (700, 5000, 1544), (2100, 33003, 2048)])
def test_head_loss(T, V, H):
    g = torch.Generator(device="cuda").manual_seed(2)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    h, w = randn(T, H).to(BF), (randn(V, H) * 2 * H ** -0.5).to(BF)
    labels = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    _check(lambda: lx.head_loss(h, w, labels))
