"""Which kernel a product takes, and so the order of its sums, goes by T, N, K and the type: y, pre and residual are the
same bits wherever their rows lie.  The sizes are such that few tokens and tiles take about the same time."""
import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn


@pytest.mark.parametrize("dtype", [BF, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", [(64, 2048, 512), (160, 1024, 1024), (250, 512, 2048), (300, 512, 2048), (400, 1024, 2048),
                                   (500, 504, 2048), (300, 2048, 4096), (700, 512, 4096)])
def test_outputs_off_the_16_byte_grid(T, N, K, dtype):
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(T, K, generator=g), torch.randn(N, K, generator=g) / K ** 0.5
    kw = {}
    if dtype == E4M3:
        w = w * 30
        kw = dict(x_scale=(0.5 + torch.rand(T, generator=g)).cuda(), w_scale=(0.5 + torch.rand(N, generator=g)).cuda())
    x, w = x.to(dtype).cuda(), w.to(dtype).cuda()
    res = torch.randn(T, N, generator=g).to(BF).cuda()
    for r in (None, res):
        want = lx.linear(x, w, act="silu", residual=r, **kw)
        for pad, at in ((1, 1), (8, 0), (5, 3), (4, 2), (8, 4)):
            wide = torch.full((T, N + pad), 7.0, dtype=BF, device="cuda")
            y = lx.linear(x, w, act="silu", residual=r, y=wide[:, at:at + N], **kw)
            assert torch.equal(y, want), (pad, at)
