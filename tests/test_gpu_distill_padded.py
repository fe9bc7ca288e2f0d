"""lx_distill_loss on ragged stores: entries at -inf are skipped whatever valid id they carry,
as entries with an id outside the vocabulary are.  A store padded with (id, -inf) therefore gives
the bits of one padded with id -1, and the entry at id 0 or the label there keeps its value."""
import pytest
import torch

from block_checks import close, f64
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau,lse", [(1.0, False), (2.0, True)])
@pytest.mark.parametrize("T,V,K", [(3000, 200, 16), (2000, 1000, 32), (700, 4104, 200), (600, 16384, 1000),
                                   (400, 40000, 64), (160, 100001, 300)])
def test_padding_is_skipped(T, V, K, tau, lse, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    z = torch.randn(T, V, generator=g, device="cuda").mul_(2.5).to(dtype)
    top, ids = torch.rand(T, V, generator=g, device="cuda").topk(K, dim=1)
    ids[::7, 0] = 0                                     # an entry of its own at the padding's id
    keep = torch.randint(1, K + 1, (T, 1), generator=g, device="cuda")
    gone = torch.arange(K, device="cuda") >= keep
    gone[5] = True                                      # a token with nothing but padding
    top = (top * 8).float()
    lab = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lab[::3] = 0
    w = torch.rand(T, generator=g, device="cuda") + 0.5
    kw = dict(temperature=tau, teacher_lse=torch.full((T,), 9.0, device="cuda") if lse else None, kd_weight=0.7,
              labels=lab, ce_weight=0.3, row_weight=w)
    inf = float("inf")
    loss, d = lx.distill_loss(z, ids.masked_fill(gone, -1).int(), top.masked_fill(gone, -inf), **kw)
    for pad in (0, V - 1):
        l2, d2 = lx.distill_loss(z, ids.masked_fill(gone, pad).int(), top.masked_fill(gone, -inf), **kw)
        assert torch.equal(l2, loss)
        assert torch.equal(d2, d), pad
    some = torch.tensor([0, 5, 6, 7, T - 1], device="cuda")
    pick = lambda t: f64(t[some])  # noqa: E731
    wl, wd, mag = block.distill(pick(z), ids.masked_fill(gone, 0)[some].cpu().numpy(), pick(top.masked_fill(gone, -inf)),
                                tau, pick(kw["teacher_lse"]) if lse else None, 0.7, lab[some].cpu().numpy(), 0.3, pick(w),
                                True)
    # bounds as in test_gpu_distill.py
    close(loss[some], wl, False, (float(z.float().abs().max()) + 10) * tau * 1.5, "loss")
    close(d[some], wd, dtype == torch.bfloat16, mag + 1e-3 * pick(w)[:, None] * (0.7 * tau + 0.3), "dlogits")
