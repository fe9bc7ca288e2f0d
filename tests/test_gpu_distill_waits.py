"""A wait that runs out in lx_distill_loss shows in its results: NaN losses and gradients
(rows of weight 0 apart), the launch ends normally, and the next call gives the bits of
the call before.  One CTA a row, a cluster a row, and rows read from L2."""
import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu

SHORT = 2_000_000  # SM clock cycles, about 1 ms


@pytest.mark.parametrize("T,V,dtype", [(300, 3000, torch.float32), (5, 33000, torch.bfloat16),
                                       (400, 100000, torch.bfloat16), (3, 1 << 20, torch.bfloat16)])
def test_gives_nan_and_recovers(T, V, dtype):
    g = torch.Generator().manual_seed(T)
    z = torch.randn(T, V, generator=g).to(dtype).cuda()
    ids = torch.randint(0, V, (T, 8), generator=g, dtype=torch.int32).cuda()
    top, w = torch.randn(T, 8, generator=g).cuda(), torch.ones(T, device="cuda")
    w[1] = 0
    run = lambda **kw: lx.distill_loss(z, ids, top, row_weight=w, **kw)  # noqa: E731
    loss, d = run()
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(d).all())
    on = w != 0
    for grad in (True, False):
        lx.inject_unmet_wait_call(lx.LX_WAIT_CALL_SUMS, SHORT)
        bad, db = run(want_grad=grad)
        torch.cuda.synchronize()
        assert bool(torch.isnan(bad[on]).all())
        assert not grad or bool(torch.isnan(db[on]).all())
        again, da = run()
        assert torch.equal(again, loss) and torch.equal(da, d)


def test_short_bound_alone_does_not_fire():
    z = torch.randn(200, 5000, device="cuda")
    ids, top = torch.zeros(200, 3, dtype=torch.int32, device="cuda"), torch.zeros(200, 3, device="cuda")
    lx.inject_unmet_wait_call(lx.LX_WAIT_NONE, SHORT)
    loss, d = lx.distill_loss(z, ids, top)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(d).all())
