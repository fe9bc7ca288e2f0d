"""A wait that runs out in the middle of lx_distill_loss: a row is right, loss and gradient to
the bit, or it is NaN throughout; rows of weight 0 are zero; the next call is right again.
Each of the kernel's waits is made to run out, in rows of one CTA, of clusters and in rows
that are not held, three rows and more to each."""
import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu

SHORT = 2_000_000  # SM clock cycles, about 1 ms


def _case(T, V, dtype, far, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(T, V, generator=g, device="cuda").mul_(2.5)
    if far:  # rows that are summed again: further from zero than their references hold
        z[::3] = torch.randint(0, 3, z[::3].shape, generator=g, device="cuda").mul(2.0 ** 27) + 2.0 ** 33
    ids = torch.randint(0, V, (T, 8), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand(T, generator=g, device="cuda") + 0.5
    w[1::5] = 0
    lab = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    return z.to(dtype), ids, torch.randn(T, 8, generator=g, device="cuda"), lab, w


@pytest.mark.parametrize("site", [lx.LX_WAIT_CALL_SUMS, lx.LX_WAIT_CALL_ENTRIES, lx.LX_WAIT_CALL_WRITTEN,
                                  lx.LX_WAIT_CALL_AGAIN])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T,V,dtype", [(1700, 8301, torch.float32), (700, 40000, torch.bfloat16),
                                       (500, 100000, torch.bfloat16), (400, 150001, torch.bfloat16),
                                       (480, 400000, torch.float32)])
def test_a_row_is_right_or_nan(T, V, dtype, in_place, site):
    z, ids, top, lab, w = _case(T, V, dtype, site == lx.LX_WAIT_CALL_AGAIN, seed=T)
    run = lambda **kw: lx.distill_loss(z, ids, top, row_weight=w, labels=lab, kd_weight=0.7, ce_weight=0.3,  # noqa: E731
                                       temperature=2.0, **kw)
    loss, d = run()
    assert torch.isfinite(loss).all() and torch.isfinite(d).all()
    off = w == 0
    for grad in (True, False):
        src = z.clone()
        lx.inject_unmet_wait_call(site, SHORT)
        bad, db = run(want_grad=grad, dlogits=z if in_place and grad else None)
        torch.cuda.synchronize()
        lost = torch.isnan(bad)
        assert not lost[off].any()
        # (losses alone are right before the wait for a row's dense values)
        assert lost.any() or (not grad and site == lx.LX_WAIT_CALL_WRITTEN)
        assert torch.equal(bad[~lost], loss[~lost])
        if grad:
            assert torch.isnan(db[lost]).all()
            assert torch.equal(db[~lost], d[~lost])
        z.copy_(src)
    again, da = run()
    assert torch.equal(again, loss) and torch.equal(da, d)
