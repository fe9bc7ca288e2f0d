"""lx_router_balance and its backward against the float64 definition (oracle/block.py)."""
import numpy as np
import pytest
import torch

from block_checks import close, f64, gen
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(T, E, k, dtype, masked=0.0, pad=0, odd_ids=False, seed=0):
    g = gen(seed)
    skew = -torch.log(1.0 + torch.randperm(E, generator=g).float())
    wide = torch.zeros(T, E + pad)
    wide[:, :E] = torch.randn(T, E, generator=g) + skew
    logits = wide.to(DT[dtype]).cuda()[:, :E]
    ids = torch.topk(wide[:, :E], min(k, E), dim=1).indices.to(torch.int32)
    if k > E:
        ids = torch.cat([ids, torch.full((T, k - E), -1, dtype=torch.int32)], 1)
    if odd_ids:  # ids out of range and repeats
        out = torch.rand(T, k, generator=g)
        ids[out < 0.1] = torch.tensor([-1, E, 1 << 30], dtype=torch.int32)[
            torch.randint(0, 3, (int((out < 0.1).sum()),), generator=g)]
        if k > 1:
            again = torch.rand(T, generator=g) < 0.3
            ids[again, k - 1] = ids[again, 0]
    mask = None if masked == 0 else (torch.rand(T, generator=g) >= masked).cuda()
    return logits, ids.cuda(), mask


def _check(logits, ids, mask, dtype, alpha=0.3, beta=0.05):
    k = ids.shape[1]
    b = lx.router_balance(logits, ids, mask=mask, balance_coef=alpha, z_coef=beta)
    up = torch.tensor([1.5], device="cuda")
    d = lx.router_balance_backward(logits, b, k, dloss=up, balance_coef=alpha, z_coef=beta)
    torch.cuda.synchronize()
    l, i, m = f64(logits), ids.cpu().numpy(), None if mask is None else mask.cpu().numpy()
    loss, counts, prob, lse = block.router_balance(l, i, m, alpha, beta)
    assert np.array_equal(b.counts.cpu().numpy(), counts)
    close(b.prob, prob, False, what="prob")
    close(b.lse, lse, False, what="lse")
    close(b.loss, loss, False, np.abs(loss) + 1e-6, "loss")
    close(d, block.router_balance_grad(l, i, m, alpha, beta, 1.5), dtype == "bf16", what="dlogits")
    return b, d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (64, 128, 8), (77, 8, 2), (700, 64, 6), (301, 256, 8), (40, 512, 32),
                                   (65, 1024, 8), (3, 1, 1), (50, 7, 3), (129, 130, 4), (33, 257, 1), (9, 1023, 32),
                                   (5, 4, 32)])
def test_against_the_definition(T, E, k, dtype):
    _check(*_inputs(T, E, k, dtype, seed=T + E), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,k", [(128, 8), (60, 12), (513, 3)])
def test_masks_odd_ids_and_slices(E, k, dtype):
    for pad in (0, 5, 8):
        _check(*_inputs(211, E, k, dtype, 0.4, pad, True, seed=E + pad), dtype)


def test_many_tokens():
    """More rows than a resident grid holds."""
    _check(*_inputs(20000, 32, 4, "f32", 0.1, seed=1), "f32")


def test_masked_garbage_is_not_read():
    logits, ids, mask = _inputs(100, 64, 4, "f32", 0.5, seed=2)
    want, dwant = _check(logits, ids, mask, "f32")
    bad = logits.clone()
    off = ~mask
    bad[off] = float("nan")
    bad[off, 0] = float("inf")
    got = lx.router_balance(bad, ids, mask=mask, balance_coef=0.3, z_coef=0.05)
    d = lx.router_balance_backward(bad, got, 4, dloss=torch.tensor([1.5], device="cuda"), balance_coef=0.3,
                                   z_coef=0.05)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(d, dwant) and (d[off] == 0).all()


@pytest.mark.parametrize("E", [16, 200, 1024])
def test_experts_masked_by_infinity_and_lowest_value(E):
    """Experts at -inf or at the type's lowest value have no probability; rows of
    nothing but -inf do not count."""
    logits, ids, mask = _inputs(60, E, 2, "f32", 0.2, seed=E)
    logits[:, E // 2:] = -float("inf")
    logits[5], logits[59] = -float("inf"), -float("inf")
    logits[7, 1:] = torch.finfo(torch.float32).min
    _check(logits, ids, mask, "f32")


def test_nothing_counts():
    logits, ids, _ = _inputs(10, 32, 4, "f32", seed=3)
    b, d = _check(logits, ids, torch.zeros(10, dtype=torch.uint8, device="cuda"), "f32")
    assert (b.loss == 0).all() and (d == 0).all() and (b.counts == 0).all()
    e = lx.router_balance(logits[:0], ids[:0], z_coef=0.1)
    assert (e.loss == 0).all() and (e.counts == 0).all()
    assert lx.router_balance_backward(logits[:0], e, 4).shape == (0, 32)


def test_nan_and_infinity_show():
    logits, ids, _ = _inputs(10, 32, 4, "f32", seed=4)
    logits[3, 3] = float("nan")
    b = lx.router_balance(logits, ids, z_coef=0.1)
    assert torch.isnan(b.loss).all() and torch.isnan(b.lse[3]) and torch.isfinite(b.lse[:3]).all()


def test_counts_are_those_of_the_statistics():
    _, ids, _ = _inputs(3000, 128, 8, "f32", odd_ids=True, seed=5)
    b = lx.router_balance(torch.zeros(3000, 128, device="cuda"), ids)
    fire, _ = lx.coact_accumulate(ids, 128)
    assert torch.equal(b.counts[:128].long(), fire) and int(b.counts[128]) == 3000


def test_in_place_repeats_and_side_stream():
    logits, ids, mask = _inputs(3000, 128, 8, "f32", 0.1, seed=6)
    b = lx.router_balance(logits, ids, mask=mask, z_coef=0.1)
    d = lx.router_balance_backward(logits, b, 8, z_coef=0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = lx.router_balance(logits, ids, mask=mask, z_coef=0.1, stream=side)
    e = lx.router_balance_backward(logits, c, 8, z_coef=0.1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((*b, d), (*c, e)):
        assert torch.equal(x, y)
    buf = logits.clone()
    assert lx.router_balance_backward(buf, b, 8, z_coef=0.1, out=buf) is buf and torch.equal(buf, d)


def test_against_differences():
    """As for the norms: slopes of the float64 loss, counts fixed, along a direction."""
    logits, ids, _ = _inputs(40, 24, 3, "f32", seed=7)
    b = lx.router_balance(logits, ids, balance_coef=1.0, z_coef=0.1)
    d = f64(lx.router_balance_backward(logits, b, 3, balance_coef=1.0, z_coef=0.1))
    l, i = f64(logits), ids.cpu().numpy()
    v = np.random.default_rng(1).normal(size=l.shape)
    f = lambda x: block.router_balance(x, i, None, 1.0, 0.1)[0][0]  # noqa: E731
    slope = (f(l + 1e-5 * v) - f(l - 1e-5 * v)) / 2e-5
    assert abs(slope - (d * v).sum()) <= 1e-4 * np.abs(d * v).sum()


def test_refusals():
    l, ids = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    b = lx.router_balance(l, ids)
    for f in (lambda: lx.router_balance(l.cpu(), ids), lambda: lx.router_balance(l.double(), ids),
              lambda: lx.router_balance(l, ids.long()), lambda: lx.router_balance(l, ids[:3]),
              lambda: lx.router_balance(l, ids, mask=torch.ones(4, device="cuda")),
              lambda: lx.router_balance(l, ids, mask=torch.ones(3, dtype=torch.bool, device="cuda")),
              lambda: lx.router_balance_backward(l, b, 2, dloss=torch.ones(2, device="cuda")),
              lambda: lx.router_balance_backward(l[:3], b, 2)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: lx.router_balance(torch.zeros(4, 1025, device="cuda"), ids),
              lambda: lx.router_balance(l, torch.zeros(4, 33, dtype=torch.int32, device="cuda")),
              lambda: lx.router_balance_backward(l, b, 0),
              lambda: lx.router_balance(l, ids, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(lx.LxError) as e:
            f()
        assert e.value.status == lx.LX_ERR_ARG
