"""lx_distill_loss against the float64 definition (oracle/block.py)."""
import numpy as np
import pytest
import torch

from block_checks import F32, close, f64, gen
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
INF = float("inf")


def _inputs(T, V, K, dtype, tau=1.0, lse=False, labels=False, pad=0, seed=0):
    g = gen(seed)
    wide = (torch.randn(T, V + pad, generator=g) * 2.5).to(DT[dtype])
    t = wide[:, :V].float() + torch.randn(T, V, generator=g)
    top = torch.topk(t, min(K, V), dim=1)
    ids, val = top.indices.to(torch.int32), top.values
    if K > V:
        ids = torch.cat([ids, torch.full((T, K - V), -1, dtype=torch.int32)], 1)
        val = torch.cat([val, torch.zeros(T, K - V)], 1)
    return dict(logits=wide.cuda()[:, :V], ids=ids.cuda().contiguous(), top=val.cuda().contiguous(), tau=tau,
                lse=torch.logsumexp(t / tau, 1).cuda() if lse else None,
                labels=torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda() if labels else None,
                w=(torch.rand(T, generator=g) + 0.5).cuda())


def _call(v, a, b, **kw):
    return lx.distill_loss(v["logits"], v["ids"], v["top"], temperature=v["tau"], teacher_lse=v["lse"], kd_weight=a,
                           labels=v["labels"], ce_weight=b, row_weight=v["w"], **kw)


def _check(v, dtype, a=0.7, b=None):
    """The losses are differences of logarithms: each is within 1e-5 of the largest
    |logit|, temperature and weights included; gradients within 1e-5 of their terms'
    magnitudes, and of a thousandth of the row's weight: the exponent of a probability
    under a thousandth is rounded where it is large."""
    b = b if b is not None else 0.3 if v["labels"] is not None else 0.0
    loss, d = _call(v, a, b)
    alone, none = _call(v, a, b, want_grad=False)
    torch.cuda.synchronize()
    assert none is None and torch.equal(torch.nan_to_num(alone), torch.nan_to_num(loss))
    n = {k: f64(t) if torch.is_tensor(t) else t for k, t in v.items()}
    wl, wd, mag = block.distill(n["logits"], v["ids"].cpu().numpy(), n["top"], v["tau"], n["lse"], a,
                                None if v["labels"] is None else v["labels"].cpu().numpy(), b, n["w"], True)
    z = n["logits"][np.isfinite(n["logits"]) & (np.abs(n["logits"]) < 1e30)]
    scale = (np.abs(z).max() if z.size else 1.0) * max(1.0, v["tau"]) + 10.0
    close(loss, wl, False, scale, "loss")
    close(d, wd, dtype == "bf16", mag + 1e-3 * n["w"][:, None] * (a * v["tau"] + b), "dlogits")
    return loss, d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,K", [(1, 32000, 16), (3, 1, 1), (5, 7, 3), (9, 130, 64), (4, 5003, 50), (2, 50021, 1),
                                   (300, 1024, 8), (2, 70000, 256), (3, 2050, 1024), (2, 9, 20), (1, 300001, 5)])
@pytest.mark.parametrize("tau,lse,labels", [(1.0, False, True), (2.0, True, True), (0.5, False, False)])
def test_against_the_definition(T, V, K, dtype, tau, lse, labels):
    _check(_inputs(T, V, K, dtype, tau, lse, labels, seed=T + V + K), dtype)


@pytest.mark.parametrize("T", [150, 310, 1300])
def test_more_rows_than_the_grid(T):
    _check(_inputs(T, 515, 12, "bf16", 2.0, False, True, seed=T), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_slices_of_wider_rows(pad, dtype):
    v = _inputs(6, 4100, 20, dtype, pad=pad, labels=True, seed=pad)
    loss, d = _check(v, dtype)
    out = torch.empty(6, 4100 + 5, dtype=DT[dtype], device="cuda").fill_(7)
    l2, d2 = _call(v, 0.7, 0.3, dlogits=out[:, :4100])
    assert torch.equal(loss, l2) and torch.equal(d2, d) and (out[:, 4100:] == 7).all()
    l3, d3 = _call(v, 0.7, 0.3, dlogits=v["logits"])               # in place
    assert d3 is v["logits"] and torch.equal(loss, l3) and torch.equal(d3, d)


def test_entries_absent_repeated_and_infinite():
    v = _inputs(8, 900, 12, "f32", 1.5, False, True, seed=3)
    v["ids"][0] = -1                                   # a token without entries: cross-entropy alone
    v["ids"][1, 4:] = 900
    v["ids"][2, 1:5] = v["ids"][2, 0]                  # repeats add up
    v["ids"][3] = v["ids"][3, 0]
    v["top"][4, 1:] = -INF
    v["top"][5] = -INF                                 # every entry without weight
    v["labels"][6], v["labels"][7] = -100, 900
    v["labels"][2] = v["ids"][2, 0]                    # the label among the entries
    v["top"][1, 4:] = float("nan")                     # values of absent entries are not used
    _check(v, "f32")
    v["lse"] = torch.zeros(8, device="cuda") + 5
    _check(v, "f32")


def test_weight_zero_rows_are_not_read():
    v = _inputs(9, 3001, 7, "bf16", labels=True, seed=4)
    v["w"][::3] = 0
    want, dwant = _check(v, "bf16")
    v["logits"][::3] = float("nan")
    v["top"][::3] = float("nan")
    loss, d = _call(v, 0.7, 0.3)
    assert torch.equal(loss, want) and torch.equal(d, dwant) and (d[::3] == 0).all() and (loss[::3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_vocabulary(dtype):
    """-inf entries have no probability, the type's lowest value neither unless the
    whole row holds it; a row of nothing but -inf has nothing to learn."""
    v = _inputs(6, 1500, 9, dtype, 0.5, False, True, seed=5)
    lowest = torch.finfo(DT[dtype]).min
    keep = torch.zeros(1500, dtype=torch.bool, device="cuda")
    keep[v["ids"].long().reshape(-1)] = True
    keep[v["labels"].long()] = True
    v["logits"][:3, ~keep] = -INF
    v["logits"][3, ~keep] = lowest
    v["logits"][4] = -INF
    v["w"][4] = 1.0
    loss, d = _check(v, dtype)
    assert loss[4] == 0 and (d[4] == 0).all()
    v = _inputs(2, 1500, 9, dtype, 1.0, False, True, seed=6)
    v["logits"][0] = lowest                            # uniform
    loss, d = _call(v, 1.0, 0.0)
    q = torch.softmax(v["top"][0].double(), 0)
    want = (q * (q.log() + np.log(1500))).sum() * v["w"][0].double()
    assert abs(float(loss[0]) - float(want)) <= F32 * 10
    v["logits"][0] = -INF
    v["logits"][0, 3] = 1.0                            # an entry at -inf: the divergence is infinite
    v["ids"][0, 0] = 5
    loss, d = _call(v, 1.0, 0.0)
    assert loss[0] == INF and torch.isfinite(d[0]).all()


def test_nan_shows():
    v = _inputs(4, 700, 5, "f32", seed=7)
    v["logits"][1, 600] = float("nan")
    v["logits"][2, 8] = INF
    loss, d = _call(v, 1.0, 0.0)
    assert torch.isnan(loss[1]) and torch.isnan(d[1]).all() and torch.isnan(loss[2])
    assert torch.isfinite(loss[[0, 3]]).all() and torch.isfinite(d[[0, 3]]).all()


def test_large_offsets():
    """Rows that start past 2^31 elements."""
    V, T = 1 << 20, 2050
    base = torch.empty(T * V, dtype=torch.bfloat16, device="cuda")
    logits = base.view(T, V)
    v = _inputs(2, V, 4, "bf16", labels=True, seed=8)
    w = torch.zeros(T, device="cuda")
    w[0], w[T - 1] = v["w"][0], v["w"][1]
    logits[0], logits[T - 1] = v["logits"][0], v["logits"][1]
    rows = torch.tensor([0, T - 1], device="cuda")
    pick = lambda x, fill: torch.full((T, *x.shape[1:]), fill, dtype=x.dtype, device="cuda").index_copy(0, rows, x)  # noqa: E731
    want, dwant = _call(v, 0.7, 0.3)
    loss, d = lx.distill_loss(logits, pick(v["ids"], -1), pick(v["top"], 0.0), kd_weight=0.7,
                              labels=pick(v["labels"], -1), ce_weight=0.3, row_weight=w, dlogits=logits)
    close(loss[rows], f64(want), False, 20.0, "loss")
    close(d[rows], f64(dwant), True, what="dlogits")
    assert (d[1000] == 0).all()


def test_repeats_and_side_stream():
    v = _inputs(40, 32000, 32, "bf16", 2.0, labels=True, seed=9)
    want, dwant = _call(v, 0.7, 0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, d = _call(v, 0.7, 0.3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(loss, want) and torch.equal(d, dwant)


def test_against_differences():
    v = _inputs(5, 60, 6, "f32", 2.0, labels=True, seed=10)
    _, d = _call(v, 0.7, 0.3)
    n = {k: f64(t) if torch.is_tensor(t) else t for k, t in v.items()}
    f = lambda z: block.distill(z, v["ids"].cpu().numpy(), n["top"], 2.0, None, 0.7, v["labels"].cpu().numpy(), 0.3,  # noqa: E731
                                n["w"])[0].sum()
    x = np.random.default_rng(2).normal(size=n["logits"].shape)
    slope = (f(n["logits"] + 1e-5 * x) - f(n["logits"] - 1e-5 * x)) / 2e-5
    terms = f64(d) * x
    assert abs(slope - terms.sum()) <= 1e-4 * np.abs(terms).sum()


def test_no_tokens():
    z = torch.empty(0, 100, device="cuda")
    loss, d = lx.distill_loss(z, torch.empty(0, 4, dtype=torch.int32, device="cuda"),
                              torch.empty(0, 4, device="cuda"))
    assert loss.shape == (0,) and d.shape == (0, 100)


def test_refusals():
    z, ids, top = (torch.zeros(4, 50, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"),
                   torch.zeros(4, 2, device="cuda"))
    for f in (lambda: lx.distill_loss(z.cpu(), ids, top), lambda: lx.distill_loss(z.half(), ids, top),
              lambda: lx.distill_loss(z, ids.long(), top), lambda: lx.distill_loss(z, ids, top.bfloat16()),
              lambda: lx.distill_loss(z, ids, top[:, :1]), lambda: lx.distill_loss(z, ids[:3], top),
              lambda: lx.distill_loss(z, ids, top, row_weight=torch.ones(3, device="cuda")),
              lambda: lx.distill_loss(z, ids, top, dlogits=torch.zeros(4, 49, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    big = torch.zeros(4, 1025, device="cuda")
    wide = torch.zeros(4, 60, device="cuda")
    for f in (lambda: lx.distill_loss(z, ids, top, temperature=0.0), lambda: lx.distill_loss(z, ids, top, temperature=INF),
              lambda: lx.distill_loss(z, ids, top, temperature=float("nan")),
              lambda: lx.distill_loss(z, ids, top, ce_weight=0.5),
              lambda: lx.distill_loss(z, big.int(), big),
              lambda: lx.distill_loss(wide[:, :50], ids, top, dlogits=wide[:, 10:])):
        with pytest.raises(lx.LxError) as e:
            f()
        assert e.value.status == lx.LX_ERR_ARG
