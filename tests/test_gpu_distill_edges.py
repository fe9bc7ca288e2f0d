"""lx_distill_loss on both sides of the sizes where its form changes: rows in registers, CTAs of
128, 256 and 512 threads, one, two, four and eight CTAs a row, rows that are not held.  The sizes
come from the constants of the source.  Bounds as in test_gpu_distill_shapes.py."""
import os
import re

import pytest
import torch

from test_gpu_distill_shapes import _case, _check

pytestmark = pytest.mark.gpu

SOURCE = open(os.path.join(os.path.dirname(__file__), "..", "paper_2608_07814_gb300", "csrc", "lx_distill.cu")).read()


def _const(name):
    return int(re.search(r"constexpr int %s = (\d+)" % name, SOURCE).group(1))


SMEM, U, BUFS, TEACHERS, SHORT_P, CTAS = (_const(n) for n in ("SMEM", "U", "BUFS", "MAX_TEACHERS", "SHORT_P",
                                                              "MAX_CLUSTER"))
AHEAD = int(re.search(r"ahead_of\(bool grad\) \{ return grad \? (\d+)", SOURCE).group(1))


def _holds(threads, K):
    """Bytes of a row's part that a CTA of that many data threads holds."""
    table = 32
    while table < 2 * K:
        table *= 2
    entries = (4 * BUFS * (K + 1) + TEACHERS * table + 3) // 4 * 16
    places = (SMEM * threads // 512 - entries) // (16 * threads)
    return max(0, (places - AHEAD - U) // U * U * 16 * threads)


def _limits(K, es):
    """Columns of the widest row of each form."""
    short = SHORT_P * 32 * 8 * 16
    held = {_holds(t, K) for t in (128, 256, 512)} | {_holds(512, K) * c for c in (2, 4, CTAS)}
    return sorted({b // es for b in held if b > short} | {short // es})


def _cases():
    for K in (1, 64, 300):
        for es in (2, 4):
            for at in _limits(K, es):
                if K == 64 or at * es <= 131072:
                    yield from ((K, es, at + d) for d in (-1, 0, 1, 16 // es))


def test_the_limits_are_apart():
    """With 64 entries: the registers, 256 threads, and 1, 2, 4 and 8 CTAs of 512."""
    assert _limits(64, 2) == [16384, 32768, 65536, 131072, 262144, 524288]
    assert _limits(64, 4) == [8192, 16384, 32768, 65536, 131072, 262144]


@pytest.mark.parametrize("K,es,V", list(_cases()))
def test_both_sides(K, es, V):
    _check(*_case(160, V, K, torch.bfloat16 if es == 2 else torch.float32, on=2, seed=V), tau=2.0 if es == 4 else 1.0)


@pytest.mark.parametrize("V", [32768, 65536, 65537])
def test_without_gradient(V):
    z, ids, top, lab, w, _ = _case(160, V, 64, torch.bfloat16, seed=V)
    loss, _ = _call(z, ids, top, lab, w, True)
    alone, none = _call(z, ids, top, lab, w, False)
    assert none is None and torch.equal(loss, alone)


def _call(z, ids, top, lab, w, grad):
    from paper_2608_07814_gb300 import lx
    return lx.distill_loss(z, ids, top, kd_weight=0.7, labels=lab, ce_weight=0.3, row_weight=w, want_grad=grad)
