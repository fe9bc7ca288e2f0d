"""Logits with a large common part: a row's dz adds up to nothing, however far from zero its logits are.

w has a column of ones, so dh there is the sum of the row's dz, 0 but for roundings.  What may be left of it, with
logits z of about 2000 and p the softmax:
  the row's log-sum-exp, in units of log 2 between 2048 and 4096, is rounded twice, half a step of 2^-12 each: 2^-12 ln 2
  of each exponential, and so of their sum (1);  the sum that it is taken of, 120 2^-24 (see test_gpu_head_loss);
  dz in bf16: 2^-8 of each p, independent, within 6 of their spread; the label's rounding is worked out;
  the product's sum over V terms, each partial sum below 1: (V / 16 + 16) 2^-23;  dh in bf16: 2^-8 of it.
Logits that were summed in another way than those of the log-sum-exp would be some 2^-23 of z for every 16 terms of H
apart, all to the same side: 0.01 and more here."""
import math

import pytest
import torch

from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
R = 2.0 ** -8


@pytest.mark.parametrize("T,V,H", [(300, 33003, 4096),     # all logits fit a piece's room and are kept
                                   (2100, 33003, 4096),    # they are formed again,
                                   (2100, 33003, 2568),    # in parts of which the last is ragged,
                                   (2100, 33003, 1032)])   # or short
def test_the_sum_of_dz(T, V, H):
    g = torch.Generator(device="cuda").manual_seed(11)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    h = (1 + 0.1 * randn(T, H)).to(BF)
    w = (2000 / H + randn(V, H) / H ** 0.5).to(BF)
    w[:, 0] = 1
    labels = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    got = lx.head_loss(h, w, labels, want_dw=False)
    rows = torch.arange(0, T, 9, device="cuda")
    p = torch.softmax(h[rows].double() @ w.double().t(), 1)
    own = p.gather(1, labels[rows].long()[:, None])[:, 0] - 1
    label = (own.to(BF).double() - own).abs() + R * (2.0 ** -12 + 2.0 ** -16)
    spread = 6 * R * p.pow(2).sum(1).sqrt()
    bound = 2.0 ** -12 * math.log(2) + 120 * 2.0 ** -24 + spread + label + (V / 16 + 16) * 2.0 ** -23
    left = got.dh[rows, 0].double().abs()
    assert float((left - bound * (1 + R)).max()) <= 0, (float(left.max()), float(bound.max()))
