"""Losses of lx_distill_loss on logits far from zero.  What the logits have in common cancels:
the references are exact, so a loss is off by the rounding of differences alone.  In each of the
two terms those are the spread of the row's logits over the temperature, and logarithms of sums
below 2^64 (below 45): 1e-5 of the spread and of 10 holds their roundings of 2^-24."""
import numpy as np
import pytest
import torch

from block_checks import F32, f64, gen
from oracle import block
from test_gpu_distill import DT, _call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1001, 70000])
@pytest.mark.parametrize("tau", [1.0, 2.0, 100.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_common_part_cancels(V, tau, dtype, sign):
    g = gen(V + 1)
    # powers of two on both sides of the references' reach, at temperature 1 and 100
    powers = [8, 10, 17, 23, 28, 29, 30, 31, 32, 33, 35, 37, 38, 60, 100, 120]
    step = 2.0 ** (-7 if dtype == "bf16" else -23)
    z = torch.stack([sign * 2.0 ** p * (1 + step * torch.randint(0, 3, (V,), generator=g).double()) for p in powers])
    K, T = 5, len(powers)
    v = dict(logits=z.to(DT[dtype]).cuda(), ids=torch.randint(0, V, (T, K), generator=g, dtype=torch.int32).cuda(),
             top=torch.randn(T, K, generator=g).cuda(), tau=tau, lse=None,
             labels=torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda(),
             w=(torch.rand(T, generator=g) + 0.5).cuda())
    a, b = 0.7, 0.3
    loss, _ = _call(v, a, b)
    want, _ = block.distill(f64(v["logits"]), v["ids"].cpu().numpy(), f64(v["top"]), tau, None, a,
                            v["labels"].cpu().numpy(), b, f64(v["w"]))
    spread = f64(z).max(1) - f64(z).min(1)
    bound = F32 * f64(v["w"]) * (a * tau ** 2 * (spread / tau + 10) + b * (spread + 10))
    off = np.abs(f64(loss) - want)
    assert (off <= bound).all(), (off / bound).max()
