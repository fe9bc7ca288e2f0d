"""lx_distill_loss on logits far from zero: a sum's reference is then off by more than the
exponents of fp32 hold, on either side, and at one temperature but not at the other."""
import numpy as np
import pytest
import torch

from block_checks import F32, close, f64, gen
from oracle import block
from test_gpu_distill import DT, _call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1001, 70000])
@pytest.mark.parametrize("tau", [1.0, 100.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("centres", [(300.0, 1e3, 5e3, 1e5, 1e6, 1e8), (1e9, 1.6e9, 3e9, 3.3e9, 5e9, 2e10, 1e20, 1e37)],
                         ids=["near", "far"])
def test_logits_far_from_zero(centres, V, tau, dtype, sign):
    """Each row's logits lie on three neighbouring numbers of the type.  Where a step is
    large the largest share the probability, at the temperature 100 the others may keep some."""
    g = gen(V)
    step = 2.0 ** (-7 if dtype == "bf16" else -23)
    rows = []
    for c in centres:
        c = 2.0 ** np.floor(np.log2(c)) * (1 + np.round((c / 2.0 ** np.floor(np.log2(c)) - 1) * 64) / 64)
        ulp = 2.0 ** np.floor(np.log2(c)) * step
        rows.append(sign * (c + ulp * torch.randint(0, 3, (V,), generator=g).double()))
    z = torch.stack(rows).to(DT[dtype])
    K, T = 5, len(centres)
    v = dict(logits=z.cuda(), ids=torch.randint(0, V, (T, K), generator=g, dtype=torch.int32).cuda(),
             top=torch.randn(T, K, generator=g).cuda(), tau=tau, lse=None,
             labels=torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda(),
             w=(torch.rand(T, generator=g) + 0.5).cuda())
    loss, d = _call(v, 0.7, 0.3)
    alone, _ = _call(v, 0.7, 0.3, want_grad=False)
    assert torch.equal(alone, loss)
    want, dwant, mag = block.distill(f64(v["logits"]), v["ids"].cpu().numpy(), f64(v["top"]), tau, None, 0.7,
                                     v["labels"].cpu().numpy(), 0.3, f64(v["w"]), True)
    # a loss is a difference of logarithms: within 1e-5 of its row's largest |logit|, of tau times it
    scale = np.abs(f64(z)).max(1) * tau + 10.0
    assert (np.abs(f64(loss) - want) <= F32 * scale).all()
    close(d, dwant, dtype == "bf16", mag + 1e-3 * f64(v["w"])[:, None] * (0.7 * tau + 0.3), "dlogits")
