"""lx_residual_norm on rows of a few bytes: a 16-byte block holds several rows, and those at
both ends of the array share it with what lies around.  Bounds as in
test_gpu_residual_norm.py."""
import pytest
import torch

import test_gpu_residual_norm as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1, 5, 7])
@pytest.mark.parametrize("H", range(1, 9))
@pytest.mark.parametrize("T", [1, 2, 3, 5, 9, 17, 40])
def test_rows_that_share_blocks(T, H, off, dtype):
    v, dr, dh = base._inputs(T, H, dtype, "full", seed=T + H)

    def wrap(t):  # contiguous rows at any address, NaN around them
        flat = torch.full((T * H + 16,), float("nan"), dtype=t.dtype, device="cuda")
        flat[off:off + T * H] = t.reshape(-1)
        return flat[off:off + T * H].view(T, H)

    v = {k: wrap(t) if k in ("r", "y", "gate") else t for k, t in v.items()}
    base._check(v, wrap(dr), wrap(dh), dtype)
