"""head_loss where few rows of a large vocabulary are kept: against the definition (bounds as in test_gpu_head_loss),
in a workspace of just the size asked for, whose surroundings stay as they were."""
import pytest
import torch

from paper_2608_07814_gb300 import lx
from test_gpu_head_loss import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,H,masked", [(1, 300001, 64, 0), (5, 270000, 40, 0.4), (33, 280003, 32, 0.2), (65, 100003, 72, 0),
                                          (96, 30011, 136, 0.1), (224, 70001, 40, 0.5)])
def test_few_rows(T, V, H, masked):
    h, w, labels, weight = _case(T, V, H, masked, seed=3)
    labels[0] = V - 1
    n = lx.head_loss_workspace_bytes(T, V, H)
    room = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    at = -room.data_ptr() % 256 + 2048
    got = lx.head_loss(h, w, labels, row_weight=weight, workspace=room[at:at + n])
    _check(got, h, w, labels, weight)
    assert bool((room[:at] == 0xA5).all()) and bool((room[at + n:] == 0xA5).all())
    again = lx.head_loss(h, w, labels, row_weight=weight)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
