"""lx_distill_loss where the work on a row's entries changes: few and many rows, one, four and
eight entries a thread, labels that are entries, entries that a row repeats.  Bounds as in
test_gpu_distill.py; the oracle skips rows of weight 0, so most rows have it."""
import pytest
import torch

from test_gpu_distill_shapes import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [70, 1216, 1217])
@pytest.mark.parametrize("V,K", [(200, 32), (1000, 33), (1000, 256), (1023, 257), (1030, 32), (1030, 129), (2049, 300),
                                 (4096, 256), (4104, 512), (8192, 513), (16384, 1024)])
def test_labels_and_repeats_among_entries(V, K, T):
    """Half of the rows have distinct entries, the others some in pairs; the labels are an
    entry of one place, of two, or none."""
    z, ids, top, lab, w, rows = _case(T, V, K, torch.bfloat16, on=12, seed=T + V + K)
    g = torch.Generator(device="cuda").manual_seed(K)
    if K <= V:
        ids = torch.rand(T, V, generator=g, device="cuda").topk(K, dim=1).indices.int()
    ids[::2, 1] = ids[::2, K - 1]
    ids[::4, 2] = ids[::4, K // 2]
    lab[rows[0::3]] = ids[rows[0::3], 1]
    lab[rows[1::3]] = ids[rows[1::3], 4]
    _check(z, ids.contiguous(), top, lab, w, rows)
    _check(z, ids.contiguous(), top, lab, w, rows, tau=2.0)


@pytest.mark.parametrize("V,K", [(1000, 256), (16384, 1024), (40000, 300)])
def test_every_entry_the_same(V, K):
    z, ids, top, lab, w, rows = _case(40, V, K, torch.float32, on=6, seed=V)
    ids[:] = ids[:, :1]
    lab[rows[::2]] = ids[rows[::2], 0]
    _check(z, ids, top, lab, w, rows)


@pytest.mark.parametrize("V", [5, 1000, 40000])
def test_first_and_last_column(V):
    """Ids 0 and V - 1, once and twice."""
    z, ids, top, lab, w, rows = _case(8, V, 4, torch.float32, on=6, seed=V)
    ids[:] = torch.tensor([[0, V - 1, 1, 2], [0, 0, V - 1, V - 1]], device="cuda", dtype=torch.int32).repeat(4, 1)
    lab[:] = torch.tensor([0, 0, V - 1, V - 1, 1, 1, 3, 3], device="cuda", dtype=torch.int32)
    w[:] = 1.0
    rows = torch.arange(8, device="cuda")
    _check(z, ids, top, lab, w, rows)
