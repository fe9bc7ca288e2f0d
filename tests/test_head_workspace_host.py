"""What lx_head_loss asks for as a workspace, against what include/lx.h says (no GPU)."""
import pytest

from paper_2608_07814_gb300 import lx

MIB = 1 << 20


def _up(v, n):
    return (v + n - 1) // n * n


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 200, 257, 512, 513, 1000, 4096, 70000])
@pytest.mark.parametrize("V,H", [(7, 8), (1000, 512), (50021, 2560), (131072, 2048), (200000, 64), (1 << 21, 1024)])
def test_the_header_s_terms_hold_it(T, V, H):
    rows, cols = _up(T, 256), _up(V, 256)
    sums = 8 * rows * _up(V, 128) // 128
    kept = 4 * _up(T, 32) * cols
    if kept <= 256 * MIB:
        logits = 2 * kept
    else:
        logits = min(2 * rows * cols, max(256 * MIB, 2 * rows * 256))
    # hidden states (twice), and dh in fp32: up to 16 ranges of the vocabulary side by side, on 76 tiles together
    hidden = rows * H * 2 * 2
    dh = max(4 * rows * _up(H, 32), 76 * 4 * 256 * 256)
    room = sums + logits + hidden + dh + 24 * rows + 16 * 256
    assert lx.head_loss_workspace_bytes(T, V, H) <= room
    assert lx.head_loss_workspace_bytes(T, V, H, False, False) <= sums + hidden + 24 * rows + 16 * 256


def test_few_tokens_of_a_large_vocabulary():
    """Kept logits and dz take the rows' room, not that of whole tiles."""
    assert lx.head_loss_workspace_bytes(1, 131072, 2048) < 64 * MIB
    assert lx.head_loss_workspace_bytes(8, 200000, 2048) < 96 * MIB
    assert lx.head_loss_workspace_bytes(64, 131072, 2048) <= lx.head_loss_workspace_bytes(128, 131072, 2048)
