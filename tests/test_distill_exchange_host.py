"""The exchange of a row's sums between the CTAs of a cluster (lx_distill_loss), as a model.

Warps send 16 bytes for a row to a barrier of every CTA and go on; what they sent may land at
any later time.  A warp may give up at a wait; then the CTAs run to their ends, and before its
shared memory goes each CTA waits until all that was sent to it has landed.  The kernel works
out what is missing from the warps' counts alone (await_sent); this test runs the same steps
under random schedules and shows that at most one phase of a barrier is open then, that the wait
ends, and that it does not end before the last byte.  It shares no code with the library: it pins
the accounting."""
import os
import random
import re

import pytest

SOURCE = open(os.path.join(os.path.dirname(__file__), "..", "paper_2608_07814_gb300", "csrc", "lx_distill.cu")).read()
SENDS = int(re.search(r"constexpr int SENDS = (\d+)", SOURCE).group(1))


class Barrier:
    """An mbarrier of one arrival: its phase ends once it has arrived and no byte is missing."""

    def __init__(self):
        self.phase, self.arrived, self.bytes = 0, False, 0

    def turn(self):
        if self.arrived and self.bytes == 0:
            self.phase, self.arrived = self.phase + 1, False

    def expect(self, n):  # arrive.expect_tx
        assert not self.arrived, "two phases open"
        self.bytes, self.arrived = self.bytes + n, True
        self.turn()

    def complete(self, n):  # bytes that land, or complete_tx
        self.bytes -= n
        self.turn()

    def past(self, parity):  # try_wait.parity
        return (self.phase - 1) & 1 == parity


def _run(rng, cols, nw, rows, unmet):
    bars = [[Barrier() for _ in range(SENDS)] for _ in range(cols)]
    sent = [[[0] * nw for _ in range(SENDS)] for _ in range(cols)]
    flying = []                                   # (CTA, barrier) of 16 bytes
    at = {(c, w): (0, 0) for c in range(cols) for w in range(nw)}  # rows sent for, rows received
    lost, gave_up = set(), [False] * cols
    quit_at = rng.randrange(200 * cols * nw)
    for step in range(10 ** 6):
        live = [k for k in at if k not in lost and at[k][1] < rows]
        if not live:
            break
        if flying and rng.random() < 0.4:
            c, b = flying.pop(rng.randrange(len(flying)))
            bars[c][b].complete(16)
            continue
        c, w = rng.choice(live)
        s, r = at[c, w]
        b = s % SENDS
        if s < rows and s - r < 2 and rng.random() < 0.6:   # row s after row s - 2
            if w == 0 and not unmet:
                bars[c][b].expect(cols * nw * 16)
            sent[c][b][w] += 1
            flying += [(to, b) for to in range(cols)]
            at[c, w] = s + 1, r
        elif r < s:                               # a wait: met, given up, or still on
            if gave_up[c] or step > quit_at:
                lost.add((c, w))
                for to in range(cols):
                    if to == c or rng.random() < 0.7:  # the others may learn of it later
                        gave_up[to] = True
            elif bars[c][r % SENDS].past(r // SENDS & 1):
                at[c, w] = s, r + 1
    return bars, sent, flying


@pytest.mark.parametrize("unmet", [False, True])
@pytest.mark.parametrize("cols,nw", [(2, 4), (4, 2), (8, 3), (3, 1)])
def test_the_wait_ends_with_the_last_byte(cols, nw, unmet):
    open_phases = 0
    for seed in range(400):
        rng = random.Random(1000 * cols + seed)
        bars, sent, flying = _run(rng, cols, nw, rng.randrange(1, 30), unmet)
        for c in range(cols):
            for b in range(SENDS):
                bar, told = bars[c][b], 0 if unmet else sent[c][b][0]
                assert told - bar.phase in (0, 1)
                more = sum(sum(sent[o][b]) for o in range(cols)) - told * cols * nw
                if more < 0:
                    bar.complete(-16 * more)
                if more > 0:
                    bar.expect(16 * more)
                    told += 1
                left = flying.count((c, b))
                open_phases += left > 0
                for _ in range(left):
                    assert not bar.past((told - 1) & 1)
                    bar.complete(16)
                assert bar.past((told - 1) & 1) and bar.bytes == 0
    assert open_phases > 50  # schedules that the wait is for


def test_the_kernel_waits_for_what_was_sent():
    """Between a cluster's last barriers stands the wait for the sends, not a time."""
    tail = SOURCE[SOURCE.index("asm volatile(\"cp.async.wait_group 0;\""):]
    tail = tail[:tail.index("__global__")]
    assert "await_sent(" in tail and "clock64" not in tail
