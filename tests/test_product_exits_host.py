"""How a pair of CTAs of the large products ends after a wait that gave up, as a model (no GPU).

Each CTA's producer asks for its half of a block of K, whose bytes the even CTA's barriers count; the even CTA's
issuer multiplies what has landed and commits to both CTAs' barriers.  A role may stop at any of its waits, so one
CTA may have asked for blocks that the other has not.  Before shared memory and TMEM go away, one thread of each CTA
waits for all that is on its way, by the roles' counts alone (settle in lx_product.cuh).  The test runs the same
steps under random schedules: the waits end, none before the last bytes and commits are there, and each barrier has
at most one phase open.  The even CTA's count alone, by which the kernel once went, leaves copies in flight.  It
shares no code with the library: it pins the accounting."""
import os
import random
import re

import pytest

SOURCE = open(os.path.join(os.path.dirname(__file__), "..", "paper_2608_07814_gb300", "csrc", "lx_product.cuh")).read()
STAGES = sorted({int(n) for n in re.findall(
    r"\d", re.search(r"int STAGES = MODE == STATS \? (\d : DEEP \? \d : \d);", SOURCE).group(1))})


class Barrier:
    """An mbarrier of one arrival: its phase ends once it has arrived and no byte is missing."""

    def __init__(self):
        self.phase, self.arrived, self.halves = 0, False, 0

    def turn(self):
        if self.arrived and self.halves == 0:
            self.phase, self.arrived = self.phase + 1, False

    def arrive(self, halves=0):  # arrive.expect_tx, or a commit
        assert not self.arrived, "two phases open"
        self.halves, self.arrived = self.halves + halves, True
        self.turn()

    def complete(self):  # a half that lands, or complete_tx
        self.halves -= 1
        self.turn()

    def past(self, parity):  # try_wait.parity
        return (self.phase - 1) & 1 == parity


def _run(rng, S, blocks, part):
    """A pair up to where all roles have stopped.  Returns its state."""
    full = [Barrier() for _ in range(S)]
    empty, tfull = [[Barrier() for _ in range(S)] for _ in range(2)], [[Barrier() for _ in range(2)] for _ in range(2)]
    asked, made, sums = [0, 0], 0, 0
    flying = []                                   # what has yet to arrive
    quits = [rng.randrange(1, 6 * blocks) for _ in range(3)]
    if rng.random() < 0.3:
        quits[rng.randrange(3)] = 10 ** 9
    stopped = [False] * 3
    read = [0, 0]                                 # sums that each CTA's epilogue has taken
    for step in range(10 ** 5):
        if all(stopped):
            break
        if flying and rng.random() < 0.35:
            flying.pop(rng.randrange(len(flying)))()
            continue
        for c in range(2):                        # the epilogues, until they give up with their CTA
            if read[c] < sums and tfull[c][read[c] & 1].past((read[c] >> 1) & 1) and not stopped[c]:
                read[c] += 1
        role = rng.randrange(3)
        if stopped[role]:
            continue
        if step >= quits[role]:
            stopped[role] = True
        elif role < 2:
            j = asked[role]
            if j == blocks:
                stopped[role] = True
            elif empty[role][j % S].past(((j // S) & 1) ^ 1):
                if role == 0:
                    full[j % S].arrive(2)
                flying.append(full[j % S].complete)
                asked[role] += 1
            elif stopped[2]:
                stopped[role] = True              # it waits for nothing that comes
        elif made == blocks:
            stopped[2] = True
        elif made % part == 0 and sums - min(read) >= 2:
            stopped[2] = stopped[0] and stopped[1]
        elif full[made % S].past((made // S) & 1):
            flying += [empty[0][made % S].arrive, empty[1][made % S].arrive]
            made += 1
            if made % part == 0 or made == blocks:
                flying += [tfull[0][sums & 1].arrive, tfull[1][sums & 1].arrive]
                sums += 1
        elif stopped[0] and stopped[1] and not any(f.__name__ == "complete" for f in flying):
            stopped[2] = True
    else:
        raise AssertionError("the roles did not stop")
    return full, empty, tfull, asked, made, sums, flying


def _waits(S, full, empty, tfull, most, made, sums):
    waits = [(full[j % S], (j // S) & 1) for j in range(max(0, most - S), most)]
    for c in range(2):
        waits += [(empty[c][j % S], (j // S) & 1) for j in range(max(0, made - S), made)]
        waits += [(tfull[c][j & 1], (j >> 1) & 1) for j in range(max(0, sums - 2), sums)]
    return waits


def _over(waits, rng, flying):
    """Lets what flies arrive one by one; what still flies when the last of the waits ends."""
    while not all(b.past(p) for b, p in waits):
        if not flying:
            raise AssertionError("a wait does not end")
        flying.pop(rng.randrange(len(flying)))()
    return flying


def test_the_stages_are_found():
    assert STAGES == [5, 6]


@pytest.mark.parametrize("S", STAGES)
def test_all_that_is_on_its_way_arrives_first(S):
    rng, uneven = random.Random(S), 0
    for _ in range(3000):
        full, empty, tfull, asked, made, sums, flying = _run(rng, S, rng.randrange(1, 60), rng.choice((3, 16, 10 ** 9)))
        even, odd, most = asked[0], asked[1], max(asked)
        assert most - min(asked) <= S
        uneven += even != odd
        for j in range(max(0, most - S), most):
            if j >= even:
                full[j % S].arrive(1)
            elif j >= odd:
                full[j % S].complete()
        assert not _over(_waits(S, full, empty, tfull, most, made, sums), rng, flying)
    assert uneven > 300


@pytest.mark.parametrize("S", STAGES)
def test_the_even_count_alone_does_not_do(S):
    rng, left, endless = random.Random(S), 0, 0
    for _ in range(1000):
        full, empty, tfull, asked, made, sums, flying = _run(rng, S, rng.randrange(1, 60), 16)
        try:
            left += bool(_over(_waits(S, full, empty, tfull, asked[0], made, sums), rng, flying))
        except AssertionError:
            endless += 1
    assert left and endless
