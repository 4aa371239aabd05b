"""The phases of the bulk copies' barriers, modelled on the CPU: a group that works through rows (or a CTA through tiles)
in a ring of stages waits for each row's own copy, whatever the order in which copies land, and asks for no stage that is
still read.  (A parity wait cannot tell a phase from the one two before it: one taken from the wrong row passes early.)"""
import random

import pytest


class Barrier:
    """mbarrier with one expected arrival: the phase ends when the arrival and its bytes are there."""

    def __init__(self):
        self.phase, self.arrived, self.bytes = 0, False, 0

    def expect(self, size):
        assert not self.arrived
        self.arrived = True
        self.bytes += size
        self._end()

    def land(self, size):
        self.bytes -= size
        self._end()

    def _end(self):
        if self.arrived and self.bytes == 0:
            self.phase, self.arrived = self.phase + 1, False

    def passed(self, parity):
        return (self.phase - 1) % 2 == parity if self.phase else parity == 1


def _ring(rows, stages, refill, r):
    """`refill(i)`: (row to ask for, its stage) once row i's readers are known to be done, or None."""
    bars, holds, flying = [Barrier() for _ in range(stages)], [None] * stages, []

    def ask(row, stage):
        assert (stage, "flying") not in [(s, "flying") for _, s in flying]
        bars[stage].expect(1)
        flying.append((row, stage))

    def land():
        row, stage = flying.pop(r.randrange(len(flying)))
        holds[stage] = row
        bars[stage].land(1)

    for i in range(min(stages, rows)):
        ask(i, i)
    for i in range(rows):
        while flying and (r.random() < 0.5 or not bars[i % stages].passed(i // stages & 1)):
            land()
        assert bars[i % stages].passed(i // stages & 1)
        assert holds[i % stages] == i, "a row that was not there yet"
        more = refill(i)
        if more is not None and more[0] < rows:
            ask(*more)
    assert not flying


@pytest.mark.parametrize("rows", [0, 1, 2, 3, 4, 5, 8, 30])
def test_every_wait_is_for_its_own_row(rows):
    r = random.Random(rows)
    for _ in range(200):
        _ring(rows, 1, lambda i: (i + 1, 0), r)  # block norm, forward: once h is in registers
        _ring(rows, 2, lambda i: (i + 1, (i + 1) % 2) if i > 0 else None, r)  # backward: the row before is done with
        _ring(rows, 3, lambda i: (i + 2, (i - 1) % 3) if i > 0 else None, r)  # recurrence: tiles, likewise


def test_the_model_sees_a_parity_of_the_wrong_row():
    with pytest.raises(AssertionError):
        bars = Barrier()
        bars.expect(1)
        bars.land(1)
        bars.expect(1)  # row 1 in a ring of one stage, waited for with row 0's parity
        assert not bars.passed(0)
