"""The weight gradient's CTAs end only when nothing is on its way to their barriers: the products'
arrivals go to both CTAs of a pair and may land late (test_weight_grad_arrivals has the model)."""
import os
import random
import re

import pytest

from paper_2110_04175_gb300 import build as rs_build

from .test_weight_grad_arrivals import LateArrivals, _instances


class Ending(LateArrivals):
    """waits: whether the role that copies dy waits for the last stages to be free before its CTA ends."""

    def __init__(self, *args, asks, waits):
        super().__init__(*args, asks=asks)
        self.waits = waits

    def dy_copies(self, r):
        yield from super().dy_copies(r)
        total = sum(self.tiles)
        for i in range(max(0, total - self.stages), total if self.waits else 0):
            s, parity = self.stage(i)
            while not self.freed[r][s].passed(parity):
                yield

    def land(self):
        late, self.sent = self.sent, []
        super().land()  # the copies
        self.sent = late
        for _ in range(self.rng.randint(0, 1 + len(late)) - 1):
            self.sent.pop(self.rng.randrange(len(self.sent))).arrive()


def _runs(waits, stages, ahead, teams, group, seeds=10):
    for seed in range(seeds):
        rng = random.Random(seed)
        tiles = [rng.choice([0, 1, 2, 3, 5, 9]) for _ in range(rng.randint(1, 3))]
        pair = Ending(stages, ahead, teams, group, tiles, rng, asks=teams < stages, waits=waits)
        pair.run()
        assert not pair.sent, "a CTA has ended before an arrival at its barriers"


@pytest.mark.parametrize("stages,ahead,teams,group", list(_instances()))
def test_no_arrival_after_the_end(stages, ahead, teams, group):
    _runs(True, stages, ahead, teams, group)


def test_the_model_sees_a_missing_wait():
    with pytest.raises(AssertionError, match="has ended"):
        _runs(False, 4, 7, 3, 8, seeds=200)


def test_the_kernel_waits_for_the_last_stages():
    """The copying role's tail, in the source: for what it copied, and for the stages to be free."""
    text = open(os.path.join(rs_build.CSRC, "weight_grad.cu")).read()
    tail = re.search(r"for \(int j = max\(0, i - kCount\); j < i; \+\+j\)(.*?)break;", text, re.S).group(1)
    assert "barrier_wait(full(j % kCount), j / kCount & 1)" in tail
    assert "barrier_wait(freed(j % kCount), j / kCount & 1)" in tail
