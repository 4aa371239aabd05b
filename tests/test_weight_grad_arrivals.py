"""The weight gradient's barriers where the products' arrivals, which go to both CTAs of a pair, land
in any order once the products are done (test_weight_grad_barriers has them in the order of the
stages): a team may meet a stage only when it has seen every phase of that stage's barrier."""
import os
import random
import re

import pytest

from paper_2110_04175_gb300 import build as rs_build

from .test_weight_grad_barriers import Pair


class LateArrivals(Pair):
    """asks: whether the codes of a stage are copied only when the role that copies dy has found the
    stage that was in its place free, and a team waits for its codes first."""

    def __init__(self, *args, asks):
        super().__init__(*args)
        self.asks, self.sent, self.passed = asks, [], [0, 0]

    def dy_copies(self, r):
        for i in range(sum(self.tiles)):
            s, parity = self.stage(i)
            while not self.freed[r][s].passed(parity ^ 1):
                yield
            assert self.consumed >= i - self.stages, "dy is copied while its stage is in use"
            self.passed[r] = i + 1
            self.full[r][s].expect()
            self.copies.append((self.full[r][s], self.holds[r][s], self.team, i))
            yield

    def code_copies(self, r):
        for i in range(sum(self.tiles)):
            f = i % self.ahead
            while not self.used[r][f].passed(i // self.ahead & 1 ^ 1):
                yield
            while self.asks and self.passed[r] < i - self.stages + 1:
                yield
            self.fetched[r][f].expect()
            self.codes[r][f] = None
            self.copies.append((self.fetched[r][f], self.codes[r], f, i))
            yield

    def writer(self, r, team, member):
        if not self.asks:
            yield from super().writer(r, team, member)
            return
        for i in range(team, sum(self.tiles), self.teams):
            (s, parity), f = self.stage(i), i % self.ahead
            while not self.fetched[r][f].passed(i // self.ahead & 1):
                yield
            while not self.freed[r][s].passed(parity ^ 1):
                yield
            assert self.consumed >= i - self.stages, "a stage is written while it is in use"
            assert self.codes[r][f] == i, "other codes"
            yield
            self.holds[r][s][member] = i
            self.full[r][s].arrive()
            self.used[r][f].arrive()
            yield

    def finish(self):
        if self.products and self.products[0][0] != "product":
            what, at, *group = self.products.pop(0)
            if what == "summed":
                self.sums[at] = ("whole", group[0])
            for r in (0, 1):
                self.sent.append((self.freed if what == "freed" else self.summed)[r][at])
        else:
            super().finish()

    def land(self):
        super().land()
        for _ in range(self.rng.randint(0, len(self.sent))):
            self.sent.pop(self.rng.randrange(len(self.sent))).arrive()


def _runs(stages, ahead, teams, group, seeds, asks):
    for seed in range(seeds):
        rng = random.Random(seed)
        tiles = [rng.choice([0, 1, 2, 3, 5, 8, 9, 17]) for _ in range(rng.randint(1, 3))]
        LateArrivals(stages, ahead, teams, group, tiles, rng, asks=asks).run()


def _instances():
    """(stages, stages of codes, teams, stages of a group) of the kernel's six instances, by the rule and
    the constants of its source."""
    text = open(os.path.join(rs_build.CSRC, "weight_grad.cu")).read()

    def constant(name):
        return int(re.search(rf"\b{name} = (\d+)\b", text).group(1))

    m, depth, teams_most, adders = (constant(k) for k in ("kM", "kDepth", "kTeams", "kAdders"))
    panel, turn = depth * 128, 32 * constant("kTurnRow") * 4 + 128 * 4
    room = 232448 - 1024 - 512 - adders * turn
    for terms, group in ((1, 8), (2, 4), (3, 3)):
        for wide in (256, 128):
            stage, codes = terms * m // 64 * panel + wide // 2 // 64 * panel, wide // 2 * depth
            stages = min((room - 4 * codes) // stage, 4)
            yield stages, min((room - stages * stage) // codes, 8), min(stages, teams_most), group


def test_instances():
    """What the rule gives: whoever changes it changes what is modelled here and there."""
    assert list(_instances()) == [(4, 7, 3, 8), (4, 8, 3, 8), (3, 5, 3, 4), (4, 6, 3, 4), (2, 7, 2, 3), (3, 4, 3, 3)]


@pytest.mark.parametrize("stages,ahead,teams,group", list(_instances()))
def test_arrivals_in_any_order(stages, ahead, teams, group):
    _runs(stages, ahead, teams, group, seeds=20, asks=teams < stages)


def test_the_model_sees_a_team_that_skips_phases():
    """Three teams on four stages, without asking: a wait passes two phases early."""
    with pytest.raises(AssertionError, match="in use|arrivals|other codes|not whole|changed"):
        _runs(4, 7, 3, 8, seeds=30, asks=False)


def test_the_model_sees_too_few_stages_of_codes():
    """With five of them a stage's place had other codes that this team has not seen."""
    with pytest.raises(AssertionError, match="in use|arrivals|other codes|not whole|changed|nothing moves"):
        _runs(4, 5, 3, 8, seeds=200, asks=True)


def test_the_kernel_asks():
    """The count, the wait for it and the order of a team's waits, in the source."""
    text = open(os.path.join(rs_build.CSRC, "weight_grad.cu")).read()
    dy, rest = text.split("} else if (warp == kIssuer + 2")
    codes, teams = rest.split("using R = Recall")
    dy, codes, teams = (re.sub(r"\s+", " ", part) for part in (dy, codes, teams))
    assert ("(ok = barrier_wait(freed(s), (i / kCount & 1) ^ 1))) break; if (S::kAsk) count_store(passed, i + 1); "
            "barrier_expect(full(s), S::kLeft);") in dy
    assert ("if (S::kAsk && !(ok = count_wait(passed, i - kCount + 1))) break; "
            "barrier_expect(fetched(f), S::kCodes);") in codes
    assert ("if (S::kAsk && !(ok = barrier_wait_warp(fetched(f), i / S::kAhead & 1))) break; "
            "if (!(ok = barrier_wait_warp(freed(s), (i / kCount & 1) ^ 1))) break;") in teams
