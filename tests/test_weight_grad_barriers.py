"""The weight gradient's barriers, modelled: the roles of a pair of CTAs (weight_grad.cu) as
coroutines over mbarriers that count arrivals, bytes and phases, stepped in random order.  Copies
land in any order, products in theirs.  The model fails where a stage is written while it is in use,
where anything is read before it is there, where a barrier gets more arrivals than it counts, and
where nothing moves any more."""
import random

import pytest


class Barrier:
    def __init__(self, arrivals):
        self.arrivals = self.pending = arrivals
        self.bytes = self.phase = 0

    def _settle(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase += 1
            self.pending = self.arrivals

    def arrive(self):
        self.pending -= 1
        assert self.pending >= 0, "more arrivals than the phase counts"
        self._settle()

    def expect(self):
        self.bytes += 1
        self.arrive()

    def land(self):
        self.bytes -= 1
        self._settle()

    def passed(self, parity):  # as mbarrier.try_wait.parity: it cannot tell phases two apart
        return (self.phase & 1) != parity


class Pair:
    """stages, ahead: of operands and of codes; teams of `team` warps; groups of `group` stages per
    accumulator; tiles: their numbers of stages."""

    def __init__(self, stages, ahead, teams, group, tiles, rng, team=2, adders=2):
        self.stages, self.ahead, self.teams, self.group, self.tiles, self.rng = stages, ahead, teams, group, tiles, rng
        self.team, self.adders = team, adders
        two = (0, 1)
        self.full = [[Barrier(team + 1 + (r == 0)) for _ in range(stages)] for r in two]
        self.freed = [[Barrier(1) for _ in range(stages)] for _ in two]
        self.summed = [[Barrier(1) for _ in two] for _ in two]
        self.read = [[Barrier(adders) for _ in two] for _ in two]
        self.fetched = [[Barrier(1) for _ in range(ahead)] for _ in two]
        self.used = [[Barrier(team) for _ in range(ahead)] for _ in two]
        self.holds = [[[None] * (team + 1) for _ in range(stages)] for _ in two]  # by writer, dy last
        self.codes = [[None] * ahead for _ in two]
        self.sums, self.reads = [None, None], [[0, 0], [0, 0]]
        self.consumed = -1  # the last stage whose products are done
        self.copies, self.products = [], []

    def stage(self, i):
        return i % self.stages, i // self.stages & 1

    def writer(self, r, team, member):
        base = 0
        for count in self.tiles:
            for n in range((team + self.teams - base % self.teams) % self.teams, count, self.teams):
                i = base + n
                (s, parity), f = self.stage(i), i % self.ahead
                while not self.freed[r][s].passed(parity ^ 1):
                    yield
                assert self.consumed >= i - self.stages, "a stage is written while it is in use"
                while not self.fetched[r][f].passed(i // self.ahead & 1):
                    yield
                assert self.codes[r][f] == i, "other codes"
                yield
                self.holds[r][s][member] = i
                self.full[r][s].arrive()
                self.used[r][f].arrive()
                yield
            base += count

    def dy_copies(self, r):
        for i in range(sum(self.tiles)):
            s, parity = self.stage(i)
            while not self.freed[r][s].passed(parity ^ 1):
                yield
            assert self.consumed >= i - self.stages, "dy is copied while its stage is in use"
            self.full[r][s].expect()
            self.copies.append((self.full[r][s], self.holds[r][s], self.team, i))
            yield

    def code_copies(self, r):
        for i in range(sum(self.tiles)):
            f = i % self.ahead
            while not self.used[r][f].passed(i // self.ahead & 1 ^ 1):
                yield
            self.fetched[r][f].expect()
            self.codes[r][f] = None
            self.copies.append((self.fetched[r][f], self.codes[r], f, i))
            yield

    def issuer(self, r):
        i = g = 0
        for count in self.tiles:
            for n in range(count):
                (s, parity), place, b = self.stage(i), n % self.group, g & 1
                if place == 0 and g > 1:
                    while not self.read[r][b].passed(g >> 1 & 1 ^ 1):
                        yield
                while not self.full[r][s].passed(parity):
                    yield
                last = place == self.group - 1 or n == count - 1
                assert self.holds[r][s] == [i] * (self.team + 1), "a stage that is not whole"
                if r == 1:
                    self.full[0][s].arrive()
                else:
                    if place == 0:
                        assert all(self.reads[q][b] == g // 2 * self.adders for q in (0, 1)), "an accumulator in use"
                    self.products += [("product", i, s, b, g), ("freed", s)] + ([("summed", b, g)] if last else [])
                g += last
                i += 1
                yield

    def adder(self, r):
        g = 0
        for count in self.tiles:
            for _ in range(0, count, self.group):
                b = g & 1
                while not self.summed[r][b].passed(g >> 1 & 1):
                    yield
                assert self.sums[b] == ("whole", g), "sums that are not whole"
                yield
                self.reads[r][b] += 1
                self.read[r][b].arrive()
                g += 1
                yield

    def land(self):
        if self.copies:
            barrier, to, at, i = self.copies.pop(self.rng.randrange(len(self.copies)))
            to[at] = i
            barrier.land()

    def finish(self):
        if not self.products:
            return
        what, *args = self.products.pop(0)
        if what == "product":
            i, s, b, g = args
            assert self.holds[0][s] == self.holds[1][s] == [i] * (self.team + 1), "an operand changed under a product"
            self.sums[b], self.consumed = ("part", g), i
        elif what == "freed":
            for r in (0, 1):
                self.freed[r][args[0]].arrive()
        else:
            self.sums[args[0]] = ("whole", args[1])
            for r in (0, 1):
                self.summed[r][args[0]].arrive()

    def run(self):
        roles = [self.writer(r, t, m) for r in (0, 1) for t in range(self.teams) for m in range(self.team)]
        roles += [f(r) for r in (0, 1) for f in (self.dy_copies, self.code_copies, self.issuer)]
        roles += [self.adder(r) for r in (0, 1) for _ in range(self.adders)]
        # every role, the copies and the products at a pace of their own
        steps = [(lambda g=g: next(g)) for g in roles] + [self.land, self.finish]
        pace = [self.rng.choice([0.02, 0.3, 1, 5]) for _ in steps]
        left = len(roles)
        for _ in range(300_000):
            if left == 0:
                return
            k = self.rng.choices(range(len(steps)), pace)[0]
            try:
                steps[k]()
            except StopIteration:
                pace[k] = 0
                left -= 1
        raise AssertionError("nothing moves any more")


def _runs(stages, ahead, teams, group, seeds):
    for seed in range(seeds):
        rng = random.Random(seed)
        tiles = [rng.choice([0, 1, 2, 3, 5, 8, 9, 17]) for _ in range(rng.randint(1, 3))]
        Pair(stages, ahead, teams, group, tiles, rng).run()


# (stages, stages of codes, teams, stages of a group) of the kernel's instances: bf16 in tiles of 256
# and 128 inputs, two terms, three terms
@pytest.mark.parametrize("stages,ahead,teams,group", [(4, 7, 3, 8), (4, 8, 3, 8), (3, 5, 3, 4), (4, 6, 3, 4), (2, 7, 2, 3),
                                                      (3, 4, 3, 3)])
def test_every_instance(stages, ahead, teams, group):
    _runs(stages, ahead, teams, group, seeds=12)


def test_the_model_sees_more_teams_than_stages():
    """Three teams on two stages: a wait passes two phases early."""
    with pytest.raises(AssertionError, match="in use|arrivals|other codes|not whole|changed"):
        _runs(2, 8, 3, 4, seeds=30)
