"""The barriers of the orthogonal update's kernels, modelled on the CPU: loader, issuer and adders of one CTA or of a pair
run in any order, copies land and products end at any time (products in their order).  Nobody reads a stage that is not
there, overwrites one that is still read, adds an accumulator twice or misses one, and everybody comes to the end."""
import random

import pytest

STAGES, ADDERS = 3, 3  # adders: fewer than in the kernel, the same protocol


class Barrier:
    def __init__(self, arrivals):
        self.need, self.left, self.phase = arrivals, arrivals, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.need

    def passed(self, parity):
        """mbarrier's parity wait: whether the phase of that parity has ended."""
        return (self.phase & 1) != parity


class Cta:
    def __init__(self, ctas, rank):
        self.full = [Barrier(2 if ctas == 2 and rank == 0 else 1) for _ in range(STAGES)]
        self.freed = [Barrier(1) for _ in range(STAGES)]
        self.summed = [Barrier(1) for _ in range(2)]
        self.read = [Barrier(ADDERS) for _ in range(2)]
        self.ready = Barrier(ADDERS)
        self.holds = [None] * STAGES      # the fill that a stage holds
        self.accumulator = [None] * 2     # the groups' stages that it sums
        self.unread = [0, 0]              # adders that have still to read it


def _run(ctas_count, roles, r):
    """Steps through the roles (generators that yield a condition to wait for, or None) in random order."""
    waiting, steps = {k: (g, next(g)) for k, g in enumerate(roles)}, 0
    while waiting:
        steps += 1
        assert steps < 100000, "nobody goes on"  # (the longest run takes a few thousand)
        k = r.choice(list(waiting))
        g, until = waiting[k]
        if until is not None and not until():
            continue
        try:
            waiting[k] = (g, next(g))
        except StopIteration:
            del waiting[k]


class Engine:
    """Copies that land in any order, and products that end in theirs."""

    def __init__(self, r):
        self.r, self.copies, self.products, self.done = r, [], [], False

    def run(self):
        while not (self.done and not self.copies and not self.products):
            if self.copies and self.r.random() < 0.5:
                self.copies.pop(self.r.randrange(len(self.copies)))()
            elif self.products and self.r.random() < 0.5:
                self.products.pop(0)()
            yield None


def _tiles(ctas, tiles, count, group_of, r):
    """relay_orthogonalise_kernel: tiles of `count` stages, summed `group_of` at a time."""
    cta, engine, ended = [Cta(ctas, k) for k in range(ctas)], Engine(r), [0]

    def loader(me):
        for i in range(tiles * count):
            s = i % STAGES
            yield lambda: cta[me].freed[s].passed((i // STAGES & 1) ^ 1)
            assert cta[me].holds[s] is None

            def land(s=s, i=i):
                cta[me].holds[s] = i
                cta[me].full[s].arrive()
            engine.copies.append(land)
            yield None
        ended[0] += 1

    def issuer(me):
        i = group = 0
        for _ in range(tiles):
            for n in range(count):
                s, place, b = i % STAGES, n % group_of, group & 1
                if place == 0 and group > 1:
                    yield lambda: cta[me].read[b].passed((group >> 1 & 1) ^ 1)
                yield lambda: cta[me].full[s].passed(i // STAGES & 1)
                assert cta[me].holds[s] == i
                last = place == group_of - 1 or n == count - 1
                if me != 0:
                    cta[0].full[s].arrive()
                else:
                    for c in cta:
                        assert c.holds[s] == i
                        if place == 0:
                            assert c.unread[b] == 0
                            c.accumulator[b] = []
                        c.accumulator[b].append(i)

                    def end(s=s, b=b, last=last):
                        for c in cta:
                            c.holds[s] = None
                            c.freed[s].arrive()
                            if last:
                                c.unread[b] = ADDERS
                                c.summed[b].arrive()
                    engine.products.append(end)
                if last:
                    group += 1
                i += 1
                yield None
        ended[0] += 1

    def adder(me, seen):
        group = 0
        for tile in range(tiles):
            for done in range(0, count, group_of):
                b = group & 1
                yield lambda: cta[me].summed[b].passed(group >> 1 & 1)
                assert cta[me].accumulator[b] == list(range(tile * count + done, tile * count + min(count, done + group_of)))
                cta[me].unread[b] -= 1
                yield None
                cta[me].read[b].arrive()
                seen.append(group)
                group += 1
        ended[0] += 1

    seen = [[[] for _ in range(ADDERS)] for _ in cta]
    roles = [f(k) for k in range(ctas) for f in (loader, issuer)] + [adder(k, s) for k in range(ctas) for s in seen[k]]

    def watch():
        yield lambda: ended[0] == len(roles)
        engine.done = True
    _run(ctas, roles + [engine.run(), watch()], r)
    groups = tiles * -(-count // group_of)
    assert all(s == list(range(groups)) for per in seen for s in per)


@pytest.mark.parametrize("ctas", [1, 2])
@pytest.mark.parametrize("count", [1, 2, 3, 4, 7])
def test_tiles(ctas, count):
    r = random.Random(count)
    for tiles in (1, 2, 3):
        for group in (1, 3):
            for _ in range(6):
                _tiles(ctas, tiles, count, group, r)


def _step(count, panels, r):
    """relay_orthogonalise_step_kernel: g, its polynomial through the operand in shared memory, and x's columns."""
    cta, engine, ended = Cta(1, 0), Engine(r), [0]
    operand = {"writes": 0, "reading": 0}

    def loader():
        for i in range(count + panels):
            s = i % STAGES
            yield lambda: cta.freed[s].passed((i // STAGES & 1) ^ 1)
            assert cta.holds[s] is None

            def land(s=s, i=i):
                cta.holds[s] = i
                cta.full[s].arrive()
            engine.copies.append(land)
            yield None
        ended[0] += 1

    def issuer():
        group = 0

        def multiply(what, stage):
            b = group & 1
            assert cta.unread[b] == 0
            cta.accumulator[b] = what
            operand["reading"] += what[0] != "g"

            def end():
                operand["reading"] -= what[0] != "g"
                if stage is not None:
                    cta.holds[stage] = None
                    cta.freed[stage].arrive()
                cta.unread[b] = ADDERS
                cta.summed[b].arrive()
            engine.products.append(end)

        def accumulator():
            return group <= 1 or cta.read[group & 1].passed((group >> 1 & 1) ^ 1)

        for i in range(count):
            yield accumulator
            yield lambda: cta.full[i % STAGES].passed(i // STAGES & 1)
            assert cta.holds[i % STAGES] == i
            multiply(("g", i), i % STAGES)
            group += 1
        yield lambda: cta.ready.passed(0)
        assert operand["writes"] == ADDERS
        for p in range(panels):
            yield accumulator
            multiply(("p", p), None)
            group += 1
        yield lambda: cta.ready.passed(1)
        assert operand["writes"] == 2 * ADDERS
        for p in range(panels):
            i = count + p
            yield accumulator
            yield lambda: cta.full[i % STAGES].passed(i // STAGES & 1)
            assert cta.holds[i % STAGES] == i
            multiply(("x", p), i % STAGES)
            group += 1
        ended[0] += 1

    def adder():
        group = 0
        for name, groups in (("g", count), ("p", panels), ("x", panels)):
            for n in range(groups):
                b = group & 1
                yield lambda: cta.summed[b].passed(group >> 1 & 1)
                assert cta.accumulator[b] == (name, n)
                cta.unread[b] -= 1
                yield None
                cta.read[b].arrive()
                group += 1
            if name != "x":
                assert operand["reading"] == 0, "written while products read it"
                operand["writes"] += 1
                yield None
                cta.ready.arrive()
        ended[0] += 1

    roles = [loader(), issuer()] + [adder() for _ in range(ADDERS)]

    def watch():
        yield lambda: ended[0] == len(roles)
        engine.done = True
    _run(1, roles + [engine.run(), watch()], r)


@pytest.mark.parametrize("panels", [1, 2])
@pytest.mark.parametrize("count", [1, 2, 3, 5, 8])
def test_whole_step(count, panels):
    r = random.Random(10 * count + panels)
    for _ in range(30):
        _step(count, panels, r)
