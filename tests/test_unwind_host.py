"""What a tensor-core kernel waits for before it ends after a role gave up: the library's plan (bimask_debug_drain_plan, the
arithmetic that the kernels run) against a model of its pipeline.  Two CTAs load the stages of a ring, the loads of a stage
complete on one mbarrier of CTA 0, a consumer hands stages back; everybody stops at a random point and loads land late.
No GPU is touched."""
import random

import pytest


@pytest.fixture(scope="module")
def bm():
    from paper_2302_06058_b200 import build
    build.build()
    import paper_2302_06058_b200 as m
    m.lib()
    return m


class Barrier:
    """An mbarrier of one arrival per phase: the phase ends when the arrival is in and no bytes are outstanding."""

    def __init__(self):
        self.phase, self.pending, self.tx = 0, 1, 0

    def _step(self):
        if self.pending == 0 and self.tx == 0:
            self.phase, self.pending = self.phase + 1, 1

    def expect(self, n):                                     # arrive.expect_tx
        assert self.pending == 1, "a second arrival in one phase"
        self.tx += n
        self.pending = 0
        self._step()

    def complete(self, n):
        self.tx -= n
        self._step()

    def passes(self, parity):
        return (self.phase & 1) != parity


class Ring:
    def __init__(self, rng, stages, ctas, total):
        self.rng, self.stages, self.ctas, self.total = rng, stages, ctas, total
        self.full = [Barrier() for _ in range(stages)]
        self.issued, self.consumed, self.in_flight = [0] * ctas, 0, []

    def land(self):
        if self.in_flight:
            k, _ = self.in_flight.pop(self.rng.randrange(len(self.in_flight)))
            self.full[k % self.stages].complete(1)

    def issue(self, r):
        k = self.issued[r]
        if k >= self.total or (k >= self.stages and self.consumed <= k - self.stages):
            return
        if r == 0:
            self.full[k % self.stages].expect(self.ctas)
        self.in_flight.append((k, r))
        self.issued[r] += 1

    def consume(self):
        k = self.consumed
        if k < self.total and k < min(self.issued) and self.full[k % self.stages].phase > k // self.stages:
            self.consumed += 1

    def run(self, steps):
        """Random steps; each role stops for good at a point of its own, and from some point on no load lands."""
        stop = [self.rng.randrange(steps) for _ in range(self.ctas + 2)]
        for t in range(steps):
            what = self.rng.randrange(self.ctas + 2)
            if what < self.ctas:
                if t < stop[what]:
                    self.issue(what)
            elif what == self.ctas:
                if t < stop[self.ctas]:
                    self.consume()
            elif t < stop[-1]:
                self.land()


@pytest.mark.parametrize("ctas", [1, 2])
@pytest.mark.parametrize("stages", [2, 3, 4, 6, 10])
def test_the_plan_waits_for_every_load_and_always_ends(bm, stages, ctas):
    rng = random.Random(100 * stages + ctas)
    late = uneven = 0
    for _ in range(400):
        ring = Ring(rng, stages, ctas, rng.randrange(0, 5 * stages))
        ring.run(rng.randrange(1, 60 * stages))
        late += bool(ring.in_flight)
        i0, i1 = ring.issued[0], ring.issued[-1]
        uneven += i0 != i1
        assert abs(i0 - i1) <= stages
        for stage, parity, settle in bm.bimask_debug_drain_plan(i0, i1, stages):
            bar = ring.full[stage]
            if settle == 1:
                bar.expect(1)
            elif settle == 2:
                bar.complete(1)
            while not bar.passes(parity):                    # only landing loads can end a wait now
                assert ring.in_flight, "a wait that nothing ends"
                ring.land()
        assert not ring.in_flight, "a load outlives the waits"
    assert late > 40 and (ctas == 1 or uneven > 40)           # the model did reach what the plan is for


def test_refusals(bm):
    assert bm.bimask_debug_drain_plan(0, 0, 4) == []
    for bad in ((-1, 0, 3), (0, -1, 3), (0, 0, 0), (9, 4, 4)):
        with pytest.raises(bm.BimaskError):
            bm.bimask_debug_drain_plan(*bad)
