"""The roles of linear_states as processes on mbarriers (CPU only), as those of the two other kernels are
(tests/test_linear_protocol.py): a wait sees only its barrier's parity, schedules starve one role, and what is read in
shared and tensor memory is what was written for it."""
import random

import pytest

from tests.test_linear_protocol import Cta


class States(Cta):
    """`pieces`: chunks of each piece; `terms` of a weighted key."""

    def __init__(self, d, group, pieces, terms):
        super().__init__(d, group, [(n, False, False) for n in pieces])
        self.terms, self.slots = terms, (3 if terms == 1 else 2) * (2 if d == 64 else 1)
        self.units = [(c, h) for c in range(sum(pieces)) for h in range(group)]     # a chunk of a key head
        self.held = {}

    def write(self, place, what):
        assert self.held.get(place, (None, True))[1], ("written before it was read", place, what)
        self.held[place] = (what, False)

    def read(self, place, what):
        assert self.held.get(place, (None,))[0] == what, (place, what, self.held.get(place))
        self.held[place] = (what, True)

    def roles(self):
        return dict(load=self.load(), mma=self.mma(), keys0=self.keys(0), keys1=self.keys(1), sums=self.sums())

    def load(self):
        for it in range(len(self.units)):
            yield "nothing", 0
            if it >= self.slots:
                yield ("kv_empty", it % self.slots), it // self.slots
            for half in range(2):
                self.write(("tile", it % self.slots, half), it)
            self.arrive(("kv_full", it % self.slots))

    def keys(self, half):
        for it in range(len(self.units)):
            yield ("kv_full", it % self.slots), it // self.slots + 1
            if self.terms > 1 and it > 0:
                yield ("term_free", half), it
            if self.terms > 1:
                self.write(("term", half), it)
            self.arrive(("kt_full", it % self.slots, half))

    def mma(self):
        for it, (un, h) in enumerate(self.units):
            slot = it % self.slots
            if h == 0 and un >= 2:
                yield ("u_free", un & 1), un // 2
            for half in range(2):
                yield ("kt_full", slot, half), it // self.slots + 1
                self.read(("tile", slot, half), it)
                if self.terms > 1:
                    self.read(("term", half), it)
                    self.arrive(("term_free", half))
            self.arrive(("kv_empty", slot))
            if h == self.group - 1:
                self.write(("u", un & 1), un)
                self.arrive(("u_full", un & 1))

    def sums(self):
        for un in range(len(self.units) // self.group):
            yield ("u_full", un & 1), un // 2 + 1
            self.read(("u", un & 1), un)
            self.arrive(("u_free", un & 1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms", [1, 3])
@pytest.mark.parametrize("group", [1, 2, 5, 8])
def test_no_schedule_deadlocks_or_misleads_a_wait(group, terms, d):
    rng = random.Random(group * 1000 + d + terms)
    for _ in range(25):
        pieces = [rng.choice([1, 1, 2, 3, 7, 20]) for _ in range(rng.randint(1, 6))]
        for starved in (*States(d, group, pieces, terms).roles(), None):
            stuck = States(d, group, pieces, terms).run(rng, starved)
            assert stuck is None, (starved, pieces, stuck)


def test_the_simulation_sees_a_term_that_is_not_waited_for():
    class Early(States):
        def keys(self, half):
            for bar, phases in super().keys(half):
                if bar[0] != "term_free":
                    yield bar, phases

    with pytest.raises(AssertionError):
        for seed in range(40):
            Early(64, 1, [9], 3).run(random.Random(seed), "mma")


def test_the_simulation_sees_a_sum_that_is_not_waited_for():
    class Early(States):
        def mma(self):
            for bar, phases in super().mma():
                if bar[0] != "u_free":
                    yield bar, phases

    with pytest.raises(AssertionError):
        for seed in range(40):
            Early(128, 1, [9], 1).run(random.Random(seed), "sums")
