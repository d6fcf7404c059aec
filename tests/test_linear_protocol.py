"""The roles of linear_out and linear_back as processes on mbarriers (CPU only).

A wait names a barrier and the number of phases it wants completed, but the hardware tells only their parity: a wait two
phases behind passes too early, one phase ahead it blocks.  Each role is a generator that yields its waits, in the order
of the kernel's code, and completes phases between them; schedules that starve one role show both, and deadlocks.
`pieces`: the chunks of each piece of a CTA's walk, whether its head forgets fast, and the tail a last chunk has.
"""
import random

import pytest


class Cta:
    def __init__(self, d, group, pieces):
        self.d, self.group, self.pieces = d, group, pieces
        self.done, self.parts = {}, {}
        self.items = [(p, n, h) for p, (chunks, *_) in enumerate(pieces) for n in range(chunks) for h in range(group)]

    def arrive(self, bar, of=1):
        self.parts[bar] = self.parts.get(bar, 0) + 1
        if self.parts[bar] % of == 0:
            self.done[bar] = self.done.get(bar, 0) + 1

    def there(self, bar, phases):
        """What an MMA reads has arrived, whichever wait it relied on."""
        assert self.done.get(bar, 0) >= phases, (bar, phases, self.pieces)

    def run(self, rng, starved):
        """None, or what each role waits for when none can go on.  A wait that the parity misleads raises."""
        roles, want = self.roles(), {}
        for k in list(roles):
            want[k] = next(roles[k], None)
            if want[k] is None:
                del roles[k]
        while roles:
            moved = False
            order = [k for k in roles if k != starved]
            rng.shuffle(order)
            for k in order + [k for k in roles if k == starved]:
                if k == starved and moved:
                    break
                while k in roles:
                    bar, phases = want[k]
                    have = self.done.get(bar, 0)
                    if (have - phases) & 1:
                        break
                    assert have == phases, (k, bar, have, phases, self.pieces)
                    moved = True
                    want[k] = next(roles[k], None)
                    if want[k] is None:
                        del roles[k]
                    if k == starved:
                        break
            if not moved:
                return {k: want[k] for k in roles}


class Out(Cta):
    """linear_out."""

    def roles(self):
        self.nq, self.nt = (4, 8) if self.d == 64 else (1, 4) if self.group == 1 else (2, 3)
        self.np = 2 if self.d == 64 else 1
        return dict(load=self.load(), s=self.scores(), o=self.outputs(), rows0=self.rows(0), rows1=self.rows(1),
                    store=self.store(), state=self.state())

    def load(self):
        q = t = 0
        for _, _, h in self.items:
            for tile in ("k", "q", "v") if h == 0 else ("q",):
                yield "nothing", 0      # loads arrive one by one
                if tile == "q":
                    if q >= self.nq:
                        yield ("q_empty", q % self.nq), q // self.nq
                    self.arrive(("q_full", q % self.nq))
                    q += 1
                else:
                    if t >= self.nt:
                        yield ("t_empty", t % self.nt), t // self.nt
                    self.arrive(("t_full", t % self.nt))
                    t += 1

    def tile(self, t):
        return ("t_full", t % self.nt), t // self.nt + 1

    def scores(self):
        us = 0
        for it, (p, n, h) in enumerate(self.items):
            chunks, fast, _ = self.pieces[p]
            weigh, last, ki = n < chunks - 1, h == self.group - 1, it // self.group
            ks, vs = 2 * ki % self.nt, (2 * ki + 1) % self.nt
            if h == 0:
                yield self.tile(2 * ki)
            yield ("q_full", it % self.nq), it // self.nq + 1
            if it >= self.np:
                yield ("o_full", (it - self.np) & 1), (it - self.np) // 2 + 1
            self.there(*self.tile(2 * ki))
            self.there(("q_full", it % self.nq), it // self.nq + 1)
            self.arrive(("s_full", it & 1))
            self.arrive(("q_empty", it % self.nq), 2)
            if fast and weigh and last:
                self.arrive("k_done")
            if weigh and h == (self.group - 1 if fast or self.group == 1 else 1):
                if fast:
                    yield self.tile(2 * ki + 1)
                yield ("wt_full", ki & 3), ki // 4 + 1
                if us > 0:
                    yield "u_free", us
                us += 1
                self.there(*self.tile(2 * ki))
                self.there(*self.tile(2 * ki + 1))
                self.arrive("u_full")
                self.arrive(("t_empty", vs), 2)
            if last:
                self.arrive(("t_empty", ks), 2)
                self.arrive(("t_empty", ks), 2)
                if not weigh:
                    self.arrive(("t_empty", vs), 2)

    def outputs(self):
        def q_s(it):
            p, _, h = self.items[it]
            if h == 0:
                yield "s_ready", it // self.group + 1
            if it >= 2:
                yield ("o_free", it & 1), (it - 2) // 2 + 1
            yield ("q_full", it % self.nq), it // self.nq + 1
            self.there("s_ready", it // self.group + 1)
            self.arrive(("q_empty", it % self.nq), 2)
            if self.pieces[p][1]:
                self.arrive(("a_full", it & 1))
            if h == self.group - 1:
                self.arrive("s_read")

        yield from q_s(0)
        for it, (p, n, h) in enumerate(self.items):
            chunks, fast, _ = self.pieces[p]
            ki = it // self.group
            if h == 0 and fast:
                yield self.tile(2 * ki + 1)
            if h == 0 and not (fast and n < chunks - 1):
                yield ("wt_full", ki & 3), ki // 4 + 1
            yield ("p_full", it & 1), it // 2 + 1
            self.there(*self.tile(2 * ki + 1))
            if not fast:
                self.there(("wt_full", ki & 3), ki // 4 + 1)
            self.arrive(("o_full", it & 1))
            if h == self.group - 1:
                self.arrive(("t_empty", (2 * ki + 1) % self.nt), 2)
            if it + 1 < len(self.items):
                yield from q_s(it + 1)

    def rows(self, mine):
        fasts = 0
        for it, (p, n, h) in enumerate(self.items):
            chunks, fast, tail = self.pieces[p]
            if it & 1 != mine:
                continue
            yield ("s_full", mine), it // 2 + 1
            if fast:
                fasts += 1
                yield ("a_full", mine), fasts
                if h == 0 and tail and n == chunks - 1:
                    yield self.tile(2 * (it // self.group) + 1)
            self.arrive(("p_full", mine))
            yield ("o_full", mine), it // 2 + 1
            if it > 0:
                yield ("out_free", (it - 1) & 1), (it - 1) // 2 + 1
            self.arrive(("o_free", mine))
            self.arrive("out_full")

    def store(self):
        for it in range(len(self.items)):
            yield "out_full", it + 1
            self.arrive(("out_free", it & 1))

    def state(self):
        ki = kept = sums = 0
        for chunks, fast, _ in self.pieces:
            for n in range(chunks):
                if ki > 0:
                    yield "s_read", ki
                self.arrive("s_ready")
                if fast and n < chunks - 1:
                    kept += 1
                    yield "k_done", kept
                    yield self.tile(2 * ki)
                else:
                    yield self.tile(2 * ki + 1)
                self.arrive(("wt_full", ki & 3))
                ki += 1
                if n < chunks - 1:
                    sums += 1
                    yield "u_full", sums
                    self.arrive("u_free")


class Back(Cta):
    """linear_back."""

    def roles(self):
        self.nkv, self.nq, self.ns = (2, 4, 1) if self.d == 64 else (1, 2, 2)
        self.steps = [(*i, s) for i in self.items for s in range(self.ns)]
        return dict(load=self.load(), dv=self.grads(0), dk=self.grads(1), u=self.sums(), rows0=self.rows(0),
                    rows1=self.rows(1), state=self.state())

    def load(self):
        for it, (_, _, h) in enumerate(self.items):
            yield "nothing", 0
            if it >= self.nq:
                yield ("q_empty", it % self.nq), it // self.nq
            self.arrive(("q_full", it % self.nq))
            c = it // self.group
            for x in range(2) if h == 0 else ():
                yield "nothing", 0
                if c >= self.nkv:
                    yield ("k_empty", x, c % self.nkv), c // self.nkv
                self.arrive(("k_full", x, c % self.nkv))

    def grads(self, x):
        def product(t):
            p, _, h, s = self.steps[t]
            it, c = t // self.ns, t // self.ns // self.group
            if s == 0:
                yield ("wt_full", it % self.nq), it // self.nq + 1
                if self.pieces[p][1]:
                    yield ("q_full", it % self.nq), it // self.nq + 1
                if h == 0:
                    yield ("k_full", x, c % self.nkv), c // self.nkv + 1
            self.there(("q_full", it % self.nq), it // self.nq + 1)
            self.there(("k_full", x, c % self.nkv), c // self.nkv + 1)
            self.arrive(("s_full", x))
            if self.nkv == 1 and s == self.ns - 1 and h == self.group - 1:
                self.arrive(("k_empty", x, 0))

        yield from product(0)
        for t, (p, n, h, s) in enumerate(self.steps):
            chunks, fast, _ = self.pieces[p]
            it, c = t // self.ns, t // self.ns // self.group
            item, end = s == self.ns - 1, s == self.ns - 1 and h == self.group - 1
            if h == s == 0 and c > 0:
                yield ("o_free", x), c
            if s == 0 and h == (0 if fast or self.group == 1 else 1):
                yield "s_ready", c + 1
                if fast:
                    self.arrive(("a_full", x))
                self.arrive("s_read", 2)
            yield ("p_full", x), t + 1
            self.there(("q_full", it % self.nq), it // self.nq + 1)
            if item:
                self.arrive(("q_empty", it % self.nq), 3)
                if fast and n < chunks - 1:
                    self.arrive("k_done", 2)
            if end:
                self.arrive(("o_full", x))
                if self.nkv > 1:
                    self.arrive(("k_empty", x, c % self.nkv))
            if t + 1 < len(self.steps):
                yield from product(t + 1)

    def sums(self):
        us = fasts = 0
        for it, (p, n, h) in enumerate(self.items):
            chunks, fast, _ = self.pieces[p]
            weigh = n < chunks - 1
            if weigh and fast:
                yield ("wt2", fasts & 3), fasts // 4 + 1
                fasts += 1
            else:
                yield ("wt_full", it % self.nq), it // self.nq + 1
            if weigh and h == 0:
                if us > 0:
                    yield "u_free", us
                us += 1
            self.there(("q_full", it % self.nq), it // self.nq + 1)
            if weigh and h == self.group - 1:
                self.arrive("u_full")
            self.arrive(("q_empty", it % self.nq), 3)

    def rows(self, x):
        fasts = 0
        for t, (p, _, h, s) in enumerate(self.steps):
            if self.pieces[p][1] and h == s == 0:
                fasts += 1
                yield ("a_full", x), fasts
            yield ("s_full", x), t + 1
            self.arrive(("p_full", x))
            if h == self.group - 1 and s == self.ns - 1:
                yield ("o_full", x), t // self.ns // self.group + 1
                self.arrive(("o_free", x))

    def state(self):
        it = c = kept = sums = 0
        for chunks, fast, _ in self.pieces:
            done = 0
            for n in range(chunks):
                if c > 0:
                    yield "s_read", c
                self.arrive("s_ready")
                c += 1
                for done in range(done, min((n + 1) * self.group + (not fast), chunks * self.group)):
                    yield ("q_full", it % self.nq), it // self.nq + 1
                    self.arrive(("wt_full", it % self.nq))
                    if fast and done // self.group < chunks - 1:
                        kept += 1
                        yield "k_done", kept
                        self.arrive(("wt2", (kept - 1) & 3))
                    it += 1
                    done += 1
                if n < chunks - 1:
                    sums += 1
                    yield "u_full", sums
                    self.arrive("u_free")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,group", [(k, g) for k in (Out, Back) for g in (1, 2, 3, 5, 8)])
def test_no_schedule_deadlocks_or_misleads_a_wait(kind, group, d):
    rng = random.Random(group * 1000 + d)
    for _ in range(25):
        pieces = [(rng.choice([1, 1, 2, 3, 4, 9]), rng.random() < 0.4, rng.random() < 0.5)
                  for _ in range(rng.randint(1, 8))]
        for starved in (*kind(d, group, pieces).roles(), None):
            stuck = kind(d, group, pieces).run(rng, starved)
            assert stuck is None, (starved, pieces, stuck)


def test_the_simulation_sees_a_tile_that_is_not_there():
    class Early(Out):
        def scores(self):   # K^T V of a head that forgets fast without waiting for V
            for bar, phases in super().scores():
                if not (bar[0] == "t_full" and bar[1] % 2 == 1):
                    yield bar, phases

    with pytest.raises(AssertionError):
        for seed in range(40):
            Early(64, 1, [(3, True, False), (2, True, True)]).run(random.Random(seed), "load")


def test_the_simulation_sees_a_wait_two_phases_behind():
    class Two(Out):
        def store(self):    # one barrier for both warpgroups, of which each waits for every other phase
            for it in range(len(self.items)):
                yield "out_full", it + 1
                self.arrive("out_free")

        def rows(self, mine):
            for bar, phases in super().rows(mine):
                if bar[0] == "out_free":
                    bar, phases = "out_free", phases * 2 - 1 + bar[1]
                yield bar, phases

    with pytest.raises(AssertionError):
        for seed in range(40):
            rng = random.Random(seed)
            for starved in ("rows0", "rows1", "store"):
                Two(64, 2, [(3, False, False), (2, True, True)]).run(rng, starved)
