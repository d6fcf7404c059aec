"""What the CTAs of a cluster that share a row tell each other in distill_held (CPU only).

In place the gradient goes over the logits.  A CTA reads no logit but its own share's: no barrier waits for another CTA's
loads.  The exchange itself as processes: every CTA's words carry the turn that they were sent in, a wait tells only its
barrier's parity, and schedules that starve one CTA show a word that is written before its readers have read the one
before, and a wait that the parity misleads.
"""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_11185_gb300", "csrc")


def body(src, name):
    """The kernel's source without its comments."""
    src = re.sub(r"//[^\n]*", "", src)
    at = src.index("{", re.search(r"\b%s\(const __grid_constant__" % name, src).end())
    depth, end = 0, at
    for end in range(at, len(src)):
        depth += (src[end] == "{") - (src[end] == "}")
        if depth == 0:
            break
    return src[at:end]


def shares_of_others(kernel):
    """Uses of the row's logits in global memory that are not its own share's."""
    own = (r"bulk_load\([^;]*reinterpret_cast<const uint4\*>\(row\.z \+ row\.head\) \+ row\.v0 \+ row\.part\(i\)[^;]*;",
           r"loose \? to_float\(row\.z\[my_loose\]\)",         # the first CTA's, outside of all shares
           r"outside\(v\) \? to_float\(row\.z\[v\]\)")
    for x in own:
        kernel = re.sub(x, "", kernel)
    return re.findall(r"[^;{}]*\brow\.z\b[^;{}]*", kernel)


def test_a_cta_reads_its_own_share():
    with open(os.path.join(CSRC, "distill.cu")) as f:
        assert shares_of_others(body(f.read(), "distill_held")) == []


def test_the_reader_sees_a_row_that_is_passed_on():
    assert shares_of_others("{ float tmax = en.check(a, row.z, ids); x = row.z[id]; }") == [
        " float tmax = en.check(a, row.z, ids)", " x = row.z[id]"]


class Cluster:
    """`size` CTAs over `turns` rows."""

    def __init__(self, size, turns, buffers=2):
        self.size, self.turns, self.buffers = size, turns, buffers
        self.tx, self.done, self.words = {}, {}, {}

    def send(self, to, bar, of, word, turn):
        old = self.words.get((to, *word))
        assert old is None or old[1], ("written before it was read", to, word, turn)
        self.words[to, *word] = [turn, False]   # read
        self.tx[to, bar] = self.tx.get((to, bar), 0) + 1
        if self.tx[to, bar] % of == 0:
            self.done[to, bar] = self.done.get((to, bar), 0) + 1

    def read(self, at, word, turn):
        got = self.words[at, *word]
        assert got[0] == turn, ("another turn's word", at, word, turn, got)
        got[1] = True

    def cta(self, rank):
        def finish(t):
            yield ("added", t & 1), t // 2 + 1
            for c in range(1, self.size):
                self.read(0, ("term", t & 1, c), t)

        for t in range(self.turns):
            b = t % self.buffers
            yield "nothing", 0
            for c in range(self.size):
                self.send(c, ("met", b), self.size, ("sum", b, rank), t)
                yield "nothing", 0
            yield ("met", b), t // self.buffers + 1
            for c in range(self.size):
                self.read(rank, ("sum", b, c), t)
            if rank == 0 and t > 0:
                yield from finish(t - 1)
            yield "nothing", 0
            if rank > 0:
                self.send(0, ("added", t & 1), self.size - 1, ("term", t & 1, rank), t)
        if rank == 0:
            yield from finish(self.turns - 1)

    def run(self, rng, starved):
        roles = {r: self.cta(r) for r in range(self.size)}
        want = {r: next(x) for r, x in roles.items()}
        while roles:
            order = [r for r in roles if r != starved]
            rng.shuffle(order)
            moved = False
            for r in order + [r for r in roles if r == starved]:
                if r == starved and moved:
                    break
                bar, phases = want[r]
                have = self.done.get((r, bar), 0) if bar != "nothing" else 0
                if (have - phases) & 1:
                    continue
                assert have == phases, (r, bar, have, phases)
                moved = True
                want[r] = next(roles[r], None)
                if want[r] is None:
                    del roles[r]
                break
            assert moved, want


@pytest.mark.parametrize("size", [2, 4, 8])
def test_no_schedule_overwrites_a_word_or_misleads_a_wait(size):
    rng = random.Random(size)
    for _ in range(30):
        for starved in (*range(size), None):
            Cluster(size, rng.randint(1, 9)).run(rng, starved)


def test_the_simulation_sees_a_word_too_few():
    with pytest.raises(AssertionError):
        for seed in range(40):
            for starved in range(4):
                Cluster(4, 6, buffers=1).run(random.Random(seed), starved)


def test_logits_are_not_read_as_data_that_nobody_writes():
    # __ldg and .nc want data that no thread writes while the kernel runs; in place the gradient goes over the logits
    with open(os.path.join(CSRC, "distill.cu")) as f:
        src = re.sub(r"//[^\n]*", "", f.read())
    reads = re.findall(r"(?:__ldg|ld\.global\.nc)\(([^;]*?)\)", src)
    assert reads and all(re.match(r"&a\.(ids|t|weights|map)\b", x) for x in reads), reads
