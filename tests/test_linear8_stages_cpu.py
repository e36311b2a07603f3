"""The order of LDS reads and writes of the 8-bit products whose rows pass through
registers (tile8 in csrc/ll_linear8.hpp), as a model on the CPU.

Between two barriers waves may be anywhere: what one of them reads there, no
other may write, unless it writes what is there already.  GPU tests of the same
sums cannot show that, since a wave is seldom late enough.
"""
import pytest

WORD = 4  # stages of which a row's scales lie in one word


class Model:
    """Buffers by name, each with what it holds; steps between barriers.

    `always`: a stage commits the slot behind it even where no stage follows."""

    def __init__(self, steps, always=False):
        self.steps, self.always, self.at = steps, always, 0
        self.held, self.reads, self.writes = {}, {}, {}
        self.faults = []

    def barrier(self):
        for name, value in self.writes.items():
            if name in self.reads and self.reads[name] != value:
                self.faults.append((name, self.reads[name], value))
            self.held[name] = value
        self.reads, self.writes = {}, {}

    def read(self, name, want):
        """A read of `want`, which has to be there since the barrier before."""
        if self.held.get(name) != want:
            self.faults.append((name, want, self.held.get(name)))
        self.reads[name] = want

    def fetch(self, s):
        """(rows' stage, word of scales) of a fetch: the next stage, or the last one again."""
        got = self.at, min(s, self.steps - 1) // WORD
        if s + 1 < self.steps:
            self.at += 1
        return got

    def commit(self, slot, s, buffer):
        rows, word = slot
        self.writes["rows", buffer] = rows
        self.writes["scales", s // WORD & 1] = word

    def stage(self, b, s, whole):
        self.read(("rows", b), s)  # the second half of its k
        if whole or self.always or s + 1 < self.steps:
            self.commit(self.ahead[b], s + 1, 1 - b)
        self.barrier()
        if whole:
            self.ahead[b] = self.fetch(s + 3)
        if s + 1 < self.steps:
            self.read(("scales", (s + 1) // WORD & 1), (s + 1) // WORD)
            self.read(("rows", 1 - b), s + 1)

    def run(self):
        first = self.fetch(0)
        self.ahead = [self.fetch(1), self.fetch(2)]
        self.commit(first, 0, 0)
        self.barrier()
        self.read(("scales", 0), 0)
        self.read(("rows", 0), 0)
        s = 0
        while s + 4 < self.steps:
            self.stage(0, s, True)
            self.stage(1, s + 1, True)
            s += 2
        if s + 3 < self.steps:
            self.stage(0, s, True)
            self.stage(1, s + 1, False)
            s += 2
        while s < self.steps:
            self.stage(0, s, False)
            if s + 1 < self.steps:
                self.stage(1, s + 1, False)
            s += 2
        return self.faults


@pytest.mark.parametrize("steps", list(range(1, 81)))
def test_no_wave_writes_what_another_may_read(steps):
    assert Model(steps).run() == []


def test_the_model_sees_a_word_written_too_late():
    """With a commit behind the last stage too, word m - 1 goes over word m at 4 m + 1 stages."""
    for steps in range(1, 81):
        faults = Model(steps, always=True).run()
        m = (steps - 1) // WORD
        assert faults == ([(("scales", m & 1), m, m - 1)] if steps % WORD == 1 and m else [])
