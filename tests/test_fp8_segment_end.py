"""The softmax threads of the attention over the 8-bit cache meet once more at the end of a segment that holds a drafted row of V with a
NaN.  After a wait that gave up, the converting warps may raise such a flag, and the producer clear one, while the threads look: a model of
that under random interleavings, and the kernel's text for which of its two forms it has (no run on a GPU may show it)."""
import random
import re
from pathlib import Path

import pytest

SOURCE = re.sub(r"//[^\n]*", "", (Path(__file__).parent.parent / "paper_2510_07535_b200" / "csrc" / "verify_attn_fp8.cuh").read_text())
# what a thread looks at before the extra meeting
CONDITION = re.search(r"if \(([^\n]*)\) \{\s*named_barrier\(1, 256\);\s*mark_nan_drafts", SOURCE).group(1)
THREADS, SEGMENTS = 4, 5


class Cta:
    def __init__(self, rng, one_verdict):
        self.rng, self.one_verdict = rng, one_verdict
        self.flag = self.left = False
        self.waiting, self.generation = {1: 0, 3: 0}, {1: 0, 3: 0}

    def sync(self, bar):
        mine = self.generation[bar]
        self.waiting[bar] += 1
        if self.waiting[bar] == THREADS:
            self.waiting[bar], self.generation[bar] = 0, mine + 1
        return lambda: self.generation[bar] > mine

    def softmax(self, leader):
        for seg in range(SEGMENTS):
            if seg > 0:
                yield self.sync(1)               # Q's block is free
            if leader and self.one_verdict:
                self.left = self.flag
            yield self.sync(3)                   # the segment's end
            yield None
            if self.left if self.one_verdict else self.flag:
                yield self.sync(1)               # the results, which other threads have stored
                yield None

    def others(self):
        """Converting and producing warps that nothing paces any more."""
        for _ in range(40):
            self.flag = self.rng.random() < 0.5
            yield None

    def run(self):
        """True if all threads come to the end having met the same number of times."""
        roles = [[r, next(r)] for r in [self.softmax(i == 0) for i in range(THREADS)] + [self.others()]]
        while roles:
            ready = [r for r in roles if r[1] is None or r[1]()]
            if not ready:
                return False                     # a barrier that nobody completes
            r = self.rng.choice(ready)
            try:
                r[1] = next(r[0])
            except StopIteration:
                roles.remove(r)
        return not any(self.waiting.values())


@pytest.mark.parametrize("one_verdict", [True, False])
def test_a_verdict_for_all_ends_and_one_for_each_may_not(one_verdict):
    ends = [Cta(random.Random(seed), one_verdict).run() for seed in range(300)]
    assert all(ends) == one_verdict


def test_the_kernel_has_one_verdict_for_all():
    assert "nan_drafts" not in CONDITION
    word = re.search(r"aux->(\w+)", CONDITION).group(1)
    writers = re.findall(rf"aux->{word}\) = [^\n]*", SOURCE)
    assert len(writers) == 1 and "abort_flag" in writers[0]
    # left by the first softmax warp before all of them meet, on every path to a segment's end
    end = re.search(r"void (\w+)\(AuxFp8\* aux, const JointSegment& js\) \{\s*if \(js\.leader(.*?)\n\}", SOURCE, re.S)
    assert end and end.group(2).index(writers[0]) < end.group(2).index("meet_before_segment(aux, js.seg_no + 1")
    assert SOURCE.count("meet_before_segment(aux, js.seg_no + 1") == 1 and SOURCE.count(f"{end.group(1)}(aux, js);") == 3
