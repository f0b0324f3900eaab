"""The waits of the layer norm's forward by bulk copies when one of them gives up: a model of its
barriers and of a block's warps under random schedules, some copies later than the limit.

A warp whose wait has given up reads its rows from global memory from then on.  It must not wait at
a stage again: a parity wait passes at once on a barrier that is a phase behind."""
import os
import random
import re

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32525_gb300", "csrc",
                   "fs_rows.cuh")
WARPS = 8


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.tx, self.phase = count, count, 0, 0

    def _turn(self):
        if self.left == 0 and self.tx == 0:
            self.left, self.phase = self.count, self.phase + 1

    def arrive(self, tx=0):
        assert self.left > 0
        self.left, self.tx = self.left - 1, self.tx + tx
        self._turn()

    def complete(self, tx):
        self.tx -= tx
        self._turn()

    def passes(self, parity):
        return self.phase & 1 != parity


def run_block(rng, stages, chunks, late, keep_on, limit=40):
    """Which chunk's rows each warp used for each chunk; late: chance of a copy that comes after the
    limit; keep_on: a warp that gave up once goes on waiting (what the kernel must not do)."""
    full, empty = [Barrier(1) for _ in range(stages)], [Barrier(WARPS) for _ in range(stages)]
    held, flying, abort, issued, used = [None] * stages, [], [False], [0], []

    def issue(chunk, s):
        assert all(f[1] != s for f in flying), "a stage is filled while a copy is on its way to it"
        full[s].arrive(tx=1)
        flying.append([rng.randint(limit * 3, limit * 60) if rng.random() < late else rng.randint(0, 4), s, chunk])
        issued[0] += 1

    def wait(bar, parity):
        for polls in range(10 ** 9):
            if bar.passes(parity):
                return True
            if abort[0] or polls > limit:
                abort[0] = True
                return False
            yield

    def warp(w):
        if w == 0:
            for s in range(min(stages - 1, chunks)):
                issue(s, s)
        s, parity, staged = 0, 0, True
        for chunk in range(chunks):
            ahead = chunk + stages - 1
            if w == 0 and staged and ahead < chunks:
                e = (s - 1) % stages
                free = chunk == 0 or (yield from wait(empty[e], parity ^ 1 if s == 0 else parity))
                if not keep_on:
                    staged = free
                if free:
                    issue(ahead, e)
            in_stage = staged and (yield from wait(full[s], parity))
            if not keep_on:
                staged = in_stage
            used.append((chunk, held[s] if in_stage else chunk))
            yield
            if staged:
                empty[s].arrive()
            s, parity = (0, parity ^ 1) if s + 1 == stages else (s + 1, parity)
        if w == 0 and not staged:  # the drain: no look at the abort flag
            for i in range(max(0, issued[0] - stages), issued[0]):
                while not full[i % stages].passes((i // stages) & 1):
                    yield

    live = [warp(w) for w in range(WARPS)]
    while live:
        for f in list(flying):
            f[0] -= 1
            if f[0] < 0:
                flying.remove(f)
                held[f[1]] = f[2]
                full[f[1]].complete(1)
        for w in rng.sample(live, len(live)):
            if rng.random() < 0.7:
                try:
                    next(w)
                except StopIteration:
                    live.remove(w)
    assert not flying, "the block ends with a copy on its way"
    return used, abort[0]


@pytest.mark.parametrize("stages", [2, 3, 6])
def test_rows_are_right_when_a_wait_gives_up(stages):
    gave_up = 0
    for seed in range(300):
        used, abort = run_block(random.Random(seed), stages, chunks=17, late=0.05, keep_on=False)
        gave_up += abort
        assert len(used) == 17 * WARPS and all(want == got for want, got in used)
    assert gave_up > 50


def test_nothing_gives_up_without_a_late_copy():
    for seed in range(50):
        used, abort = run_block(random.Random(seed), 3, chunks=20, late=0.0, keep_on=False, limit=10 ** 6)
        assert not abort and all(want == got for want, got in used)


def test_the_model_sees_a_warp_that_waits_again():
    wrong = 0
    for seed in range(300):
        try:
            used, _ = run_block(random.Random(seed), 3, chunks=17, late=0.05, keep_on=True)
            wrong += any(want != got for want, got in used)
        except AssertionError:  # a stage filled anew, or an arrival too many
            wrong += 1
    assert wrong > 20


def test_the_kernel_does_as_the_model():
    text = open(SRC).read()
    body = text[text.index("void __launch_bounds__(256, 3) k_norm_fwd_bulk("):]
    body = body[:body.index("\n}\n")]
    lines = [line.strip() for line in body.splitlines()]
    waits = [line for line in lines if "mbar_wait" in line]
    assert waits == ["staged = chunk == first || tc::mbar_wait_w(&empty[w], s == 0 ? parity ^ 1u : parity, &ab, nullptr);",
                     "if (whole && staged) staged = tc::mbar_wait_w(&full[s], parity, &ab, nullptr);"]
    assert "if (warp == 0 && staged && ahead < chunks) {" in lines and "if (staged && t == 0) issue(ahead, w);" in lines
    assert [line for line in lines if "mbar_arrive" in line] == ["if (t == 0 && staged) tc::mbar_arrive(&empty[s]);"]
    drain = re.search(r"if \(threadIdx.x == 0 && !staged\).*?\n\s*for \(int i = max\(0, issued - plan.stages\); i < issued; i\+\+\)\s*"
                      r"tc::mbar_drain\(&full\[i % plan.stages\], \(uint32_t\)\(i / plan.stages\) & 1u\);", body, re.S)
    assert drain
