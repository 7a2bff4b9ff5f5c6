"""The named barriers of the 8-bit products after a wait that ran out, as a model on the CPU.

A warp that watches the accumulators (`watcher`) lets the epilogue warps go through named barriers, a set of them
per accumulator read, a barrier of the set per slice of columns, five warps each: the watcher arrives, four
epilogue warps wait.  The sets are used in turn.  A healthy GPU never lets the watcher's wait run out, so that
path is run here, under random schedules: every warp is a generator, any of them may take the next step, and
from some accumulator on none completes.  A barrier whose five arrivals belong to different accumulators
would release warps too early or leave one behind; neither may happen, all warps have to end, and no
barrier may be left half full."""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_17572_gb300", "csrc")


class Fault(Exception):
    pass


class Barriers:
    def __init__(self):
        self.open, self.phase = {}, {}

    def arrive(self, at, k):
        here = self.open.setdefault(at, [])
        here.append(k)
        if len(here) == 5:
            if len(set(here)) != 1:
                raise Fault(f"barrier {at} joins the reads {here}")
            self.open[at] = []
            self.phase[at] = self.phase.get(at, 0) + 1

    def wait(self, at, k):
        phase = self.phase.get(at, 0)
        self.arrive(at, k)
        while self.phase.get(at, 0) == phase:
            yield


def run(rng, tiles, k_blocks, accumulators, sets, slices):
    """One CTA's watcher and epilogue warps over `tiles` tiles; Fault where the protocol fails."""
    bars = Barriers()
    fails_at = rng.randrange(tiles * k_blocks + 1)  # reads from here on never find their accumulator complete
    read = [0] * (4 * slices)                       # accumulators that each epilogue warp has read
    last_tile = [-1]

    def complete(k):  # products into an accumulator start when all warps have read what it held
        return k < fails_at and all(n >= k - accumulators + 1 for n in read)

    def watcher():
        ok, k = True, 0
        for t in range(tiles):
            left = False
            for kb in range(k_blocks):
                at = k % sets * slices
                if ok:
                    while not complete(k):
                        if rng.random() < (0.05 if k >= fails_at else 0.002):
                            ok = False  # the wait ran out
                            break
                        yield
                    for s in range(slices):
                        bars.arrive(at + s, k)
                        yield
                else:
                    if kb == k_blocks - 1:
                        last_tile[0], left = t, True
                    for s in range(slices):
                        yield from bars.wait(at + s, k)
                k += 1
            if left:
                return

    def epilogue(w):
        k = 0
        for t in range(tiles):
            for _ in range(k_blocks):
                for _ in range(rng.randrange(60) if rng.random() < 0.05 else 1):
                    yield  # now and then a warp is far behind
                yield from bars.wait(k % sets * slices + w // 4, k)
                yield
                k += 1
                read[w] = k
            yield
            if last_tile[0] == t:
                return

    warps = [watcher()] + [epilogue(w) for w in range(4 * slices)]
    for _ in range(500_000):
        if not warps:
            break
        w = rng.choice(warps)
        try:
            next(w)
        except StopIteration:
            warps.remove(w)
    if warps:
        raise Fault(f"{len(warps)} warps never end")
    if any(bars.open.values()):
        raise Fault("a barrier is left half full")


def _constant(path, name):
    return re.search(rf"constexpr int {name} = ([^;]+);", open(os.path.join(CSRC, path)).read()).group(1)


def test_the_kernels_have_two_sets_more_than_accumulators():
    assert _constant("gemm_fp8.cu", "F_ACCS") == "4" and _constant("gemm_fp8.cu", "F_BARS") == "F_ACCS + 2"
    assert _constant("gemm_fp8_pair.cu", "W_ACCS") == "2" and _constant("gemm_fp8_pair.cu", "W_BARS") == "W_ACCS + 2"


@pytest.mark.parametrize("seed", range(4))
def test_pairs(seed):
    rng = random.Random(seed)
    for _ in range(300):
        run(rng, rng.randrange(1, 5), rng.randrange(1, 7), 2, 4, rng.choice((2, 4)))


@pytest.mark.parametrize("seed", range(4))
def test_single_ctas(seed):
    rng = random.Random(100 + seed)
    for _ in range(200):
        run(rng, 1, rng.randrange(1, 20), 4, 6, rng.choice((1, 2)))


def test_one_set_more_is_not_enough():
    """The model sees the fault that the number of sets avoids."""
    rng, faults = random.Random(7), 0
    for _ in range(300):
        try:
            run(rng, 3, 5, 2, 3, 1)
        except Fault:
            faults += 1
    assert faults > 0
