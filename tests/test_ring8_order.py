"""The 8-bit attention's ring on the CPU: over sequences of units with any split of warps, no wait for a stage passes before
it has landed, none is overwritten before all of its readers have left it, and every sequence comes to its end."""
import random

import pytest

STAGES, WARPS, LOADERS = 24, 8, 2


class Barrier:
    """An mbarrier: a wait on a parity passes when the phase of that parity is the one before the current one."""

    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self, n=1):
        self.left -= n
        assert self.left >= 0
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1

    def passes(self, parity):
        return (self.phase - 1) & 1 == parity


def _loader(own, units, full, empty, held):
    base = 0
    for stages, _ in units:
        for i in range(stages):
            k = base + i
            if k % LOADERS != own:
                continue
            s = k % STAGES
            while k >= STAGES and not empty[s].passes((k // STAGES - 1) & 1):
                yield False
            held[s] = (k, WARPS)
            yield True                     # the copy lands some time later
            full[s].arrive()
        base += stages


def _warp(w, units, full, empty, held, meet):
    base = 0
    for u, (stages, rgroups) in enumerate(units):
        groups = WARPS // rgroups
        for i in range(w // rgroups, stages, groups):
            k = base + i
            s = k % STAGES
            while not full[s].passes((k // STAGES) & 1):
                yield False
            assert held[s][0] == k, "a wait passed on another stage"
            yield True
            assert held[s][0] == k, "overwritten while it is read"
            held[s] = (k, held[s][1] - groups)
            empty[s].arrive(groups)
        base += stages
        meet[u] += 1                       # the warps start a unit together
        while meet[u] < WARPS:
            yield False
        yield True


@pytest.mark.parametrize("seed", range(60))
def test_ring(seed):
    rng = random.Random(seed)
    units = [(rng.choice([1, 2, 7, 12, 24, 25, rng.randrange(1, 90)]), rng.choice([1, 2, 4, 8])) for _ in range(rng.randrange(1, 14))]
    full, empty = [Barrier(1) for _ in range(STAGES)], [Barrier(WARPS) for _ in range(STAGES)]
    held, meet = [None] * STAGES, [0] * len(units)
    tasks = [_loader(i, units, full, empty, held) for i in range(LOADERS)] + [_warp(w, units, full, empty, held, meet) for w in range(WARPS)]
    speed = [rng.choice([1, 1, 3, 20]) for _ in tasks]
    idle = 0
    while tasks:
        i = rng.choices(range(len(tasks)), speed)[0]
        try:
            idle = 0 if next(tasks[i]) else idle + 1
        except StopIteration:
            del tasks[i], speed[i]
            idle = 0
        assert idle < 20000, "nobody goes on"


def test_the_sizes_are_the_kernels():
    from pathlib import Path
    text = (Path(__file__).parents[1] / "paper_2608_08020_gb300" / "csrc" / "decode8.cu").read_text()
    for line in (f"kStages8 = {STAGES};", f"kConsumers8 = {WARPS};", f"kLoaders8 = {LOADERS};"):
        assert line in text
