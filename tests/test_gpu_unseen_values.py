"""Not-finite values in rows that nobody sees cost next to nothing, and never a wait that runs out."""
import math

import numpy as np
import pytest

from tests.test_gpu_draft import Trees, seen
from tests.test_gpu_draft import attend as attend_tree
from tests.test_gpu_prompt import bound, make

pytestmark = pytest.mark.gpu


def milliseconds(call, n=5):
    """The median of n calls' device times."""
    import torch
    call()
    times = []
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return sorted(times)[n // 2]


@pytest.mark.parametrize("t", [9, 12, 16])
def test_drafted_rows_past_the_count(cuda, t):
    """Padding of NaN: the same bits as padding of zeros, in the same time (within a factor of 3; row by row it took some 100)."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", hq=32, hkv=8, slots=24, beams=20, prompt=2000, room=150, pages=24 * 20 + 150, seed=t)
    trees = DraftTrees(x.pool, t)
    x.append(100)
    parent, count = x.trees(t, True)
    q, k, v = (x.rand(x.slots, t, h, 128) for h in (32, 8, 8))
    dp, dc = x.ints(parent), x.ints(count)
    past = torch.arange(t, device="cuda")[None] >= dc[:, None]
    out, times = [], []
    for fill in (0.0, float("nan"), float("inf")):
        for y in (q, k, v):
            y[past] = fill
        times.append(milliseconds(lambda: out.append(trees.attention(0, q, k, v, dp, x.scale, count=dc))))
    assert all(torch.equal(o, out[0]) for o in out)
    assert max(times) < 3 * times[0], times
    assert x.pool.status() == 0
