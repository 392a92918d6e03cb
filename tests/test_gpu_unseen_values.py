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


def rows_of(q, k, v, rows, scale):
    """(softmax(scale q.k) v, the same of |v|) of some rows of one causal sequence, in 64 bits."""
    import torch
    g = q.shape[1] // k.shape[1]
    o, a = [], []
    for i in rows:
        kk, vv = (x[:i + 1].double().repeat_interleave(g, 1) for x in (k, v))
        p = torch.softmax(torch.einsum("hd,thd->ht", q[i].double(), kk) * scale, -1)
        o.append(torch.einsum("ht,thd->hd", p, vv))
        a.append(torch.einsum("ht,thd->hd", p, vv.abs()))
    return torch.stack(o), torch.stack(a)


def test_behind_a_long_prompt(cuda):
    """131072 tokens whose last one, and the next sequence, hold NaN: every row of the last tile but one is summed again over
    all its keys, which takes longer than the other warps' usual waits, and none runs out."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    n = 1 << 17
    q, k, v = make("bf16", n + 300, 2, 1, 41)
    v[n - 1:] = float("nan")
    op = PromptAttention(2, 1, 128, "bf16", max_tokens=n + 300, max_seqs=2)
    cu = torch.tensor([0, n, n + 300], dtype=torch.int32, device="cuda")
    out = op(q, k, v, cu, 1 / math.sqrt(128))
    assert op.status() == 0
    assert bool(out[:n - 1].isfinite().all()) and not bool(out[n - 1:].isfinite().any())
    rows = [n - 2, n - 3, n - 64, n - 65, n - 100, n - 128, n - 129]
    o, a = rows_of(q, k, v, rows, 1 / math.sqrt(128))
    assert bool(((out[rows].double() - o).abs() <= bound(o, a, "bf16")).all())


def test_a_token_of_nan_in_a_prompt(cuda):
    """Rows before it do not see it, rows from it on do and have nothing to sum again: it costs little."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    n, at = 6000, 1001
    q, k, v = make("bf16", n, 8, 2, 42)
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=n, max_seqs=1)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    times = []
    for fill in (0.0, float("nan")):
        v[at, :, 7] = fill
        times.append(milliseconds(lambda: op(q, k, v, cu, 1 / math.sqrt(128), out)))
    assert op.status() == 0
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[at:, :, 7] = True
    assert torch.equal(out.isnan(), bad)
    rows = [at - 1, at - 2, at - 20, 960, 959, at, 1100, 5999]
    vv = v.clone()
    vv[at, :, 7] = 0
    o, a = rows_of(q, k, vv, rows, 1 / math.sqrt(128))
    ok = (out[rows].double() - o).abs() <= bound(o, a, "bf16")
    assert bool((ok | bad[rows]).all())
    assert times[1] < times[0] + 5, times


def test_a_drafted_token_of_nan(cuda):
    """Over a long context: its descendants see it, the tree's other tokens do not."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", hq=16, hkv=4, slots=3, beams=2, prompt=9000, room=600, pages=1200, seed=43)
    trees = DraftTrees(x.pool, 20)
    x.append(33)
    parent = np.array([[-1, 0, 1, -1, 3, 4, 0, 6, 7, 2, 9, 5, 11, 12, 13, -1, 15, 16, 17, 18]] * 3)
    q, k, v = (x.rand(3, 20, h, 128) for h in (16, 4, 4))
    bad = v.clone()
    bad[:, 4, :, 3] = float("nan")
    bad[:, 6] = float("inf")
    out = trees.attention(0, q, k, bad, x.ints(parent), x.scale)
    assert x.pool.status() == 0
    sees = seen(parent[0], 0)
    for s in range(2):
        K, V = (torch.cat([c[0], y[s]]) for c, y in zip(x.ctx[s], (k, v)))
        o, a = attend_tree(q[s], K, V, x.scale, seen(parent[s], K.shape[0] - 20))
        nan, inf = sees[:, 4], sees[:, 6]
        want = torch.zeros_like(out[s], dtype=torch.bool)
        want[nan, :, 3] = True
        want[inf] = True
        assert torch.equal(~out[s].isfinite(), want)
        assert bool((((out[s].double() - o).abs() <= bound(o, a, "bf16")) | want).all())


@pytest.mark.parametrize("lengths", [[700, 33, 1, 129, 900, 64], [4000, 90]])
def test_rows_behind_a_sequence(cuda, lengths):
    """Padding behind each sequence of a batch: whatever it holds, the same bits in the same time (within a factor of 3, and
    a millisecond for the padding's own rows, which are not finite; row by row it took some 100 times as long)."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    pad = 37
    total = sum(lengths) + pad * len(lengths)
    q, k, v = make("bf16", total, 16, 4, 44)
    cu, past, at = [0], torch.ones(total, dtype=torch.bool, device="cuda"), 0
    for n in lengths:                          # a sequence, then its padding as a sequence of its own, whose results nobody wants
        past[at:at + n] = False
        cu += [at + n, at + n + pad]
        at += n + pad
    op = PromptAttention(16, 4, 128, "bf16", max_tokens=total, max_seqs=2 * len(lengths))
    at = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, times = [], []
    for fill in (0.0, float("nan"), float("-inf")):
        v[past] = fill
        out.append(op(q, k, v, at, 1 / math.sqrt(128))[~past])
        times.append(milliseconds(lambda: op(q, k, v, at, 1 / math.sqrt(128))))
    assert op.status() == 0
    assert all(torch.equal(o, out[0]) for o in out) and bool(out[0].isfinite().all())
    assert max(times) < 3 * times[0] + 1, times


def test_scores_of_minus_infinity_first(cuda):
    """Rows whose first keys all score minus infinity, answered anew because of a later token: those keys weigh nothing."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    n, low, at = 300, 50, 200
    q, k, v = make("bf16", n, 8, 2, 45)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    k[:low, :, 0] = float("-inf")
    v[at, 1] = float("nan")
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=n, max_seqs=1)
    out = op(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), 1 / math.sqrt(128))
    assert op.status() == 0
    want = torch.zeros_like(out, dtype=torch.bool)
    want[:low] = True                          # nothing but minus infinity
    want[at:, 4:] = True                       # the heads that see the NaN
    assert torch.equal(out.isnan(), want)
    rows = [low, low + 1, 127, 128, 180, at - 1]
    vv = v.clone()
    vv[at, 1] = 0
    o, a = rows_of(q[:, :, :], k, vv, rows, 1 / math.sqrt(128))
    assert bool(((out[rows].double() - o).abs() <= bound(o, a, "bf16")).all())


def test_nan_within_and_behind(cuda):
    """Rows that are not finite by a token they see are not answered anew for what lies behind their sequence."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    n = 8000
    q, k, v = make("bf16", n + 40, 16, 4, 46)
    op = PromptAttention(16, 4, 128, "bf16", max_tokens=n + 40, max_seqs=1)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    times = []
    for at in ([], [0], [0, n]):
        for i in at:
            v[i:n + 40 if i else 1] = float("nan")
        times.append(milliseconds(lambda: op(q, k, v, cu, 1 / math.sqrt(128), out)))
    assert op.status() == 0 and not bool(out[:n].isfinite().any())
    assert times[2] < times[1] + 1, times
