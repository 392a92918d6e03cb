"""Every key counts once: queries of zero weigh all keys a row sees alike, and V has a single 1 a key, in the column that the key's
place gives.  A result is then a count of keys over their number, every sum on the way is exact, and the only error is the result's
rounding (bf16 2^-8 of the value, fp32 a few 2^-24); a key left out or taken twice moves a column by 1 of its keys: at least 1 in
128 where a column has up to 128.

Long prompts and contexts, runs split over units, and the sizes at which prompts change from half units to whole ones, which are
also compared with random values in 64 bits."""
import math

import numpy as np
import pytest

from tests.test_gpu_draft import Trees, seen
from tests.test_gpu_prompt import attend, bound, make

pytestmark = pytest.mark.gpu


def few_tokens(hq, hkv):
    """The longest single prompt that takes half units: one and a half units an SM."""
    import torch
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return 3 * sms // (2 * hkv) * (256 * hkv // hq)


def column(i, d, by):
    """Keys by turns, or in runs of d."""
    return i % d if by == "turns" else i // d % d


def limit(o, dtype):
    return o * (2.0 ** -8 + 1e-6) if dtype == "bf16" else o * 1e-6


@pytest.mark.parametrize("by", ["turns", "runs"])
@pytest.mark.parametrize("hq,hkv,dtype", [(32, 8, "bf16"), (8, 2, "bf16"), (8, 8, "bf16"), (64, 8, "bf16"), (16, 1, "bf16"), (4, 2, "f32")])
def test_long_prompts(cuda, hq, hkv, dtype, by):
    """All rows of one prompt below, at and above the change of unit, and of a packed batch."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    edge = few_tokens(hq, hkv) if dtype == "bf16" else 700
    lengths = [[edge - 1], [edge], [edge + 1], [min(2 * edge + 77, 15001)], [2001], [edge // 2 + 3, 1, 130, edge // 3, 0, 64, 700, 2000]]
    d = 128 if dtype == "bf16" else 64
    for case in lengths:
        cu = np.concatenate([[0], np.cumsum(case)])
        n = int(cu[-1])
        q, k, v = make(dtype, n, hq, hkv, 51)
        q.zero_()
        v.zero_()
        i = torch.arange(n, device="cuda")
        v[i, :, column(i, d, by)] = 1
        op = PromptAttention(hq, hkv, d, dtype, max_tokens=n, max_seqs=len(case))
        out = op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1)
        assert op.status() == 0
        for s, e in zip(cu, cu[1:]):
            count = v[s:e, 0].double().cumsum(0) / torch.arange(1, e - s + 1, device="cuda")[:, None]
            err = (out[s:e].double() - count[:, None]).abs()
            assert bool((err <= limit(count, dtype)[:, None]).all()), (case, s, float(err.max()))


class Marked(Trees):
    """Contexts whose V are marks: a key's column is its place in the order of writing, moved by its slot."""
    by, written, turn = "turns", 0, False

    def rand(self, *shape):
        import torch
        x = super().rand(*shape)
        self.turn = not self.turn            # K, then V
        if not self.turn:
            i = self.written + torch.arange(shape[1], device="cuda")
            self.written += shape[1]
            x.zero_()
            if len(shape) == 4:
                x[:, torch.arange(shape[1]), :, column(i, self.d, self.by)] = 1
            else:
                for s in range(shape[2]):
                    x[:, torch.arange(shape[1]), s, :, column(i + 5 * s, self.d, self.by)] = 1
        return x


@pytest.mark.parametrize("by", ["turns", "runs"])
@pytest.mark.parametrize("dtype,beams,prompt,t,hq,hkv,page,grown", [
    ("bf16", 1, 9000, 4, 32, 8, 16, (70, 1)), ("bf16", 1, 15800, 1, 32, 8, 16, (3, 60)), ("bf16", 2, 5000, 64, 16, 2, 64, (70, 40)),
    ("bf16", 40, 700, 16, 16, 2, 16, (130, 200)), ("bf16", 64, 2000, 12, 32, 8, 32, (513, 130)), ("bf16", 130, 300, 3, 8, 2, 16, (70, 40)),
    ("f32", 2, 6000, 5, 4, 2, 16, (50, 7)), ("f32", 5, 100, 33, 8, 2, 32, (200, 31))])
def test_long_contexts(cuda, dtype, beams, prompt, t, hq, hkv, page, grown, by):
    """Contexts in long runs that are split, shared or a beam's own, with pages, tiles and pieces that end anywhere."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    kind = type("Kind", (Marked,), dict(by=by))
    room = (prompt + sum(grown)) // page + 8
    x = kind(dtype, hq=hq, hkv=hkv, slots=beams + 1, beams=beams, prompt=prompt, page=page, room=room,
             pages=room + (sum(grown) // page + 8) * (beams + 1) * 2, seed=52)
    trees = DraftTrees(x.pool, t)
    for step, n in enumerate(grown):
        x.append(n)
        parent, count = x.trees(t, step == 0)
        count = np.maximum(count, 1)
        q = torch.zeros(x.slots, t, hq, x.d, dtype=x.dt, device="cuda")
        k = Trees.rand(x, x.slots, t, hkv, x.d)
        v = torch.zeros(x.slots, t, hkv, x.d, dtype=x.dt, device="cuda")
        i = torch.arange(t, device="cuda")
        v[:, i, :, i % x.d] = 1
        out = trees.attention(0, q, k, v, x.ints(parent), x.scale, count=x.ints(count))
        assert x.pool.status() == 0
        for s in range(x.slots):
            if x.ctx[s] is None:
                assert not bool(out[s].any())
                continue
            c = int(count[s])
            V = torch.cat([x.ctx[s][1][0], v[s, :c]])[:, 0].double()
            sees = seen(parent[s, :c], V.shape[0] - c).double()
            want = (sees @ V / sees.sum(1, keepdim=True))[:, None]
            err = (out[s, :c].double() - want).abs()
            assert bool((err <= limit(want, dtype)).all()), (s, float(err.max()))
        x.fork([0] * (beams // 2) + list(range(beams // 2, beams)) + [-1] if beams > 1 and step == 0 else list(range(beams)) + [-1])


def chunked(q, k, v, scale, rows=512):
    """attend of one causal sequence, its rows in chunks."""
    import torch
    n, g = q.shape[0], q.shape[1] // k.shape[1]
    o, a = [], []
    kk, vv = (x.double().repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))
    for r in range(0, n, rows):
        x = q[r:r + rows].double().transpose(0, 1) @ kk[:, :r + rows].transpose(1, 2) * scale
        i = torch.arange(r, min(r + rows, n), device=q.device)
        x.masked_fill_(torch.arange(x.shape[2], device=q.device)[None] > i[:, None], -math.inf)
        p = torch.softmax(x, -1)
        o.append((p @ vv[:, :r + rows]).transpose(0, 1))
        a.append((p @ vv[:, :r + rows].abs()).transpose(0, 1))
    return torch.cat(o), torch.cat(a)


@pytest.mark.parametrize("hq,hkv,n", [(32, 8, 2001), (8, 2, 7400), (8, 8, 7301), (64, 8, 1111), (32, 2, 1999), (16, 1, 5003)])
def test_whole_units_of_one_prompt(cuda, hq, hkv, n):
    """Single prompts past the change of unit, several units a CTA, random values."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    assert n > few_tokens(hq, hkv)
    q, k, v = make("bf16", n, hq, hkv, 53)
    op = PromptAttention(hq, hkv, 128, "bf16", max_tokens=n, max_seqs=1)
    out = op(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), 1 / math.sqrt(128))
    assert op.status() == 0
    o, a = chunked(q, k, v, 1 / math.sqrt(128))
    assert bool(((out.double() - o).abs() <= bound(o, a, "bf16")).all())


def test_many_whole_units(cuda):
    """A packed batch whose units are whole ones, against the definition."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    cu = [0]
    for i in range(70):
        cu.append(cu[-1] + 37 * (1 + i % 9))
    q, k, v = make("bf16", cu[-1], 8, 2, 15)
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=cu[-1], max_seqs=70)
    out = op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1)
    assert op.status() == 0
    o, a = attend(q, k, v, cu, 0.1)
    assert bool(((out.double() - o).abs() <= bound(o, a, "bf16")).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cu,kept", [([0, 100, 90, 200, 300], [(0, 100), (200, 300)]), ([-5, 100, 200, 300, 400], [(100, 200), (200, 300)]),
                                     ([0, 301, 50, 300], [(50, 300)]), ([300, 0, 100, 100, 200], [])])
def test_sequences_that_are_left_out(cuda, cu, kept, dtype):
    """Out of range, out of order, or begun before an earlier bound: their rows stay as they were, the others are computed."""
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make(dtype, 300, 4, 2, 10)
    op = PromptAttention(4, 2, q.shape[2], dtype, max_tokens=300, max_seqs=len(cu) - 1)
    out = torch.full_like(q, 7.0)
    op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1, out)
    assert B.STATUS_NAMES[op.status()] == "GB_ERR_INVALID"
    left = torch.ones(300, dtype=torch.bool, device="cuda")
    for s, e in kept:
        o, a = attend(q, k, v, [s, e], 0.1)
        assert bool(((out.double() - o).abs() <= bound(o, a, dtype))[s:e].all()), (s, e)
        left[s:e] = False
    assert bool((out[left] == 7).all())
