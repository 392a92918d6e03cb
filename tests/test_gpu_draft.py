"""Trees of drafted tokens: their attention against the definition in 64 bits, accepting and cutting against the
pool's plain-Python model, and whole rounds of both with decode steps, forks and tournaments between them.

Bounds, elementwise, with A = sum_j p_j |v_j|: as for prompts, bf16 rounds each p and the result by at most 2^-8 of
the value, fp32 sums and exponentials add 2e-5 A; fp32 pools 4e-5 A."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


class Trees:
    """A pool beside copies of every slot's context (K, V [layers][tokens][Hkv][D]) and the page model."""

    def __init__(self, dtype="bf16", layers=1, hq=8, hkv=2, page=16, slots=6, beams=4, prompt=40, room=40, pages=None, seed=0):
        import torch
        from oracle.pool import PoolOracle
        from paper_2608_08020_gb300.pool import BeamPool, TORCH_DT
        self.dt, self.dtype, self.layers, self.hq, self.hkv = TORCH_DT[dtype], dtype, layers, hq, hkv
        self.d, self.slots = 128 if dtype == "bf16" else 64, slots
        self.scale = 1 / math.sqrt(self.d)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        pages = pages or slots * room
        self.pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=self.d, page_size=page,
                             kv_dtype=dtype, num_pages=pages, max_beams=slots, max_pages_per_beam=room)
        self.pool.kv.fill_(0xFF)          # NaN wherever no token has been written
        self.model = PoolOracle(pages, slots, room, page)
        kv = [self.rand(layers, prompt, hkv, self.d) for _ in range(2)]
        self.pool.seed(beams, prompt, *kv)
        self.model.seed(beams, prompt)
        self.ctx = [tuple(kv) if s < beams else None for s in range(slots)]

    def rand(self, *shape):
        import torch
        return torch.randn(shape, generator=self.g, device="cuda").to(self.dt)

    def ints(self, x):
        import torch
        return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

    def append(self, n):
        import torch
        k, v = (self.rand(self.layers, n, self.slots, self.hkv, self.d) for _ in range(2))
        for layer in range(self.layers):
            self.pool.append_kv(layer, n, k[layer], v[layer])
        for s, c in enumerate(self.ctx):
            if c is not None:
                self.ctx[s] = tuple(torch.cat([a, x[:, :, s]], 1) for a, x in zip(c, (k, v)))
        for _ in range(n):
            assert self.model.begin_step()

    def decode(self):
        import torch
        k, v = (self.rand(self.layers, self.slots, self.hkv, self.d) for _ in range(2))
        q = self.rand(self.layers, self.slots, self.hq, self.d)
        out = torch.empty(self.slots, self.hq, self.d, device="cuda")
        assert self.model.begin_step()
        for s, c in enumerate(self.ctx):
            if c is not None:
                self.ctx[s] = tuple(torch.cat([a, x[:, s, None]], 1) for a, x in zip(c, (k, v)))
        for layer in range(self.layers):
            self.pool.decode_attention(layer, q[layer], k[layer], v[layer], self.scale, out)
            for s, c in enumerate(self.ctx):
                if c is not None:
                    o, a = attend(q[layer, s, None], c[0][layer], c[1][layer], self.scale)
                    assert bool(((out[s].double() - o[0]).abs() <= bound(o, a, self.dtype)[0]).all())

    def fork(self, parents):
        self.pool.fork_slots(self.ints(parents))
        self.model.fork_slots(parents)
        self.ctx = [None if p < 0 and self.ctx[s] is None else self.ctx[p if p >= 0 else s] for s, p in enumerate(parents)]

    def release(self, slots):
        self.pool.release(self.ints(slots))
        self.model.release(slots)
        for s in slots:
            self.ctx[s] = None

    def truncate(self, lengths):
        self.pool.truncate(self.ints(lengths))
        if self.model.truncate(lengths):
            for s, n in enumerate(lengths):
                if self.ctx[s] is not None and 0 <= n <= self.ctx[s][0].shape[1]:
                    self.ctx[s] = tuple(x[:, :n] for x in self.ctx[s])

    def trees(self, t, ragged):
        i = np.arange(t)
        other = self.rng.integers(0, 1 << 30, (self.slots, t)) % (i + 1) - 1
        parent = np.where(self.rng.random((self.slots, t)) < 0.6, i - 1, other)
        count = self.rng.integers(0, t + 1, self.slots) if ragged else np.full(self.slots, t)
        return parent, count

    def attention(self, trees, t, ragged=True, poison=True, check=True):
        """One round of attention; returns what accept takes."""
        import torch
        parent, count = self.trees(t, ragged)
        q = self.rand(self.layers, self.slots, t, self.hq, self.d)
        k, v = (self.rand(self.layers, self.slots, t, self.hkv, self.d) for _ in range(2))
        if poison:                        # rows that hold no token
            for s in range(self.slots):
                n = 0 if self.ctx[s] is None else int(count[s])
                for x in (q, k, v):
                    x[:, s, n:] = float("nan")
        dp, dc = self.ints(parent), self.ints(count) if ragged else None
        for layer in range(self.layers):
            out = torch.full((self.slots, t, self.hq, self.d), 7.0, dtype=self.dt, device="cuda")
            assert trees.attention(layer, q[layer], k[layer], v[layer], dp, self.scale, out, count=dc) is out
            for s in range(self.slots):
                n = 0 if self.ctx[s] is None else int(count[s])
                assert not bool(out[s, n:].any()), (layer, s)
                if n and check:
                    self.check(out[s, :n], q[layer, s, :n], s, layer, k[layer, s, :n], v[layer, s, :n], parent[s, :n])
        return parent, count, k, v, dp, dc

    def check(self, out, q, s, layer, k, v, parent):
        import torch
        K, V = (torch.cat([c[layer], x]) for c, x in zip(self.ctx[s], (k, v)))
        o, a = attend(q, K, V, self.scale, seen(parent, K.shape[0] - len(parent)))
        err, lim = (out.double() - o).abs(), bound(o, a, self.dtype)
        assert bool((err <= lim).all()), (layer, s, float((err / lim).nan_to_num(9e9).max()))

    def accept(self, trees, rnd, accepted):
        import torch
        parent, count, k, v, dp, dc = rnd
        n, path = trees.accept(k, v, dp, self.ints(accepted), count=dc)
        paths = []
        for s in range(self.slots):
            p, i = [], int(accepted[s]) if self.ctx[s] is not None else -1
            while i >= 0:
                p.insert(0, i)
                i = int(parent[s, i])
            paths.append(p)
        if not self.model.accept([len(p) for p in paths]):
            paths = [[] for _ in paths]
        assert n.tolist() == [len(p) for p in paths]
        assert path.tolist() == [p + [-1] * (parent.shape[1] - len(p)) for p in paths]
        for s, p in enumerate(paths):
            if p:
                self.ctx[s] = tuple(torch.cat([c, x[:, s, p]], 1) for c, x in zip(self.ctx[s], (k, v)))

    def pick(self, rnd):
        parent, count = rnd[:2]
        return [-1 if c == 0 or self.rng.random() < 0.15 else int(self.rng.integers(c)) for c in count]

    def same_pages(self):
        st, m = self.pool.read_state(), self.model
        assert st["seq_len"].tolist() == m.seq_len.tolist() and st["active"].tolist() == m.active.astype(int).tolist()
        assert st["gen"].tolist() == m.gen.tolist()
        assert st["refcnt"].tolist() == m.refcnt.tolist() and np.array_equal(st["free_bits"], m.free_bits())
        for s in np.flatnonzero(m.active):
            assert st["tables"][s, :len(m.tables[s])].tolist() == m.tables[s], s
        m.check_invariants()


def seen(parent, before):
    """[tokens][before + tokens]: the context, the token itself and its ancestors."""
    import torch
    n = len(parent)
    m = torch.zeros(n, before + n, dtype=torch.bool)
    m[:, :before] = True
    for i in range(n):
        j = i
        while j >= 0:
            m[i, before + j] = True
            j = int(parent[j])
    return m.cuda()


def attend(q, k, v, scale, sees=None):
    """(softmax(scale q.k) v, the same of |v|) in 64 bits: q [rows][hq][d] over k, v [keys][hkv][d]."""
    import torch
    g = q.shape[1] // k.shape[1]
    kk, vv = (x.double().repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))
    x = q.double().transpose(0, 1) @ kk.transpose(1, 2) * scale
    if sees is not None:
        x = x.masked_fill(~sees, -math.inf)
    p = torch.softmax(x, -1)
    return (p @ vv).transpose(0, 1), (p @ vv.abs()).transpose(0, 1)


def bound(o, a, dtype):
    return (a + o.abs()) * 2.0 ** -8 + 2e-5 * a if dtype == "bf16" else 4e-5 * a


def both(*cases):
    return [(d, *c) for d in ("f32", "bf16") for c in cases]


@pytest.mark.parametrize("dtype,t", both((1,), (2,), (7,), (16,), (33,), (64,)))
def test_tree_sizes(cuda, dtype, t):
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, seed=t)
    trees = DraftTrees(x.pool, t)
    for ragged in (False, True):
        x.attention(trees, t, ragged)
    assert x.pool.status() == 0
    x.same_pages()


@pytest.mark.parametrize("dtype,prompt", both((1,), (15,), (16,), (63,), (64,), (65,), (127,), (128,), (129,), (190,), (257,), (1000,)))
def test_context_lengths(cuda, dtype, prompt):
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, prompt=prompt, room=70, page=16 if prompt % 2 else 64, seed=prompt)
    trees = DraftTrees(x.pool, 9)
    x.attention(trees, 9)
    x.fork([0, 1, 1, 3, 0, 3])
    x.append(3)
    x.attention(trees, 9)
    x.append(130)
    x.fork([0, 1, 2, 3, 1, 1])
    x.append(20)
    x.attention(trees, 9)
    assert x.pool.status() == 0
    x.same_pages()


@pytest.mark.parametrize("dtype,hq,hkv,page", both((4, 2, 16), (16, 2, 32), (8, 4, 64), (32, 8, 16), (8, 1, 32)))
def test_head_layouts_and_pages(cuda, dtype, hq, hkv, page):
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, layers=2, hq=hq, hkv=hkv, page=page, slots=20, beams=16, prompt=100, seed=hq)
    trees = DraftTrees(x.pool, 12)
    x.append(77)
    x.fork([0, 1, 2, 3, 4, 5, 6, 7, 0, 1, 2, 3, 4, 5, 6, 7, 0, 0, 1, 7])
    x.append(150)
    x.release([3, 9])
    x.attention(trees, 12)
    assert x.pool.status() == 0


@pytest.mark.parametrize("beams,prompt,t,hq,hkv", [(1, 9000, 4, 32, 8), (2, 5000, 64, 16, 2), (40, 700, 16, 16, 2),
                                                   (130, 300, 3, 8, 2), (1, 20000, 1, 8, 4)])
def test_split_runs_and_many_sharers(cuda, beams, prompt, t, hq, hkv):
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", hq=hq, hkv=hkv, slots=beams + 1, beams=beams, prompt=prompt, room=prompt // 16 + 20,
              pages=prompt // 16 + 30 * (beams + 1), seed=beams)
    trees = DraftTrees(x.pool, t)
    x.append(70)
    x.attention(trees, t)
    x.fork([0] * (beams // 2) + list(range(beams // 2, beams)) + [-1] if beams > 1 else [0, 0])
    x.append(40)
    x.attention(trees, t)
    assert x.pool.status() == 0


def test_long_fp32(cuda):
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("f32", hq=4, hkv=2, slots=3, beams=2, prompt=6000, room=400, pages=800, seed=1)
    trees = DraftTrees(x.pool, 5)
    x.append(50)
    x.attention(trees, 5)
    assert x.pool.status() == 0


@pytest.mark.parametrize("dtype,layers,page,t", both((1, 16, 1), (3, 16, 8), (2, 32, 20), (2, 64, 64), (1, 16, 64)))
def test_rounds(cuda, dtype, layers, page, t):
    """Whole rounds: attention, accept, decode steps, forks, releases, cuts; every call against the model."""
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, layers=layers, page=page, slots=7, beams=5, prompt=37, room=60, seed=t)
    trees = DraftTrees(x.pool, t)
    for step in range(6):
        rnd = x.attention(trees, t, ragged=step != 1)
        x.accept(trees, rnd, x.pick(rnd))
        x.same_pages()
        if step == 1:
            x.fork([0, 1, 2, 3, 4, 2, 0])
        if step == 2:
            x.decode()
        if step == 3:
            x.release([1])
            x.fork([0, 4, 2, 3, 4, 5, 6])
            x.same_pages()
        if step == 4:
            x.truncate([-1 if c is None else max(0, c[0].shape[1] - int(x.rng.integers(0, 30))) for c in x.ctx])
            x.same_pages()
    x.decode()
    x.attention(trees, t)
    assert x.pool.status() == 0
    x.same_pages()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cuts(cuda, dtype):
    """Cuts at and inside pages, shared and not: every holder inside a page, some, one; to zero; none."""
    from paper_2608_08020_gb300.draft import DraftTrees
    for i, lengths in enumerate(([35, 36, 37, 38, 39, 40], [35] * 6, [-1, 35, 35, -1, 48, 33], [0, -1, 16, 0, 1, 32],
                                 [-1] * 6, [200, 201, 202, 40, 41, -1], [250, 250, 250, 250, 250, 36])):
        x = Trees(dtype, layers=2, slots=6, beams=3, prompt=70, room=30, seed=i)
        trees = DraftTrees(x.pool, 6)
        x.append(130)
        x.fork([0, 1, 2, 0, 1, 0])
        x.append(50)
        x.truncate(lengths)
        x.same_pages()
        x.attention(trees, 6)
        x.decode()
        rnd = x.attention(trees, 6)
        x.accept(trees, rnd, x.pick(rnd))
        x.same_pages()
        x.attention(trees, 6)
        assert x.pool.status() == 0


def test_cut_to_the_fork(cuda):
    """Children cut back to their fork, inside their parents' pages, then grown again."""
    x = Trees("bf16", slots=8, beams=2, prompt=20, room=40, seed=3)
    x.append(200)
    x.fork([0, 1, 0, 1, 0, 1, 0, 1])
    for n in (3, 40):
        x.append(n)
    x.truncate([-1, 100, 100, 220, -1, 215, 101, 3])
    x.same_pages()
    for _ in range(3):
        x.decode()
    x.append(17)
    x.same_pages()
    assert x.pool.status() == 0


def test_values_out_of_sight(cuda):
    """Infinities and NaN in drafted tokens reach their descendants only."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    for dtype in ("bf16", "f32"):
        x = Trees(dtype, slots=2, beams=2, prompt=150, seed=8)
        trees = DraftTrees(x.pool, 4)
        q = x.rand(2, 4, x.hq, x.d)
        k, v = x.rand(2, 4, x.hkv, x.d), x.rand(2, 4, x.hkv, x.d)
        parent = np.array([[-1, 0, -1, 2]] * 2)
        bad = v.clone()
        bad[0, 1, :, 5] = float("inf")
        bad[0, 1, :, x.d - 3] = float("nan")
        kb = k.clone()
        kb[1, 2] = float("nan")
        out = trees.attention(0, q, kb, bad, x.ints(parent), x.scale)
        for s in (0, 1):
            for i in range(4):
                anc = [j for j in range(4) if j == i or (i == 1 and j == 0) or (i == 3 and j == 2)]
                K, V = (torch.cat([c[0], y[s, anc]]) for c, y in zip(x.ctx[s], (kb, bad)))
                o, a = attend(q[s, i, None], K, V, x.scale)
                ok = o.isfinite()
                assert torch.equal(out[s, i].isfinite(), ok[0]), (dtype, s, i)
                err = (out[s, i, None].double() - o).abs()
                assert bool((err <= bound(o, a, dtype))[ok].all()), (dtype, s, i)


def test_device_errors(cuda):
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", slots=3, beams=2, prompt=30, room=4, pages=9, seed=2)
    trees = DraftTrees(x.pool, 4)
    q, k, v = x.rand(3, 4, x.hq, x.d), x.rand(1, 3, 4, x.hkv, x.d), x.rand(1, 3, 4, x.hkv, x.d)
    chain = x.ints([[-1, 0, 1, 2]] * 3)

    def status():
        st = x.pool.status()
        x.pool.clear_status()
        return B.STATUS_NAMES[st]

    for parent, count in (([[-1, 1, 0, 0]] * 3, None), ([[-1, -2, 0, 0]] * 3, None), ([[-1, 0, 1, 2]] * 3, [4, 5, 0]),
                          ([[-1, 0, 1, 2]] * 3, [-1, 4, 4])):
        trees.attention(0, q, k[0], v[0], x.ints(parent), x.scale, count=None if count is None else x.ints(count))
        assert status() == "GB_ERR_INVALID"
    # Vacant slots are not looked at.
    trees.attention(0, q, k[0], v[0], x.ints([[-1, 0, 1, 2]] * 2 + [[9, 9, 9, 9]]), x.scale, count=x.ints([4, 4, 99]))
    assert status() == "GB_OK"
    for accepted, n in (([4, 1, 0], [0, 2, 0]), ([-2, 3, 0], [0, 4, 0])):
        before = x.pool.read_state()["seq_len"].tolist()
        got, path = trees.accept(k, v, chain, x.ints(accepted))
        assert got.tolist() == n and status() == "GB_ERR_INVALID"
        assert x.pool.read_state()["seq_len"].tolist() == [a + b for a, b in zip(before, n)]
    x.pool.truncate(x.ints([30, 30, 5]))
    assert status() == "GB_OK"
    x.pool.truncate(x.ints([31, 29, 0]))
    assert status() == "GB_ERR_INVALID"
    assert x.pool.read_state()["seq_len"].tolist() == [30, 29, 0]


def test_out_of_pages(cuda):
    """Without the pages for every slot nothing is accepted, and nothing is cut that would need a copy."""
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", slots=4, beams=4, prompt=64, room=8, pages=7, seed=2)
    trees = DraftTrees(x.pool, 4)
    rnd = x.attention(trees, 4, ragged=False)
    x.accept(trees, rnd, [3, 3, 3, 3])              # three free pages for four slots
    assert x.pool.status() == 2
    x.pool.clear_status()
    x.same_pages()
    x.accept(trees, rnd, [3, -1, 3, 0])
    x.same_pages()
    x.truncate([40, -1, -1, -1])                    # inside a page of four holders, and none free
    assert x.pool.status() == 2
    x.pool.clear_status()
    x.same_pages()
    x.truncate([48, -1, -1, -1])
    x.truncate([40, -1, -1, -1])
    assert x.pool.status() == 0
    x.same_pages()
    rnd = x.attention(trees, 4, ragged=False)
    full = Trees("bf16", slots=2, beams=1, prompt=30, room=2, pages=9, seed=2)
    trees = DraftTrees(full.pool, 4)
    rnd = full.attention(trees, 4, ragged=False)
    full.accept(trees, rnd, [3, -1])                # the block table has room for two tokens
    assert full.pool.status() == 2
    full.same_pages()


def test_order_of_calls(cuda):
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=2, seed=4)
    trees = DraftTrees(x.pool, 4)
    q, k, v = x.rand(x.slots, 4, x.hq, x.d), x.rand(x.slots, 4, x.hkv, x.d), x.rand(x.slots, 4, x.hkv, x.d)
    parent = x.ints([[-1, 0, 1, 2]] * x.slots)

    def refused(layer, t=trees):
        with pytest.raises(B.GambitError) as e:
            t.attention(layer, q, k, v, parent, x.scale)
        return "GB_ERR_STATE" in str(e.value)

    assert refused(1)
    a = trees.attention(0, q, k, v, parent, x.scale)
    trees.attention(1, q, k, v, parent, x.scale)
    assert torch.equal(trees.attention(0, q, k, v, parent, x.scale), a)
    trees.attention(1, q, k, v, parent, x.scale)
    assert refused(1, DraftTrees(x.pool, 4))        # another workspace has no plan
    x.append(1)
    assert refused(1)
    x.pool.append_kv(0, 1, x.rand(1, x.slots, x.hkv, x.d), x.rand(1, x.slots, x.hkv, x.d))
    assert refused(0)                               # inside an open step
    with pytest.raises(B.GambitError):
        x.pool.truncate(x.ints([0] * x.slots))
    x.pool.append_kv(1, 1, x.rand(1, x.slots, x.hkv, x.d), x.rand(1, x.slots, x.hkv, x.d))
    trees.attention(0, q, k, v, parent, x.scale)
    x.fork([0, 1, 2, 3, 0, 1])
    assert refused(1)


def test_graph(cuda):
    """A round captured and replayed on another stream, the pool growing and forking between the replays."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=2, slots=5, beams=4, prompt=200, room=60, seed=6)
    t = 6
    trees = DraftTrees(x.pool, t)
    parent, count = x.trees(t, False)
    dp, acc = x.ints(parent), x.ints([0] * 5)
    q = x.rand(2, 5, t, x.hq, x.d)
    k, v = x.rand(2, 5, t, x.hkv, x.d), x.rand(2, 5, t, x.hkv, x.d)
    out = [torch.empty_like(q[0]) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        trees.attention(0, q[0], k[0], v[0], dp, x.scale, out[0])    # what a first call sets up is not captured
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for layer in range(2):
            trees.attention(layer, q[layer], k[layer], v[layer], dp, x.scale, out[layer])
        n, path = trees.accept(k, v, dp, acc)
    for step in range(4):
        parent, count = x.trees(t, False)
        for y in (q, k, v):
            y.copy_(x.rand(*y.shape))
        picked = x.pick((parent, count))
        dp.copy_(x.ints(parent))
        acc.copy_(x.ints(picked))
        graph.replay()
        torch.cuda.synchronize()
        for layer in range(2):
            for s in range(5):
                if x.ctx[s] is not None:
                    x.check(out[layer][s], q[layer, s], s, layer, k[layer, s], v[layer, s], parent[s])
        paths = []
        for s in range(5):
            p, i = [], picked[s] if x.ctx[s] is not None else -1
            while i >= 0:
                p.insert(0, i)
                i = int(parent[s, i])
            paths.append(p)
        assert x.model.accept([len(p) for p in paths]) and n.tolist() == [len(p) for p in paths]
        for s, p in enumerate(paths):
            if p:
                x.ctx[s] = tuple(torch.cat([c, y[:, s, p]], 1) for c, y in zip(x.ctx[s], (k, v)))
        x.same_pages()
        if step == 1:
            x.fork([0, 1, 2, 3, 2])
        if step == 2:
            x.append(20)
    assert x.pool.status() == 0


def test_refusals(cuda):
    """Bad arguments fail on the host, with the pool's reason, before anything is enqueued."""
    import ctypes
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=2, seed=5)
    t, lib = DraftTrees(x.pool, 4), B.load()
    q, k, v, out = x.rand(x.slots, 4, x.hq, x.d), x.rand(2, x.slots, 4, x.hkv, x.d), x.rand(2, x.slots, 4, x.hkv, x.d), x.rand(x.slots, 4, x.hq, x.d)
    parent, acc, launches = x.ints([[-1, 0, 1, 2]] * x.slots), x.ints([0] * x.slots), B.gb_pool_launch_count(x.pool.handle)
    base = dict(parent_dev=parent.data_ptr(), count_dev=None, workspace_dev=t.workspace.data_ptr(),
                workspace_bytes=t.workspace.numel(), n_draft=4)

    def attention(layer=0, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), scale=0.1, out=out.data_ptr(), **kw):
        return B.STATUS_NAMES[lib.gb_draft_attention(x.pool.handle, layer, ctypes.byref(B.GbDraft(**{**base, **kw})), q, k, v,
                                                     scale, out, None)]

    def accept(k=k.data_ptr(), v=v.data_ptr(), a=acc.data_ptr(), **kw):
        return B.STATUS_NAMES[lib.gb_accept_draft(x.pool.handle, ctypes.byref(B.GbDraft(**{**base, **kw})), k, v, a, None,
                                                  None, None)]

    for kw in (dict(n_draft=0), dict(n_draft=65), dict(parent_dev=None), dict(workspace_dev=None),
               dict(workspace_dev=t.workspace.data_ptr() + 16), dict(workspace_bytes=t.workspace.numel() - 1), dict(n_draft=5)):
        assert attention(**kw) == accept(**kw) == "GB_ERR_INVALID", kw
    for kw in (dict(layer=-1), dict(layer=2), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=q.data_ptr() + 8),
               dict(k=k.data_ptr() + 2), dict(out=out.data_ptr() + 16), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(out=q.data_ptr()), dict(out=k.data_ptr() + 256)):
        assert attention(**kw) == "GB_ERR_INVALID", kw
    for kw in (dict(k=None), dict(v=None), dict(a=None), dict(v=v.data_ptr() + 4)):
        assert accept(**kw) == "GB_ERR_INVALID", kw
    assert attention(layer=1) == "GB_ERR_STATE"
    assert B.STATUS_NAMES[lib.gb_truncate(x.pool.handle, None, None)] == "GB_ERR_INVALID"
    n = ctypes.c_size_t()
    for tokens in (0, 65):
        assert lib.gb_draft_workspace_bytes(x.pool.handle, tokens, ctypes.byref(n)) == B.GB_ERR_INVALID
    assert lib.gb_draft_workspace_bytes(None, 4, ctypes.byref(n)) == B.GB_ERR_INVALID
    assert B.gb_pool_launch_count(x.pool.handle) == launches and x.pool.status() == 0
    for bad in (dict(q=q[:, :2]), dict(q=q.float()), dict(k=k[0].transpose(0, 1)), dict(parent=parent.long()),
                dict(parent=parent[:, :3]), dict(count=acc[:2]), dict(out=out[:2])):
        with pytest.raises(ValueError):
            t.attention(**{**dict(layer=0, q=q, k=k[0], v=v[0], parent=parent, scale=0.1, out=out), **bad})
    for bad in (dict(k=k[0]), dict(accepted=acc.long()), dict(accepted=acc[:2])):
        with pytest.raises(ValueError):
            t.accept(**{**dict(k=k, v=v, parent=parent, accepted=acc), **bad})
    for bad in (acc.long(), acc[:3], acc.cpu()):
        with pytest.raises(ValueError):
            x.pool.truncate(bad)
    from paper_2608_08020_gb300.pool import BeamPool
    pool = BeamPool(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, kv_dtype="bf16", num_pages=9,
                    max_beams=x.slots, max_pages_per_beam=4)
    u = DraftTrees(pool, 4)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        u.attention(0, q, k[0], v[0], parent, 0.1)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        pool.truncate(acc)


@pytest.mark.parametrize("beams,hq,hkv,t", [(3, 8, 2, 6), (40, 16, 2, 16), (24, 32, 8, 9)])
def test_the_same_each_time(cuda, beams, hq, hkv, t):
    """Segments are found in an order that may differ; the results may not."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", hq=hq, hkv=hkv, slots=beams, beams=beams, prompt=300, room=80, seed=9)
    trees = DraftTrees(x.pool, t)
    for n in (130, 200, 77):
        x.append(n)
        x.fork([b if b % 3 else (b + 1) % beams if (b + 1) % 3 else b for b in range(beams)])
    x.append(50)
    parent, count = x.trees(t, True)
    q, k, v = x.rand(beams, t, hq, 128), x.rand(beams, t, hkv, 128), x.rand(beams, t, hkv, 128)
    out = None
    for _ in range(12):
        got = trees.attention(0, q, k, v, x.ints(parent), x.scale, count=x.ints(count))
        assert out is None or torch.equal(got, out)
        out = got
        x.fork(list(range(beams)))       # nothing moves, the segments are found again
    assert x.pool.status() == 0


@pytest.mark.parametrize("long,short,beams", [(1200, 40, 1000), (1200, 130, 1000), (700, 10, 935), (0, 0, 900), (0, 0, 1024)])
def test_units_of_unequal_lengths(cuda, long, short, beams):
    """Five long beams to an SM, then short ones: pairs whose halves differ, single units behind them (0: lengths drawn)."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    sms, t, room = torch.cuda.get_device_properties(0).multi_processor_count, 8, max(long, 600)
    x = Trees("bf16", hq=8, hkv=1, slots=beams, beams=beams, prompt=1, room=room // 16 + 2, seed=beams)
    trees = DraftTrees(x.pool, t)
    k, v = x.rand(room, beams, 1, 128), x.rand(room, beams, 1, 128)
    x.pool.append_kv(0, room, k, v)
    lengths = np.where(np.arange(beams) < 5 * sms, long, short) if long else x.rng.integers(0, room, beams)
    x.pool.truncate(x.ints(lengths + 1))
    q, dk, dv = x.rand(beams, t, 8, 128), x.rand(beams, t, 1, 128), x.rand(beams, t, 1, 128)
    parent = np.tile(np.arange(t) - 1, (beams, 1))
    parent[::2, 3] = 0
    out = trees.attention(0, q, dk, dv, x.ints(parent), x.scale)
    assert x.pool.status() == 0
    assert torch.equal(out, trees.attention(0, q, dk, dv, x.ints(parent), x.scale))
    sees = torch.zeros(beams, t, 1 + room + t, dtype=torch.bool, device="cuda")
    sees[:, :, 1:1 + room] = (torch.arange(room, device="cuda") < torch.tensor(lengths, device="cuda")[:, None])[:, None]
    sees[:, :, 0] = True
    for kind in (0, 1):
        sees[kind::2, :, 1 + room:] = seen(parent[kind], 0)
    for b in range(0, beams, 100):
        at = slice(b, min(b + 100, beams))
        K, V = (torch.cat([c[0].expand(at.stop - b, -1, -1, -1), y[:, at].transpose(0, 1), d[at]], 1).double()[:, :, 0]
                for c, y, d in zip(x.ctx[0], (k, v), (dk, dv)))
        p = torch.einsum("bthd,bkd->bthk", q[at].double(), K) * x.scale
        p = torch.softmax(p.masked_fill(~sees[at, :, None], -math.inf), -1)
        o, a = torch.einsum("bthk,bkd->bthd", p, V), torch.einsum("bthk,bkd->bthd", p, V.abs())
        err = (out[at].double() - o).abs()
        assert bool((err <= bound(o, a, "bf16")).all()), (b, float((err / bound(o, a, "bf16")).max()))


def test_a_captured_plan_stays_in_its_graph(cuda):
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=2, seed=4)
    trees = DraftTrees(x.pool, 4)
    q, k, v = x.rand(x.slots, 4, x.hq, x.d), x.rand(x.slots, 4, x.hkv, x.d), x.rand(x.slots, 4, x.hkv, x.d)
    parent, out = x.ints([[-1, 0, 1, 2]] * x.slots), x.rand(x.slots, 4, x.hq, x.d)
    want = [trees.attention(layer, q, k, v, parent, x.scale) for layer in (0, 1)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
            trees.attention(1, q, k, v, parent, x.scale, out)
        trees.attention(0, q, k, v, parent, x.scale, out)
        trees.attention(1, q, k, v, parent, x.scale, out)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        trees.attention(1, q, k, v, parent, x.scale, out)
    graph.replay()
    assert torch.equal(out, want[1])
    assert torch.equal(trees.attention(0, q, k, v, parent, x.scale), want[0])
    assert x.pool.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_pool(cuda, dtype):
    """1024 slots of 64 drafted tokens, tables of millions of tokens: sizes at which sums of the plan's costs are kept in range,
    lists are not staged and trees do not fit in shared memory."""
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, hq=8, hkv=1, page=16, slots=1024, beams=1000, prompt=30, room=70000, pages=16000, seed=7)
    trees = DraftTrees(x.pool, 64)
    x.append(5)
    x.fork([s if s % 7 else s + 3 for s in range(994)] + list(range(994, 1000)) + [1 + 7 * (s % 5) for s in range(24)])
    x.append(3)
    rnd = x.attention(trees, 64)
    x.accept(trees, rnd, x.pick(rnd))
    assert x.pool.status() == 0
    x.same_pages()


def test_streams(cuda):
    """New results belong to the stream of the call; a raw stream needs them given."""
    import torch
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", seed=4)
    trees = DraftTrees(x.pool, 4)
    q, k, v = x.rand(x.slots, 4, x.hq, x.d), x.rand(x.slots, 4, x.hkv, x.d), x.rand(1, x.slots, 4, x.hkv, x.d)
    parent, acc = x.ints([[-1, 0, 1, 2]] * x.slots), x.ints([2] * x.slots)
    want = trees.attention(0, q, k, v[0], parent, x.scale)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [trees.attention(0, q, k, v[0], parent, x.scale, stream=side) for _ in range(5)]
    n, path = trees.accept(v, v, parent, acc, stream=side)
    side.synchronize()
    assert all(torch.equal(y, want) for y in got)
    assert n.tolist() == [3] * 4 + [0] * 2 and path.tolist() == [[0, 1, 2, -1]] * 4 + [[-1] * 4] * 2
    for call in (lambda s: trees.attention(0, q, k, v[0], parent, x.scale, stream=s), lambda s: trees.accept(v, v, parent, acc, stream=s)):
        with pytest.raises(ValueError):
            call(side.cuda_stream)
    assert x.pool.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(cuda, dtype):
    """A pool whose last layer begins behind 2^31 elements."""
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, layers=3, hq=16, hkv=8, slots=3, beams=2, prompt=200, room=40, pages=70000, seed=12)
    trees = DraftTrees(x.pool, 7)
    x.append(30)
    x.fork([0, 1, 1])
    rnd = x.attention(trees, 7)
    x.accept(trees, rnd, [6 if c == 7 else c - 1 for c in rnd[1]])
    x.truncate([225, -1, 210])
    x.attention(trees, 7)
    x.decode()
    assert x.pool.status() == 0
    x.same_pages()


def test_fork_refusals(cuda):
    x = Trees("bf16", seed=4)
    good = x.ints([0, 1, 2, 3, 0, 1])
    for bad in (good.long(), good[:5], good.cpu(), good.repeat(2)[::2]):
        with pytest.raises(ValueError):
            x.pool.fork_slots(bad)
    x.fork([0, 1, 2, 3, 0, 1])
    assert x.pool.status() == 0
    x.same_pages()
