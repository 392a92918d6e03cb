"""Which plan a layer above 0 of a draft round runs with: never one that a graph's replay has overtaken."""
import pytest

from tests.test_gpu_draft import Trees

pytestmark = pytest.mark.gpu


def rounds(x, t, seed=0):
    """Inputs of a round of one layer's shape, and a parent array per kind of tree."""
    q, k, v = x.rand(x.slots, t, x.hq, x.d), x.rand(x.slots, t, x.hkv, x.d), x.rand(x.slots, t, x.hkv, x.d)
    return q, k, v, x.ints([[i - 1 for i in range(t)]] * x.slots), x.ints([[-1] * t] * x.slots)


def captured(call):
    import torch
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = call()
    torch.cuda.synchronize()
    return graph, kept


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("change", ["accept", "truncate", "append", "fork", "release", "prune"])
def test_a_replay_that_changes_the_pool(cuda, dtype, change):
    """Layer 0, a replay that changes the contexts, layer 1: the plan is of contexts that are no more."""
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, layers=2, slots=6, beams=4, prompt=40, seed=21)
    t = 4
    trees = DraftTrees(x.pool, t)
    q, k, v, chain, _ = rounds(x, t)
    kk, vv = x.rand(2, x.slots, t, x.hkv, x.d), x.rand(2, x.slots, t, x.hkv, x.d)
    new = x.rand(2, 1, x.slots, x.hkv, x.d)
    out = torch.full_like(q, 7.0)
    calls = dict(accept=(lambda a: trees.accept(kk, vv, chain, a), x.ints([3, 2, 1, 0, 0, 0])),
                 truncate=(x.pool.truncate, x.ints([30, 35, 40, 17, 0, 0])),
                 append=(lambda a: [x.pool.append_kv(layer, 1, new[layer], new[layer]) for layer in (0, 1)], None),
                 fork=(x.pool.fork_slots, x.ints([0, 1, 2, 3, 0, 1])),
                 release=(x.pool.release, x.ints([2])),
                 prune=(lambda a: x.pool.prune_branch(K=2, fanout=2, parent_out=a), x.ints([0] * x.slots)))
    call, arg = calls[change]
    graph, _ = captured(lambda: call(arg))
    trees.attention(0, q, k, v, chain, x.scale)
    trees.attention(1, q, k, v, chain, x.scale)
    assert x.pool.status() == B.GB_OK
    trees.attention(0, q, k, v, chain, x.scale)
    graph.replay()
    trees.attention(1, q, k, v, chain, x.scale, out)
    assert x.pool.status() == B.GB_ERR_STATE
    assert bool((out == 7).all())
    x.pool.clear_status()
    want = trees.attention(0, q, k, v, chain, x.scale)               # a round of the contexts as they are
    got = trees.attention(1, q, k, v, chain, x.scale)
    assert x.pool.status() == B.GB_OK and not torch.equal(got, want)  # (the layers differ)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_replay_that_plans_in_the_same_workspace(cuda, dtype):
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees(dtype, layers=2, slots=5, beams=4, prompt=50, seed=22)
    t = 5
    trees, other = DraftTrees(x.pool, t), DraftTrees(x.pool, t)
    q, k, v, chain, flat = rounds(x, t)
    out = torch.full_like(q, 7.0)
    graph, kept = captured(lambda: [trees.attention(layer, q, k, v, flat, x.scale) for layer in (0, 1)])
    beside, _ = captured(lambda: [other.attention(layer, q, k, v, flat, x.scale) for layer in (0, 1)])
    trees.attention(0, q, k, v, chain, x.scale)
    want = trees.attention(1, q, k, v, chain, x.scale)
    trees.attention(0, q, k, v, chain, x.scale)
    beside.replay()                                                  # another workspace: the plan stands
    assert torch.equal(trees.attention(1, q, k, v, chain, x.scale), want)
    assert x.pool.status() == B.GB_OK
    graph.replay()                                                   # trees without edges, in this one
    trees.attention(1, q, k, v, chain, x.scale, out)
    assert x.pool.status() == B.GB_ERR_STATE and bool((out == 7).all())
    x.pool.clear_status()
    for _ in range(2):                                               # the graph's own layers have their plan each time
        x.append(1)
        graph.replay()
        assert x.pool.status() == B.GB_OK
        assert torch.equal(kept[0], trees.attention(0, q, k, v, flat, x.scale))
        assert torch.equal(kept[1], trees.attention(1, q, k, v, flat, x.scale))


def test_an_object_at_the_address_of_one_before(cuda):
    """A new object has no plan, whatever the object whose memory it got had planned and wherever that memory has been."""
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=2, seed=23)
    q, k, v, chain, _ = rounds(x, 4)
    trees = DraftTrees(x.pool, 4)
    trees.attention(0, q, k, v, chain, x.scale)
    at = trees.workspace.data_ptr()
    del trees
    trees = DraftTrees(x.pool, 4)
    assert trees.workspace.data_ptr() == at
    launches = B.gb_pool_launch_count(x.pool.handle)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        trees.attention(1, q, k, v, chain, x.scale)
    assert B.gb_pool_launch_count(x.pool.handle) == launches and x.pool.status() == B.GB_OK
    trees.attention(0, q, k, v, chain, x.scale)
    trees.attention(1, q, k, v, chain, x.scale)
    assert x.pool.status() == B.GB_OK


def test_rounds_side_by_side(cuda):
    """Rounds in workspaces of their own, their layers by turns, one of them of shorter trees."""
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    x = Trees("bf16", layers=3, seed=24)
    a, b = DraftTrees(x.pool, 4), DraftTrees(x.pool, 3)
    qa, ka, va, chain, flat = rounds(x, 4)
    qb, kb, vb, short, _ = rounds(x, 3)
    want_a = [a.attention(layer, qa, ka, va, flat, x.scale) for layer in range(3)]
    want_b = [b.attention(layer, qb, kb, vb, short, x.scale) for layer in range(3)]
    got_a, got_b = [a.attention(0, qa, ka, va, flat, x.scale)], [b.attention(0, qb, kb, vb, short, x.scale)]
    for layer in (1, 2):
        got_a.append(a.attention(layer, qa, ka, va, flat, x.scale))
        got_b.append(b.attention(layer, qb, kb, vb, short, x.scale))
    assert all(torch.equal(g, w) for g, w in zip(got_a + got_b, want_a + want_b))
    many = [DraftTrees(x.pool, 4) for _ in range(17)]
    for m in many:
        m.attention(0, qa, ka, va, chain, x.scale)
    for m in many[1:]:
        m.attention(1, qa, ka, va, chain, x.scale)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        many[0].attention(1, qa, ka, va, chain, x.scale)
    assert x.pool.status() == B.GB_OK
    x.append(1)
    for m in (a, b, many[5]):
        q, k, v = (qb, kb, vb) if m is b else (qa, ka, va)
        with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
            m.attention(1, q, k, v, short if m is b else chain, x.scale)
    a.attention(0, qa, ka, va, chain, x.scale)
    a.attention(1, qa, ka, va, chain, x.scale)
    assert x.pool.status() == B.GB_OK


def test_workspaces_that_overlap(cuda):
    """A plan whose memory another one's shares gives way to it."""
    import torch
    from paper_2608_08020_gb300 import binding as B
    x = Trees("bf16", layers=2, seed=25)
    q, k, v, chain, _ = rounds(x, 4)
    n = B.gb_draft_workspace_bytes(x.pool.handle, 4)
    memory, out = torch.empty(n + 256, dtype=torch.uint8, device="cuda"), torch.empty_like(q)

    def attention(layer, at):
        d = B.GbDraft(parent_dev=chain.data_ptr(), workspace_dev=memory.data_ptr() + at, workspace_bytes=n, n_draft=4)
        B.gb_draft_attention(x.pool.handle, layer, d, q, k, v, x.scale, out)

    attention(0, 0)
    attention(0, 256)
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        attention(1, 0)
    attention(1, 256)
    assert x.pool.status() == B.GB_OK
