"""The page model of accepted paths and cuts, on the CPU: a path accepted by every slot is that many decode steps, a cut
frees what nobody holds, a round of both restores the pool."""
import numpy as np
import pytest

from oracle.pool import PoolOracle


def pool(rng, page, slots=9):
    m = PoolOracle(400, slots, 40, page)
    m.seed(int(rng.integers(1, slots)), int(rng.integers(1, 70)))
    for _ in range(int(rng.integers(0, 50))):
        assert m.begin_step()
    live = np.flatnonzero(m.active)
    m.fork_slots([int(rng.choice(live)) if s not in live and rng.random() < 0.7 else s if s in live else -1 for s in range(slots)])
    return m


def state(m):
    return ([list(t) for t, a in zip(m.tables, m.active) if a], m.refcnt.tolist(), m.seq_len.tolist(), m.gen.tolist(),
            m.free_bits().tolist(), m.num_free())


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("seed", range(6))
def test_a_path_of_all_slots_is_decode_steps(page, seed):
    rng = np.random.default_rng(seed)
    m = pool(rng, page)
    rng = np.random.default_rng(seed)
    n = pool(rng, page)
    k = int(rng.integers(1, 64))
    assert m.accept([k] * 9)
    for _ in range(k):
        assert n.begin_step()
    assert state(m) == state(n)
    m.check_invariants()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("seed", range(8))
def test_paths_and_cuts(page, seed):
    rng = np.random.default_rng(100 + seed)
    m = pool(rng, page)
    for _ in range(12):
        before, lengths = state(m), m.seq_len.copy()
        tables = [list(t) for t in m.tables]
        alone = all(m.refcnt[t[-1]] == 1 for t, a in zip(tables, m.active) if a and t)   # no copies to come
        counts = rng.integers(0, 20, 9)
        assert m.accept(counts)
        m.check_invariants()
        assert m.seq_len.tolist() == [int(n + c) if a else int(n) for n, c, a in zip(lengths, counts, m.active)]
        for s in np.flatnonzero(m.active):           # what was there stays, but for a shared tail page
            full = lengths[s] // page
            assert m.tables[s][:full] == tables[s][:full]
        assert m.truncate([int(n) for n in lengths])
        m.check_invariants()
        assert m.seq_len.tolist() == lengths.tolist()
        if alone:
            assert state(m)[1:] == before[1:]
        cut = [int(rng.integers(0, n + 1)) if a and rng.random() < 0.4 else -1 for n, a in zip(m.seq_len, m.active)]
        m.truncate(cut)
        m.check_invariants()
        assert all(c < 0 or m.seq_len[s] == c for s, c in enumerate(cut))


def test_all_or_nothing():
    m = PoolOracle(6, 4, 8, 16)
    m.seed(4, 32)
    before = state(m)
    assert not m.accept([1, 1, 1, 2 * 16 + 1])       # four free pages, six needed
    assert state(m) == before
    assert m.accept([1, 1, 1, 1]) and m.num_free() == 0
    assert not m.truncate([20, -1, -1, -1])          # inside a page of four holders, none free
    assert m.seq_len.tolist() == [33] * 4
    assert m.truncate([32, -1, -1, -1]) and m.num_free() == 1
    assert m.truncate([20, -1, -1, -1]) and m.num_free() == 0
    m.check_invariants()
