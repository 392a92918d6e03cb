"""Pools of 8 bits: what the cache holds, bit by bit, through every call that moves rows, and the attention over it,
against the definition in 64 bits (tests/cache8.py)."""
import pytest
import torch

from tests.cache8 import Cache8, attention

pytestmark = pytest.mark.gpu


def _rand(g, *shape, wide=True):
    """bf16 rows whose size differs from token to token by powers of ten where `wide`."""
    x = torch.randn(shape, generator=g)
    if wide:
        x = x * 10 ** torch.empty(shape[:-1]).uniform_(-3, 3, generator=g)[..., None]
    return x.to(torch.bfloat16)


class Both:
    """A pool and its model, moved together."""

    def __init__(self, *, layers=1, hq=8, hkv=2, page=16, slots=4, pages=64, width=12, seed=0, garbage=True):
        from paper_2608_08020_gb300.pool import BeamPool
        self.pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, page_size=page, kv_dtype="fp8",
                             num_pages=pages, max_beams=slots, max_pages_per_beam=width)
        if garbage:   # NaN codes and scales of 2^-1: nothing of a page that was not written may be used
            self.pool.kv.fill_(0xFF)
        self.model = Cache8(layers, slots, hkv, 128)
        self.layers, self.hq, self.hkv, self.slots = layers, hq, hkv, slots
        self.g = torch.Generator().manual_seed(seed)
        self.live = []

    def seed(self, n, length, wide=True):
        k, v = (_rand(self.g, self.layers, length, self.hkv, 128, wide=wide) for _ in range(2))
        self.pool.seed(n, length, k.cuda(), v.cuda())
        self.live = list(range(n))
        for b in range(n):
            for i in range(self.layers):
                self.model.append(b, i, k[i].double(), v[i].double())

    def append(self, n, k=None, v=None, wide=True):
        for i in range(self.layers):
            kk, vv = (x if x is not None else _rand(self.g, n, self.slots, self.hkv, 128, wide=wide) for x in (k, v))
            self.pool.append_kv(i, n, kk.cuda(), vv.cuda())
            for b in self.live:
                self.model.append(b, i, kk[:, b].double(), vv[:, b].double())

    def truncate(self, lengths):
        self.pool.truncate(torch.tensor(lengths, dtype=torch.int32).cuda())
        for b in self.live:
            if lengths[b] >= 0:
                self.model.truncate(b, lengths[b])

    def fork(self, parent_of):
        self.pool.fork_slots(torch.tensor(parent_of, dtype=torch.int32).cuda())
        self.model.fork(parent_of)
        self.live = [b for b in range(self.slots) if b in self.live or parent_of[b] >= 0]

    def release(self, b):
        self.pool.release(torch.tensor([b], dtype=torch.int32).cuda())
        self.model.release(b)
        self.live.remove(b)

    def decode(self, wide=False, flags=0, scale=128 ** -0.5, size=1.0):
        """One step of every layer; compares its attention with the definition."""
        for i in range(self.layers):
            q = (_rand(self.g, self.slots, self.hq, 128, wide=False).float() * size).to(torch.bfloat16)
            k, v = (_rand(self.g, self.slots, self.hkv, 128, wide=wide) for _ in range(2))
            out = torch.full((self.slots, self.hq, 128), float("nan"), device="cuda")
            self.pool.decode_attention(i, q.cuda(), k.cuda(), v.cuda(), scale, out, flags)
            for b in self.live:
                self.model.append(b, i, k[b:b + 1].double(), v[b:b + 1].double())
            self.check_out(out.cpu(), q, i, scale)
        assert self.pool.status() == 0

    def check_out(self, out, q, layer, scale):
        for b in range(self.slots):
            if b not in self.live:
                assert (out[b] == 0).all(), f"slot {b}"
                continue
            held = self.model.kv[b][layer]
            ref, a, dot, top = attention(q[b].double(), held, scale)
            # A score is a sum of 128 products in fp32: off by at most 128 x 2^-24 of their sizes' sum (products of an fp16 and
            # a code are exact), and each weight by as much, twice (softmax over them); its exponential, its two fp16 terms and
            # the fp32 sums over the tokens and records by 2^-18 together.
            # A weight times its block's 2^e is held to 2^-31 of the largest such (the second term's last place, a subnormal's,
            # against a maximum that gets 2^7), and multiplies codes of up to 448: together at most that for every token.
            tol = a * (2 * dot[:, None] * 2.0 ** -17 + 2.0 ** -18) + held[0].shape[1] * 448 * 2.0 ** -31 * top[:, None]
            err = (out[b].double() - ref).abs()
            assert (err <= tol).all(), f"layer {layer} slot {b}: {(err / tol).max():.2f} of the bound"

    def check_cache(self):
        for i in range(self.layers):
            most = max(self.model.length(b) for b in range(self.slots))
            k, v = self.pool.read_kv(i, torch.full((self.slots,), -1, dtype=torch.int32).cuda(), most + 3)
            got = torch.stack([k, v]).cpu().double()
            ref = self.model.read(i, [-1] * self.slots, most + 3)
            assert torch.equal(got.isnan(), ref.isnan())
            bad = (got != ref) & ~ref.isnan()
            assert not bad.any(), f"layer {i}: {int(bad.sum())} values, first at {bad.nonzero()[0].tolist()}"
        assert self.pool.status() == 0


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("length", [1, 15, 16, 37, 100])
def test_seed(cuda, page, length):
    t = Both(layers=2, page=page, seed=length)
    t.seed(3, length)
    t.check_cache()


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("n", [1, 2, 5, 16, 17, 40])
def test_append(cuda, page, n):
    """Chunks that begin inside a block, end inside it, span blocks and pages; the first one copies the shared tail page."""
    t = Both(layers=2, page=page, seed=n)
    t.seed(4, 21)
    for _ in range(3):
        t.append(n)
        t.check_cache()


@pytest.mark.parametrize("page", [16, 64])
def test_forks_cuts_and_releases(cuda, page):
    t = Both(layers=2, page=page, pages=128, width=16)
    t.seed(4, 30)
    t.append(7)
    t.fork([0, 0, 2, 2])
    t.append(3)
    t.check_cache()
    t.truncate([20, -1, 33, 16])
    t.append(1)
    t.check_cache()
    t.fork([0, 1, 0, 3])
    t.truncate([18, -1, 17, 12])
    t.check_cache()
    t.append(18)
    t.check_cache()
    t.release(1)
    t.append(2)
    t.check_cache()


def test_values_at_the_ends_of_the_range(cuda):
    t = Both(slots=1)
    t.seed(1, 3)
    inf, nan = float("inf"), float("nan")
    rows = torch.zeros(6, 1, 2, 128)
    rows[0, 0, 0, :8] = torch.tensor([inf, -inf, nan, 448.0, -448.0, 449.0, 2.0 ** -9, 2.0 ** -10])
    rows[1, 0, 0, :4] = torch.tensor([3e38, -1e-38, 0.0, -0.0])
    rows[2, 0, 0, :2] = torch.tensor([2.0 ** -60, 2.0 ** -70])
    rows[3, 0, 1] = 1e-30
    rows[4, 0, 1, 0] = nan
    rows[5, 0, 1] = torch.linspace(-500, 500, 128)
    rows = rows.to(torch.bfloat16)
    for i in (5, 4, 3, 2, 0, 1):
        t.append(1, rows[i:i + 1], rows[i:i + 1])
        t.check_cache()
    t.append(6, rows, rows.flip(0))
    t.check_cache()


@pytest.mark.parametrize("hq,hkv,page,layers", [(2, 2, 16, 1), (4, 2, 16, 1), (8, 1, 32, 2), (32, 8, 64, 1), (16, 2, 16, 3)])
@pytest.mark.parametrize("flags", [0, 1, 2])
def test_decode(cuda, hq, hkv, page, layers, flags):
    """Steps over trees: unaligned prompts, shared prefixes, copies on write, a slot without a beam."""
    t = Both(layers=layers, hq=hq, hkv=hkv, page=page, slots=6, pages=400, width=24, seed=hq + page)
    t.seed(5, 85, wide=False)
    for _ in range(3):
        t.decode(flags=flags)
    t.fork([0, 0, 2, 2, 4, -1])
    t.append(50, wide=False)
    for _ in range(18):
        t.decode(flags=flags)
    t.fork([0, 1, 0, 3, 0, -1])
    for _ in range(2):
        t.decode(flags=flags)
    t.check_cache()


@pytest.mark.parametrize("length", [0, 1, 14, 15, 16, 17, 31, 32, 33, 250])
def test_decode_lengths(cuda, length):
    t = Both(slots=3, hq=16, pages=64, width=20, seed=length)
    t.seed(3, max(length, 1), wide=False)
    if length == 0:
        t.truncate([0, 1, 0])
    t.decode()
    t.decode()


def test_decode_over_blocks_of_very_different_sizes(cuda):
    """K and V whose blocks lie a factor of 10^12 apart: each block's weights are taken relative to its own scale."""
    t = Both(slots=2, pages=64, width=20)
    n = 150
    sizes = 10.0 ** torch.empty(2, n, 1, 2, 1).uniform_(-6, 6, generator=t.g)
    sizes[0] = sizes[0].clamp(max=1.0)
    k, v = (torch.randn(2, n, 1, 2, 128, generator=t.g) * sizes).to(torch.bfloat16)
    t.seed(2, 5, wide=False)
    t.append(n, k.expand(-1, 2, -1, -1).contiguous(), v.expand(-1, 2, -1, -1).contiguous())
    for _ in range(3):
        t.decode()
    t.decode(size=0.0)
    t.decode(size=1e-30, scale=1e30)
    t.decode(size=1e20, scale=1e-21)


def test_decode_without_values(cuda):
    t = Both(slots=2)
    t.seed(2, 40, wide=False)
    z = torch.zeros(20, 2, 2, 128, dtype=torch.bfloat16)
    t.append(20, z, z)
    t.decode()
    t.append(20, torch.randn(20, 2, 2, 128, generator=t.g).to(torch.bfloat16), z)
    t.decode()


def test_nan_reaches_those_that_see_it(cuda):
    t = Both(slots=2, width=20)
    t.seed(2, 30, wide=False)
    v = _rand(t.g, 1, 2, 2, 128, wide=False)
    v[0, 0, 1, 5] = float("inf")
    t.append(1, None, v)
    q, k, w = (_rand(t.g, 2, h, 128, wide=False) for h in (8, 2, 2))
    out = torch.zeros(2, 8, 128, device="cuda")
    t.pool.decode_attention(0, q.cuda(), k.cuda(), w.cuda(), 0.1, out)
    seen = torch.zeros(2, 8, 128, dtype=torch.bool)
    seen[0, 4:, 5] = True
    assert torch.equal(out.isnan().cpu(), seen)


def test_out_of_pages_changes_nothing(cuda):
    t = Both(slots=2, pages=4, width=4)
    t.seed(2, 32, wide=False)
    t.decode()
    t.decode()
    t.append(14, wide=False)      # both slots' third pages are full, and no page is left
    q, k = _rand(t.g, 2, 8, 128), _rand(t.g, 2, 2, 128)
    out = torch.ones(2, 8, 128, device="cuda")
    t.pool.decode_attention(0, q.cuda(), k.cuda(), k.cuda(), 0.1, out)
    assert (out == 0).all() and t.pool.status() == 2
    t.pool.clear_status()
    t.check_cache()


def test_captured_steps(cuda):
    """Steps replayed from a graph give what eager steps give, bit by bit."""
    a, b = Both(layers=2, seed=5), Both(layers=2, seed=5)
    for t in (a, b):
        t.seed(4, 40, wide=False)
        t.decode()                # (loads the kernels)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(2, 4, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (8, 2, 2))
    outs = [torch.zeros(2, 4, 8, 128, device="cuda") for _ in range(2)]

    def step(t, out):
        for i in range(2):
            t.pool.decode_attention(i, q[i], k[i], v[i], 0.1, out[i])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, outs[0])
    for _ in range(20):
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        k.mul_(1.1)
        graph.replay()
        step(b, outs[1])
        assert torch.equal(outs[0], outs[1])
    assert a.pool.status() == 0 and b.pool.status() == 0


def test_refusals(cuda):
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.draft import DraftTrees
    t = Both()
    first = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(B.GambitError, match="GB_ERR_STATE"):
        t.pool.read_kv(0, first, 1)
    t.seed(4, 10)
    with pytest.raises(B.GambitError, match="GB_ERR_UNSUPPORTED"):
        DraftTrees(t.pool, 4)
    for layer, n in ((-1, 1), (1, 1), (0, -1)):
        with pytest.raises((B.GambitError, RuntimeError)):
            t.pool.read_kv(layer, first, n)
    with pytest.raises(ValueError):
        t.pool.read_kv(0, first[:3], 1)
    q = torch.zeros(4, 8, 136, dtype=torch.bfloat16, device="cuda").flatten()
    k = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.GambitError, match="GB_ERR_INVALID"):
        t.pool.decode_attention(0, q[1:], k, k, 0.1, torch.zeros(4, 8, 128, device="cuda"))
    t.check_cache()
