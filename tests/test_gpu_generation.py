"""Steps of a search as a user runs them: sampled tokens become rotated rows of an 8-bit pool, their attention the next logits;
thoughts appended whole, forks and cuts in between.  Each step against the definitions in 64 bits, and as a replayed graph."""
import pytest
import torch

from tests.cache8 import rotated
from tests.sampling_reference import pick
from tests.test_gpu_pool8 import Both

pytestmark = pytest.mark.gpu
BASE, D, VOCAB = 1e4, 128, 3001


class Search:
    """A pool of 8 bits with its model, a table of rows for each token, and a last product."""

    def __init__(self, seed, hq, hkv, slots=5, layers=2):
        from paper_2608_08020_gb300.rotation import Rotation
        from paper_2608_08020_gb300.sampling import TokenSampler
        self.both = Both(layers=layers, hq=hq, hkv=hkv, slots=slots, pages=128, width=16, seed=seed)
        self.pool, self.layers, self.hq, self.hkv, self.slots = self.both.pool, layers, hq, hkv, slots
        g = torch.Generator().manual_seed(seed)
        self.rows = (torch.randn(VOCAB, layers, hq + 2 * hkv, D, generator=g)).to(torch.bfloat16).cuda()
        self.last = (torch.randn(hq * D, VOCAB, generator=g) / 8).cuda()
        self.rotation = Rotation(D, max_positions=256, base=BASE)
        self.sampler = TokenSampler(slots, VOCAB)
        self.out = torch.zeros(layers, slots, hq, D, device="cuda")
        self.g = g

    def split(self, token, layer):
        x = self.rows[token.clamp(min=0).long(), layer]
        return (y.contiguous() for y in x.split([self.hq, self.hkv, self.hkv], 1))

    def step(self, token, u, temperature):
        for i in range(self.layers):
            q, k, v = self.split(token, i)
            self.pool.decode_attention(i, q, k, v, D ** -0.5, self.out[i], rotation=self.rotation)
        logits = self.out[-1].reshape(self.slots, -1) @ self.last
        return logits, *self.sampler(logits, u, temperature=temperature, top_k=40, top_p=0.9, min_p=0.01)

    def thought(self, tokens):
        """tokens [n][slots]: a thought made elsewhere."""
        for i in range(self.layers):
            x = self.rows[tokens.long(), i]
            k, v = (y.contiguous() for y in x[:, :, self.hq:].split(self.hkv, 2))
            self.pool.append_kv(i, len(tokens), k, v, rotation=self.rotation)


def _turned(x, at):
    return rotated(x.double(), at, D, BASE)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (8, 8), (8, 1)])
def test_a_search(cuda, hq, hkv):
    s = Search(hq * 10 + hkv, hq, hkv)
    model, both = s.both.model, s.both
    both.seed(4, 30, wide=False)
    temperature = torch.tensor([0.7, 1.0, 0.0, 1.3, 1.0]).cuda()
    token = torch.randint(0, VOCAB, (s.slots,), generator=s.g).int().cuda()
    for n in range(12):
        u = torch.rand(s.slots, generator=s.g)
        logits, new, logprob = s.step(token, u.cuda(), temperature)
        for i in range(s.layers):
            q, k, v = (x.cpu() for x in s.split(token, i))
            for b in both.live:
                # K goes in as the cache's 8 bits of the turned row (rounded to fp32 first, as the library turns it); q to bf16.
                at = model.length(b) if i == 0 else model.kv[b][i][0].shape[1]
                model.append(b, i, _turned(k[b:b + 1], at).float().double(), v[b:b + 1].double())
                q[b] = _turned(q[b], at).float().to(torch.bfloat16)
            both.check_out(s.out[i].cpu(), q, i, D ** -0.5)
        for b in range(s.slots):
            t, p = pick(logits[b].cpu().numpy(), float(u[b]), temperature=float(temperature[b]), top_k=40, top_p=float(torch.tensor(0.9)),
                        min_p=float(torch.tensor(0.01)))
            assert int(new[b]) == t and abs(float(logprob[b]) - p) <= 1e-6 + 2.0 ** -23 * abs(p)
        token = new
        if n == 4:
            both.fork([0, 0, 2, 2, -1])
            token = token[torch.tensor([0, 0, 2, 2, 4]).cuda()]
        if n == 7:
            tokens = torch.randint(0, VOCAB, (19, s.slots), generator=s.g)
            s.thought(tokens.cuda())
            for i in range(s.layers):
                for b in both.live:
                    x = s.rows[tokens[:, b].long().cuda(), i].cpu()
                    at = model.kv[b][i][0].shape[1]
                    k = torch.stack([_turned(x[j, hq:hq + hkv], at + j) for j in range(len(tokens))])
                    model.append(b, i, k.float().double(), x[:, hq + hkv:].double())
        if n == 9:
            both.truncate([35, -1, 47, 40, -1])
    both.check_cache()


def test_a_replayed_step(cuda):
    """One captured step of attention and draw, replayed over a growing cache, against eager calls of a twin."""
    a, b = (Search(7, 8, 2) for _ in range(2))
    for s in (a, b):
        s.both.seed(4, 30, wide=False)
    token, u = torch.arange(5, dtype=torch.int32).cuda(), torch.zeros(5).cuda()
    temperature = torch.full((5,), 1.1).cuda()
    logprob = torch.zeros(5).cuda()

    def step():
        _, t, p = a.step(token, u, temperature)
        token.copy_(t.clamp(min=0))
        logprob.copy_(p)

    expected = torch.arange(5, dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(1)
    graph = None
    for n in range(40):
        u.copy_(torch.rand(5, generator=g))
        if n == 2:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        _, t, p = b.step(expected, u, temperature)
        expected = t.clamp(min=0)
        assert torch.equal(token, expected) and torch.equal(logprob, p) and torch.equal(a.out, b.out)
    for i in range(2):
        first = torch.zeros(5, dtype=torch.int32).cuda()
        for x, y in zip(a.pool.read_kv(i, first, 70), b.pool.read_kv(i, first, 70)):
            assert torch.equal(x, y)
    assert a.pool.status() == 0 and b.pool.status() == 0
