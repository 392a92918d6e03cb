"""Sampled tokens against the definition in 64 bits."""
import itertools
import math

import numpy as np
import pytest
import torch

from tests.sampling_reference import kept_mass, pick

pytestmark = pytest.mark.gpu


def _sampler(rows, vocab):
    from paper_2608_08020_gb300.sampling import TokenSampler
    return TokenSampler(rows, vocab)


def check(logits, u, **kw):
    """One call on every row against the definition; kw: numbers, or a list for every row."""
    rows, vocab = logits.shape
    types = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}
    given = {n: torch.tensor(x, dtype=types[n], device="cuda") if isinstance(x, list) else x for n, x in kw.items()}
    token, logprob = _sampler(rows, vocab)(logits, u, **given)
    token, logprob = token.cpu().numpy(), logprob.cpu().double().numpy()
    x, uu = logits.float().cpu().double().numpy(), u.cpu().double().numpy()
    f32 = {n: [float(np.float32(y)) for y in (x_ if isinstance(x_, list) else [x_] * rows)] if n != "top_k"
           else (x_ if isinstance(x_, list) else [x_] * rows) for n, x_ in kw.items()}
    for r in range(rows):
        want, lp = pick(x[r], uu[r], **{n: v[r] for n, v in f32.items()})
        assert token[r] == want, f"row {r}: token {token[r]}, not {want}"
        # A rounding to fp32, and a total of weights of 2^-33 each.
        assert logprob[r] == lp or abs(logprob[r] - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -32, f"row {r}"
    return token


def _logits(g, rows, vocab, dtype, sharp=2.0, banned=0.0, pad=0, off=0):
    x = torch.randn(rows, vocab + pad + off, generator=g) * sharp
    if banned:
        x[torch.rand(x.shape, generator=g) < banned] = -math.inf
    return x.to(dtype).cuda()[:, off:off + vocab]


FILTERS = [{}, {"top_k": 5}, {"top_k": 50, "top_p": 0.9}, {"top_p": 0.95}, {"top_p": 0.3, "temperature": 0.2}, {"min_p": 0.05},
           {"min_p": 0.1, "top_p": 0.8, "temperature": 1.7}, {"top_k": 300, "min_p": 0.001, "top_p": 0.99}, {"temperature": 0.0}, {"top_k": 1},
           {"top_k": 2000, "top_p": 0.999}]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 32, 100, 257, 1000, 4097, 32000])
@pytest.mark.parametrize("kw", FILTERS)
def test_tokens(cuda, dtype, vocab, kw):
    g = torch.Generator().manual_seed(vocab)
    rows = 5 if vocab > 4000 else 13
    for pad, off, banned in ((0, 0, 0.0), (1, 3, 0.3)):
        check(_logits(g, rows, vocab, dtype, banned=banned, pad=pad, off=off), torch.rand(rows, generator=g).cuda(), **kw)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 151000, torch.float32), (3, 200003, torch.bfloat16), (40, 128000, torch.bfloat16),
                                              (300, 20000, torch.bfloat16), (2, 524288, torch.bfloat16), (2, 524288, torch.float32)])
@pytest.mark.parametrize("sharp", [0.0, 0.3, 3.0, 30.0])
def test_long_rows(cuda, rows, vocab, dtype, sharp):
    """Flat rows, where thousands of tokens are kept and tie, and sharp ones; every row with parameters of its own."""
    g = torch.Generator().manual_seed(rows)
    x, u = _logits(g, rows, vocab, dtype, sharp=sharp), torch.rand(rows, generator=g).cuda()
    combos = itertools.cycle(itertools.product((0.7, 1.0), (0, 40, 5000), (0.9, 1.0, 0.5), (0.0, 0.02)))
    picked = list(itertools.islice(combos, 7, 7 + rows))
    check(x, u, temperature=[c[0] for c in picked], top_k=[c[1] for c in picked], top_p=[c[2] for c in picked], min_p=[c[3] for c in picked])


@pytest.mark.parametrize("vocab", [64, 999, 30000])
def test_ties(cuda, vocab):
    """Logits of a few values: most borders fall inside a run of equal ones, which goes to the lowest indexes."""
    g = torch.Generator().manual_seed(vocab)
    x = torch.randint(-3, 4, (24, vocab), generator=g).to(torch.bfloat16).cuda()
    x[:, ::7] = -0.0
    u = torch.rand(24, generator=g).cuda()
    for kw in ({"top_k": 9}, {"top_k": vocab // 3}, {"top_p": 0.5}, {"top_p": 0.97}, {"min_p": math.exp(-2.0)}, {"top_k": vocab // 2, "top_p": 0.7},
               {"temperature": 0.0}):
        check(x, u, **kw)
    flat = torch.full((8, vocab), 3.5, device="cuda")
    u = torch.arange(8, device="cuda") / 8
    assert check(flat, u).tolist() == [i * vocab // 8 if i * vocab % 8 == 0 else -(-i * vocab // 8) - 1 for i in range(8)]
    check(flat, u, top_p=0.5)
    check(flat, u, top_k=17)


def test_rows_that_are_not_finite(cuda):
    inf, nan = math.inf, math.nan
    x = torch.zeros(8, 40, device="cuda")
    x[0] = -inf
    x[1] = nan
    x[2, ::2] = nan
    x[3, 5] = x[3, 30] = inf
    x[4] = -inf
    x[4, 39] = -3e38
    x[5, 1:] = -3e38
    x[5, 0] = 3e38
    x[6, 3:] = -inf
    x[7, 7] = inf
    u = torch.full((8,), 0.7, device="cuda")
    for kw in ({}, {"top_k": 3}, {"top_p": 0.6}, {"min_p": 0.5}, {"temperature": 0.0}, {"temperature": 1e-6}, {"temperature": 1e6, "top_p": 0.9}):
        for t in (x, x.to(torch.bfloat16)):
            check(t, u, **kw)


def test_random_numbers_at_the_ends(cuda):
    g = torch.Generator().manual_seed(0)
    x = _logits(g, 8, 500, torch.float32, banned=0.2)
    x[:, 0] = x[:, -1] = -math.inf
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, 1e-30, math.inf], device="cuda")
    check(x, u)
    check(x, u, top_p=0.9)


@pytest.mark.parametrize("name,values", [("temperature", [0.0, -1.0, math.nan, math.inf, 1e-30, 1e-40]), ("top_k", [-5, 0, 500, 499, 1 << 30, 2]),
                                         ("top_p", [0.0, -1.0, 1.0, 2.0, math.nan, 1e-9]), ("min_p", [0.0, -1.0, 1.0, 2.0, math.nan, 1e-30])])
def test_parameters_at_the_ends(cuda, name, values):
    g = torch.Generator().manual_seed(1)
    x, u = _logits(g, 6, 500, torch.float32), torch.rand(6, generator=g).cuda()
    if name == "temperature":   # an endless one makes the row flat
        token = check(x, u, temperature=[v if v != math.inf else 1e38 for v in values])
        given = torch.tensor(values, device="cuda")
        assert _sampler(6, 500)(x, u, temperature=given)[0].tolist() == token.tolist()
    else:
        check(x, u, **{name: values})


def test_shares(cuda):
    """Over an even grid of random numbers every token comes up as often as its share says, within one."""
    g = torch.Generator().manual_seed(3)
    n = 4000
    row = _logits(g, 1, 300, torch.float32, sharp=1.5)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    kw = {"temperature": 0.8, "top_p": 0.9, "min_p": 0.01}
    token, _ = _sampler(n, 300)(row.expand(n, -1).contiguous(), u, **kw)
    w = kept_mass(row[0].cpu().double().numpy(), **{k: float(np.float32(v)) for k, v in kw.items()})
    count = np.bincount(token.cpu().numpy(), minlength=300)
    assert (np.abs(count - n * w / w.sum()) <= 1 + 1e-6).all()


def test_numbers_and_tensors_say_the_same(cuda):
    g = torch.Generator().manual_seed(4)
    x, u = _logits(g, 9, 5000, torch.bfloat16), torch.rand(9, generator=g).cuda()
    s = _sampler(20, 5000)
    full = lambda v, t: torch.full((9,), v, dtype=t, device="cuda")  # noqa: E731
    a = s(x, u, temperature=0.7, top_k=30, top_p=0.9, min_p=0.01)
    out = full(-7, torch.int32), full(7.0, torch.float32)
    b = s(x, u, temperature=full(0.7, torch.float32), top_k=full(30, torch.int32), top_p=full(0.9, torch.float32),
          min_p=full(0.01, torch.float32), token=out[0], logprob=out[1])
    assert b[0] is out[0] and b[1] is out[1]
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = s(x[4:5], u[4:5], temperature=0.7, top_k=30, top_p=0.9, min_p=0.01)     # a row alone draws what it draws among others
    assert one[0].item() == a[0][4].item() and one[1].item() == a[1][4].item()
    assert s(x[:0], u[:0])[0].shape == (0,)


def test_streams_and_graphs(cuda):
    g = torch.Generator().manual_seed(5)
    x, u = _logits(g, 16, 30000, torch.bfloat16), torch.rand(16, generator=g).cuda()
    s = _sampler(16, 30000)
    ref = s(x, u, top_p=0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = s(x, u, top_p=0.9, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(ref[0], out[0]) and torch.equal(ref[1], out[1])
    with pytest.raises(ValueError):
        s(x, u, stream=side.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s(x, u, top_p=0.9)
    for i in range(3):
        u.copy_(torch.rand(16, generator=g))
        x.mul_(0.9)
        graph.replay()
        ref = s(x, u, top_p=0.9)
        assert torch.equal(ref[0], out[0]) and torch.equal(ref[1], out[1])


def test_refusals(cuda):
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.sampling import TokenSampler
    x, u = torch.zeros(4, 100, device="cuda"), torch.zeros(4, device="cuda")
    s = _sampler(4, 100)
    for bad in (x[:, :99], x.half(), x.cpu(), x.t(), torch.zeros(5, 100, device="cuda"), x[0], torch.zeros(1, 100, device="cuda").expand(4, -1)):
        with pytest.raises(ValueError):
            s(bad, u)
    for kw in ({"temperature": u[:3]}, {"top_k": u}, {"top_p": u.double()}, {"min_p": u.cpu()}, {"token": u}, {"logprob": u[::2]}):
        with pytest.raises(ValueError):
            s(x, u, **kw)
    with pytest.raises(ValueError):
        s(x, u[:3])
    for n in ((0, 5), (5, 0)):
        with pytest.raises(ValueError):
            TokenSampler(*n)
    with pytest.raises(B.GambitError, match="GB_ERR_UNSUPPORTED"):
        _sampler(1, 524289)(torch.zeros(1, 524289, device="cuda"), u[:1])
