"""Sampled tokens where top-k's border, min-p's and the largest temperatures meet."""
import itertools
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_sampling import _logits, _sampler, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [3000, 60001])
@pytest.mark.parametrize("c", [1, 4])
def test_top_k_ends_in_a_run_just_below_min_p(cuda, dtype, vocab, c):
    """Whole logits: fp32(exp(-c)) lies above exp(-c), so the tokens c below the largest are out, and the cut by count ends among them."""
    p = float(np.float32(math.exp(-c)))
    assert math.log(p) > -c
    g = torch.Generator().manual_seed(vocab + c)
    x = torch.randint(-9, 4 - c, (6, vocab), generator=g).float()
    x[:, 7::vocab // 600] = 3.0 - c                       # more than 600 one step below the border
    for r in range(6):
        x[r, torch.randperm(vocab, generator=g)[:5 + 20 * r]] = 3.0
    x, u = x.to(dtype).cuda(), torch.rand(6, generator=g).cuda()
    for k in (513, 600, 5 + 20 * 3 + 513):
        for q in (1.0, 0.6):
            token = check(x, u, top_k=k, min_p=p, top_p=q)
            assert (x.float().cpu().gather(1, torch.as_tensor(token).long()[:, None]) == 3.0).all() or c > 1
    check(x, torch.full((6,), 1 - 2.0 ** -24, device="cuda"), top_k=700, min_p=p)


@pytest.mark.parametrize("vocab", [5, 500, 40000])
@pytest.mark.parametrize("min_p", [0.0, 1e-30, 0.5, 1.0, 2.0, math.inf])
def test_endless_temperatures(cuda, vocab, min_p):
    """They make a row flat: every token stays, and comes up as often as the others.  (The largest finite one says the same.)"""
    g = torch.Generator().manual_seed(vocab)
    x, u = _logits(g, 7, vocab, torch.float32, banned=0.2), torch.rand(7, generator=g).cuda()
    x[:, 0] = 1.0
    s = _sampler(7, vocab)
    inf = torch.full((7,), math.inf, device="cuda")
    for kw in ({}, {"top_k": 3}, {"top_k": 600}, {"top_p": 0.7}, {"top_k": 4, "top_p": 0.5}):
        token, logprob = s(x, u, temperature=inf, min_p=min_p, **kw)
        kept = (x > -math.inf).sum(1)
        if kw.get("top_k", vocab) < vocab:
            kept = kept.clamp(max=kw["top_k"])
        if "top_p" in kw:
            kept = torch.ceil(kept.double() * float(np.float32(kw["top_p"])) - 1e-9).long()
        assert (token >= 0).all() and (x.gather(1, token.long()[:, None]) > -math.inf).all()
        assert ((logprob.double() + kept.double().log()).abs() <= 2.0 ** -24 * kept.double().log() + 2.0 ** -30).all()


def test_parameters_at_the_ends_together(cuda):
    """Every pairing of extremes, a row each."""
    temps = [1e-40, 1e-30, 1e-6, 0.5, 1.0, 1e6, 1e30, 3e38]
    ps = [0.0, 1e-9, 0.5, 1 - 2.0 ** -24, 1.0]
    mins = [0.0, 1e-40, 1e-30, 1e-3, 1 - 2.0 ** -24, 1.0, 3.0]
    combos = list(itertools.product(temps, ps, mins))
    g = torch.Generator().manual_seed(11)
    for vocab, k in ((300, 0), (300, 7), (9000, 0), (9000, 100), (9000, 2000)):
        x = torch.randint(-40, 40, (len(combos), vocab), generator=g).float() / 4
        x[:, 3] = 11.0                                    # one likeliest token: no draw by a share of a tie
        check(x.cuda(), torch.rand(len(combos), generator=g).cuda(), temperature=[c[0] for c in combos], top_p=[c[1] for c in combos],
              min_p=[c[2] for c in combos], top_k=k)


@pytest.mark.parametrize("top_k", [1 << 31, (1 << 32) + 1, 1 << 40, -(1 << 31) - 1, -(1 << 32) + 2, 0, -3, 500, 501])
def test_numbers_that_keep_every_token(cuda, top_k):
    g = torch.Generator().manual_seed(5)
    x, u = _logits(g, 6, 500, torch.float32), torch.rand(6, generator=g).cuda()
    a, b = _sampler(6, 500)(x, u, top_k=top_k), _sampler(6, 500)(x, u)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
