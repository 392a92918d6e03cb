"""Sampled tokens where many tokens stay: nuclei longer than any list, cuts among equal weights, lists of every length, and the same
draw however many rows are in the call."""
import pytest
import torch

from tests.test_gpu_sampling import _logits, _sampler, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows", [(4500, 7), (9000, 5), (60001, 3), (151000, 2)])
@pytest.mark.parametrize("sharp", [0.1, 0.5, 1.5])
def test_flat_rows(cuda, dtype, vocab, rows, sharp):
    g = torch.Generator().manual_seed(vocab + rows)
    x = _logits(g, rows, vocab, dtype, sharp=sharp, banned=0.05, pad=1, off=1)
    for p in (0.0, 0.5, 0.95, 0.9995, 0.99999):
        for kw in ({}, {"min_p": 0.002}, {"temperature": 2.5}):
            check(x, torch.rand(rows, generator=g).cuda(), top_p=p, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [5000, 20001, 140000])
def test_equal_weights(cuda, dtype, vocab):
    """Every logit the same; two levels; steps of a few thousand equal ones."""
    g = torch.Generator().manual_seed(vocab)
    x = torch.zeros(4, vocab)
    x[1, torch.randperm(vocab, generator=g)[:vocab // 2]] = -0.5
    x[2] = torch.randint(0, 12, (vocab,), generator=g) * -0.75
    x[3] = torch.randint(0, 3, (vocab,), generator=g) * -2.0 + 100
    x = x.to(dtype).cuda()
    for p in (0.01, 0.25, 0.5, 0.9, 0.999):
        check(x, torch.rand(4, generator=g).cuda(), top_p=p)
        check(x, torch.tensor([0.0, 0.999999, 0.5, 0.25]).cuda(), top_p=p, min_p=0.3)


@pytest.mark.parametrize("n", [1, 31, 64, 65, 128, 129, 255, 256, 257, 511, 512, 513, 1500, 4095, 4096, 4097, 4500])
@pytest.mark.parametrize("vocab", [5000, 50000])
def test_lists_of_every_length(cuda, n, vocab):
    """n tokens that can be kept, by each of the filters."""
    g = torch.Generator().manual_seed(n)
    x = torch.full((3, vocab), -40.0)
    for r in range(3):
        at = torch.randperm(vocab, generator=g)[:n]
        x[r, at] = torch.rand(n, generator=g) * (0.0 if r == 2 else 3.0)
    x = x.cuda()
    u = torch.rand(3, generator=g).cuda()
    for kw in ({"top_p": 0.9}, {"top_p": 0.99999}, {"min_p": 0.01}, {"min_p": 0.01, "top_p": 0.7}, {"top_k": n}, {"top_k": n, "top_p": 0.6},
               {"top_k": max(1, n // 2), "top_p": 0.9}, {"top_k": n + 1}):
        check(x, u, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [3000, 70001])
def test_a_row_alone_and_among_many(cuda, dtype, vocab):
    g = torch.Generator().manual_seed(5)
    x = torch.cat([_logits(g, 3, vocab, dtype, sharp=s) for s in (0.2, 1.0, 4.0, 20.0)])
    rows, many = len(x), 50
    u = torch.rand(rows, generator=g).cuda()
    for kw in ({"top_p": 0.9}, {"top_p": 0.999, "min_p": 1e-4}, {"top_k": 40, "top_p": 0.9}, {"top_k": 1000}, {}):
        token, logprob = _sampler(rows * many, vocab)(x.repeat(many, 1), u.repeat(many), **kw)
        for r in range(rows):
            t, p = _sampler(1, vocab)(x[r:r + 1], u[r:r + 1], **kw)
            assert (token[r::rows] == t).all() and (logprob[r::rows] == p).all(), f"row {r} {kw}"


def test_rows_past_32_bits(cuda):
    """Rows so far apart that the last one begins behind 2^31 logits."""
    rows, vocab, stride = 3, 5000, 1_100_000_003
    buf = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, vocab), (stride, 1))
    g = torch.Generator().manual_seed(0)
    x.copy_(_logits(g, rows, vocab, torch.bfloat16))
    check(x, torch.rand(rows, generator=g).cuda(), top_p=0.9)
    check(x, torch.rand(rows, generator=g).cuda(), top_k=20)
