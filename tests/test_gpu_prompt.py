"""Attention over packed prompts against the definition in 64 bits.

Bounds, elementwise, with A = sum_j p_j |v_j|: bf16 rounds each p and the result by at most eps / 2 = 2^-8 of
the value, so |err| <= 2^-8 (A + |o|); the sums in fp32 and the exponentials (2^-22 relative in ex2, and
an exponent off by 2^-23 of its size, |exponent| <= 64 here) stay below 2e-5 A.  fp32: the scores' sums of 64
products and the exponents are off by at most 64 x 2^-24 x sum |q k| (below 2e-5 here), so 4e-5 A."""
import math

import pytest

pytestmark = pytest.mark.gpu


def attend(q, k, v, cu, scale):
    """(out, sum p |v|) in 64 bits, sequence by sequence; zeros outside them."""
    import torch
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    a = torch.zeros_like(o)
    g = q.shape[1] // k.shape[1]
    for s, e in zip(cu, cu[1:]):
        n = e - s
        if n <= 0:
            continue
        kk, vv = (x[s:e].double().repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))
        x = q[s:e].double().transpose(0, 1) @ kk.transpose(1, 2) * scale
        x.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1), -math.inf)
        p = torch.softmax(x, -1)
        o[s:e] = (p @ vv).transpose(0, 1)
        a[s:e] = (p @ vv.abs()).transpose(0, 1)
    return o, a


def bound(o, a, dtype):
    return (a + o.abs()) * 2.0 ** -8 + 2e-5 * a if dtype == "bf16" else 4e-5 * a


def make(dtype, total, hq, hkv, seed, fused=False, scale_q=1.0):
    import torch
    from paper_2608_08020_gb300.pool import TORCH_DT
    d = 128 if dtype == "bf16" else 64
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(total, hq + 2 * hkv, d, generator=g, device="cuda")
    x[:, :hq] *= scale_q
    x = x.to(TORCH_DT[dtype])
    parts = x.split([hq, hkv, hkv], 1)
    return parts if fused else [t.contiguous() for t in parts]


def run(dtype, lengths, hq, hkv, *, seed=0, fused=False, pad=0, scale=None, scale_q=1.0):
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    total = cu[-1] + pad
    q, k, v = make(dtype, total, hq, hkv, seed, fused, scale_q)
    d = q.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    op = PromptAttention(hq, hkv, d, dtype, max_tokens=total, max_seqs=len(lengths))
    out = torch.full((total, hq, d), 7.0, dtype=q.dtype, device="cuda")
    assert op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), scale, out) is out
    assert op.status() == 0
    o, a = attend(q, k, v, cu, scale)
    err = (out.double() - o).abs()[:cu[-1]]
    lim = bound(o, a, dtype)[:cu[-1]]
    assert bool((err <= lim).all()), float((err / lim).nan_to_num(9e9).max())
    assert bool((out[cu[-1]:] == 7).all())
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1025])
def test_one_prompt(cuda, dtype, n):
    run(dtype, [n], 8, 2, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (2, 1), (6, 3), (32, 8), (8, 1), (16, 1)])
def test_head_layouts(cuda, dtype, hq, hkv):
    run(dtype, [1, 40, 0, 300, 17, 129], hq, hkv, seed=hq, fused=True, pad=5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed(cuda, dtype):
    run(dtype, [0, 0, 3, 700, 1, 1, 64, 0, 1300, 128, 33, 0], 16, 4, seed=3, pad=200)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_short_sequences(cuda, dtype):
    run(dtype, [i % 4 for i in range(2500)], 4, 2, seed=4)


@pytest.mark.parametrize("scale_q", [0.0, 1e-3, 6.0])
def test_flat_and_sharp_scores(cuda, scale_q):
    run("bf16", [900], 8, 2, seed=5, scale_q=scale_q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_out_of_sight(cuda, dtype):
    """Infinities and NaN in later tokens and in other sequences do not reach a row; where it sees them they do."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make(dtype, 400, 8, 2, 9)
    d = q.shape[2]
    v[100, 0, 5] = float("inf")                # sequence 0: rows from 100 on
    v[130, :, d - 1] = float("nan")
    k[250] = float("nan")                      # sequence 1: rows from 250 on
    v[251] = float("nan")
    q[390:], k[390:], v[390:] = float("nan"), float("nan"), float("nan")
    cu = [0, 160, 300, 380]
    op = PromptAttention(8, 2, d, dtype, max_tokens=400, max_seqs=3)
    out = op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 1 / math.sqrt(d))
    clean = [x.clone() for x in (k, v)]
    clean[1][100, 0, 5], clean[1][130, :, d - 1], clean[0][250], clean[1][251] = 0, 0, 0, 0
    for s, e in zip(cu, cu[1:]):
        for i in range(s, e):
            # What row i sees, in 64 bits.
            kk, vv = (x[s:i + 1].double().repeat_interleave(4, 1) for x in (k, v))
            p = torch.softmax(torch.einsum("hd,thd->ht", q[i].double(), kk) / math.sqrt(d), -1)
            o, a = torch.einsum("ht,thd->hd", p, vv), torch.einsum("ht,thd->hd", p, vv.abs())
            ok = o.isfinite()
            assert torch.equal(out[i].isfinite(), ok), i
            assert bool(((out[i].double() - o).abs() <= bound(o, a, dtype))[ok].all()), i
    assert op.status() == 0


def test_bad_sequences_are_left_out(cuda):
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make("bf16", 300, 4, 2, 10)
    op = PromptAttention(4, 2, 128, "bf16", max_tokens=300, max_seqs=4)
    for cu, fine in (([0, 100, 90, 200, 300], [(0, 100), (90, 200), (200, 300)]), ([-5, 100, 200, 300, 400], [(100, 200), (200, 300)])):
        out = torch.full_like(q, 7.0)
        op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1, out)
        assert B.STATUS_NAMES[op.status()] == "GB_ERR_INVALID"
        assert bool(out.isfinite().all())
        for s, e in fine[-1:]:
            o, a = attend(q, k, v, [s, e], 0.1)
            assert bool(((out.double() - o).abs() <= bound(o, a, "bf16"))[s:e].all())
    op(q, k, v, torch.tensor([0, 300], dtype=torch.int32, device="cuda"), 0.1)
    assert op.status() == 0


def test_streams_and_graphs(cuda):
    """On another stream, and captured once and replayed with other lengths and values."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make("bf16", 700, 8, 2, 11)
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=700, max_seqs=5)
    cu = torch.tensor([0, 1, 300, 300, 650, 700], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op(q, k, v, cu, 0.1, out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        op(q, k, v, cu, 0.1, out)
    for lengths in ([0, 1, 300, 300, 650, 700], [0, 0, 0, 64, 600, 700], [0, 700, 700, 700, 700, 700]):
        cu.copy_(torch.tensor(lengths, dtype=torch.int32))
        for x, y in zip((q, k, v), make("bf16", 700, 8, 2, lengths[3])):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        o, a = attend(q, k, v, lengths, 0.1)
        assert bool(((out.double() - o).abs() <= bound(o, a, "bf16")).all())


def test_wrapper_refuses(cuda):
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make("bf16", 64, 4, 2, 12)
    op = PromptAttention(4, 2, 128, "bf16", max_tokens=64, max_seqs=2)
    cu = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    for args in ((q[:, :2], k, v, cu), (q.float(), k, v, cu), (q, k[:60], v, cu), (q, k, v.transpose(0, 1).contiguous().transpose(0, 1), cu),
                 (q, k, v, cu.long()), (q, k, v, cu.cpu()), (q, k, v, torch.zeros(4, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            op(*args, 0.1)


def test_units_of_one_tile_in_a_row(cuda):
    """Many sequences within one tile of keys, where one of a unit's two groups has nothing to do, over and over: the
    same result each time."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    lengths = [1 + (7 * i) % 32 for i in range(900)]
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    q, k, v = make("bf16", cu[-1], 8, 2, 13)
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=cu[-1], max_seqs=900)
    at = torch.tensor(cu, dtype=torch.int32, device="cuda")
    first = op(q, k, v, at, 0.1)
    o, a = attend(q, k, v, cu, 0.1)
    assert bool(((first.double() - o).abs() <= bound(o, a, "bf16")).all())
    for _ in range(200):
        out = op(q, k, v, at, 0.1)
    assert torch.equal(out, first) and op.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_sequence_and_empty_ones(cuda, dtype):
    run(dtype, [], 4, 2, pad=7)
    run(dtype, [0], 4, 2, pad=7)
    run(dtype, [0, 0, 0], 4, 2, pad=300)
    run(dtype, [5], 4, 2, pad=300)
    run(dtype, [], 4, 2)


def test_one_bad_sequence(cuda):
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.prompt import PromptAttention
    for dtype in ("bf16", "f32"):
        q, k, v = make(dtype, 200, 4, 2, 14)
        op = PromptAttention(4, 2, q.shape[2], dtype, max_tokens=200, max_seqs=1)
        assert op.status() == 0
        out = torch.full_like(q, 7.0)
        for cu, code in (([0, 201], "GB_ERR_INVALID"), ([10, 5], "GB_ERR_INVALID"), ([-1, 100], "GB_ERR_INVALID"), ([3, 3], "GB_OK")):
            op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1, out)
            assert B.STATUS_NAMES[op.status()] == code and bool((out == 7).all()), (dtype, cu)
        op(q, k, v, torch.tensor([50, 200], dtype=torch.int32, device="cuda"), 0.1, out)   # not from the first row
        o, a = attend(q, k, v, [50, 200], 0.1)
        assert op.status() == 0 and bool((out[:50] == 7).all())
        assert bool(((out.double() - o).abs() <= bound(o, a, dtype))[50:].all())


def test_the_same_each_time(cuda):
    """Lists of many units of one length: the same bits from every call, on any stream, with a new output."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    lengths = [37 * (1 + i % 9) for i in range(70)]
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    q, k, v = make("bf16", cu[-1], 8, 2, 15)
    op = PromptAttention(8, 2, 128, "bf16", max_tokens=cu[-1], max_seqs=70)
    at = torch.tensor(cu, dtype=torch.int32, device="cuda")
    first = op(q, k, v, at, 0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):
        out = op(q, k, v, at, 0.1, stream=side)
        side.synchronize()
        assert torch.equal(out, first)
    with pytest.raises(ValueError):
        op(q, k, v, at, 0.1, stream=side.cuda_stream)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bounds_that_name_rows_again(cuda, dtype):
    """Sequences that begin before an earlier one's end are left out, thousands of them too."""
    import torch
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.prompt import PromptAttention
    q, k, v = make(dtype, 2000, 4, 2, 16)
    op = PromptAttention(4, 2, q.shape[2], dtype, max_tokens=2000, max_seqs=200000)
    out = torch.full_like(q, 7.0)
    op(q, k, v, torch.tensor([0, 2000] * 100000, dtype=torch.int32, device="cuda"), 0.1, out)
    assert B.STATUS_NAMES[op.status()] == "GB_ERR_INVALID"
    o, a = attend(q, k, v, [0, 2000], 0.1)
    assert bool(((out.double() - o).abs() <= bound(o, a, dtype)).all())
    op(q, k, v, torch.tensor([0, 2000, 1000, 1500], dtype=torch.int32, device="cuda"), 0.1, out)
    assert B.STATUS_NAMES[op.status()] == "GB_ERR_INVALID"
    assert bool(((out.double() - o).abs() <= bound(o, a, dtype)).all())
    cu = [-1, 0] + [2 * i // 3 for i in range(1500)] + [9999, 500, 1000, 1200, 1100, 1150, 1200, 2000]   # ... 999, then past the end
    out.fill_(7.0)
    op(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.1, out)
    assert B.STATUS_NAMES[op.status()] == "GB_ERR_INVALID"
    o, a = attend(q, k, v, sorted({2 * i // 3 for i in range(1500)}), 0.1)
    fine = (out.double() - o).abs() <= bound(o, a, dtype)
    assert bool(fine[:999].all()) and bool((out[999] == 7).all())
    o, a = attend(q, k, v, [1000, 1200, 2000], 0.1)
    assert bool(((out.double() - o).abs() <= bound(o, a, dtype))[1000:].all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(cuda, dtype):
    """Token strides with which the last rows lie behind 2^31 elements."""
    import torch
    from paper_2608_08020_gb300.prompt import PromptAttention
    n, stride = 2300, 1 << 20
    q, k, v = make(dtype, n, 4, 2, 17)
    d = q.shape[2]
    rows, res = (torch.zeros(n, stride, dtype=q.dtype, device="cuda") for _ in range(2))
    wide = [rows[:, a * d:b * d].unflatten(1, (-1, d)) for a, b in ((0, 4), (4, 6), (6, 8))]
    for x, y in zip(wide, (q, k, v)):
        x.copy_(y)
    out = res[:, :4 * d].unflatten(1, (-1, d))
    op = PromptAttention(4, 2, d, dtype, max_tokens=n, max_seqs=2)
    op(*wide, torch.tensor([0, 100, n], dtype=torch.int32, device="cuda"), 0.1, out)
    o, a = attend(q, k, v, [0, 100, n], 0.1)
    assert op.status() == 0
    assert bool(((out.double() - o).abs() <= bound(o, a, dtype)).all())
    assert not bool(res[:, 4 * d:5 * d].any())
