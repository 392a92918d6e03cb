"""Attention over long caches of 8 bits, whose chunks the CTAs share out in even parts and small ones: against the definition over
the cache as it is read back, in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _check(pool, lengths, q, out, scale):
    slots, hq, d = q.shape
    most = max(lengths)
    k, v = (x.double() for x in pool.read_kv(0, torch.zeros(slots, dtype=torch.int32, device="cuda"), most))
    g = hq // k.shape[2]
    for b in range(slots):
        if lengths[b] == 0:
            assert (out[b] == 0).all()
            continue
        kk, vv = (x[:lengths[b], b].transpose(0, 1).repeat_interleave(g, 0) for x in (k, v))      # [hq][T][d]
        qq = q[b].double()[:, :, None]
        p = ((kk @ qq)[..., 0] * scale).softmax(-1)[:, None]
        ref, a = (p @ vv)[:, 0], (p @ vv.abs())[:, 0]
        dot = ((kk.abs() @ qq.abs())[..., 0] * scale).amax(-1, keepdim=True)
        # As in test_gpu_pool8: 128 products in fp32, twice; exponential, terms and sums; the second term's last place, for which
        # 448 2^e of a block is at most twice its largest value.
        tol = a * (2 * dot * 2.0 ** -17 + 2.0 ** -18) + lengths[b] * 2.0 ** -30 * vv.abs().amax((1, 2))[:, None] * p[:, 0].amax(-1)[:, None]
        err = (out[b].double() - ref).abs()
        assert (err <= tol).all(), f"slot {b}: {float((err / tol).max()):.2f} of the bound"


@pytest.mark.parametrize("hq,hkv,slots,length", [(8, 8, 9, 6500), (32, 8, 6, 9000), (32, 4, 11, 9000), (2, 1, 3, 70000), (4, 2, 150, 1500)])
def test_traces_that_share_nothing(cuda, hq, hkv, slots, length):
    from paper_2608_08020_gb300.pool import BeamPool
    g = torch.Generator(device="cuda").manual_seed(hq + slots)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    width = length // 16 + 3
    pool = BeamPool(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, page_size=16, kv_dtype="fp8",
                    num_pages=width * slots, max_beams=slots, max_pages_per_beam=width)
    pool.seed(slots - 1, 1, rand(1, 1, hkv, 128), rand(1, 1, hkv, 128))           # (the last slot stays empty)
    for n in (length // 3, length - length // 3 - 1):
        pool.append_kv(0, n, rand(n, slots, hkv, 128), rand(n, slots, hkv, 128))
    lengths = [length - 37 * b for b in range(slots - 1)] + [0] if length > 37 * slots else [length - 9 * b for b in range(slots - 1)] + [0]
    pool.truncate(torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    out = torch.full((slots, hq, 128), float("nan"), device="cuda")
    for flags in (0, 1, 2):
        q = rand(slots, hq, 128)
        pool.decode_attention(0, q, rand(slots, hkv, 128), rand(slots, hkv, 128), 128 ** -0.5, out.fill_(float("nan")), flags)
        lengths = [x + 1 if x else 0 for x in lengths]
        _check(pool, lengths, q, out, 128 ** -0.5)
    assert pool.status() == 0


@pytest.mark.parametrize("hq,hkv,slots", [(8, 8, 40), (16, 8, 30), (32, 8, 21), (32, 4, 50)])
def test_traces_with_shared_prefixes(cuda, hq, hkv, slots):
    from paper_2608_08020_gb300.pool import BeamPool
    g = torch.Generator(device="cuda").manual_seed(hq + slots)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    rng = torch.Generator().manual_seed(slots)
    pool = BeamPool(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, page_size=16, kv_dtype="fp8",
                    num_pages=400 * slots, max_beams=slots, max_pages_per_beam=220)
    prompt = 700
    pool.seed(slots, prompt, rand(1, prompt, hkv, 128), rand(1, prompt, hkv, 128))
    length = prompt
    for n in (300, 517, 650):
        pool.append_kv(0, n, rand(n, slots, hkv, 128), rand(n, slots, hkv, 128))
        length += n
        parents = torch.arange(slots, dtype=torch.int32)
        order = torch.randperm(slots, generator=rng)
        lost = order[:slots // 2]
        parents[lost] = order[slots // 2:][torch.randint(0, slots - slots // 2, (len(lost),), generator=rng)].int()
        pool.fork_slots(parents.cuda())
    out = torch.empty(slots, hq, 128, device="cuda")
    for flags in (2, 1, 0):
        q = rand(slots, hq, 128)
        pool.decode_attention(0, q, rand(slots, hkv, 128), rand(slots, hkv, 128), 128 ** -0.5, out.fill_(float("nan")), flags)
        length += 1
        _check(pool, [length] * slots, q, out, 128 ** -0.5)
    assert pool.status() == 0


def test_offsets_past_32_bits(cuda):
    """The last layer of a pool of 25 GB: its rows and scales written, copied on write, read and attended to."""
    from paper_2608_08020_gb300.pool import BeamPool
    from paper_2608_08020_gb300.rotation import Rotation
    layers, hq, hkv, slots = 40, 16, 8, 4
    pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, page_size=16, kv_dtype="fp8", num_pages=19000,
                    max_beams=slots, max_pages_per_beam=16)
    assert pool.kv.numel() > 5 << 32
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    rotation = Rotation(128, max_positions=300)
    seed, new = rand(2, layers, 70, hkv, 128), rand(2, layers, 30, slots, hkv, 128)
    pool.seed(slots, 70, seed[0], seed[1])
    for i in range(layers):
        pool.append_kv(i, 30, new[0, i], new[1, i], rotation=rotation)
    first = torch.zeros(slots, dtype=torch.int32, device="cuda")
    top = pool.read_kv(layers - 1, first, 100)
    for b in range(slots):                                  # 4 significant bits, and those of a block whose scale rose
        exact = torch.cat([seed[1, -1], new[1, -1, :, b]]).double()
        assert ((top[1][:, b].double() - exact).abs() <= 2.0 ** -3 * exact.abs() + 2.0 ** -8).all()
    q, k, v = rand(layers, slots, hq, 128), rand(layers, slots, hkv, 128), rand(layers, slots, hkv, 128)
    out = torch.empty(slots, hq, 128, device="cuda")
    for i in range(layers):
        pool.decode_attention(i, q[i], k[i], v[i], 128 ** -0.5, out)
    kc, vc = (x.double() for x in pool.read_kv(layers - 1, first, 101))
    for b in range(slots):
        kk, vv = (x[:, b].transpose(0, 1).repeat_interleave(2, 0) for x in (kc, vc))
        p = ((kk @ q[-1, b].double()[:, :, None])[..., 0] * 128 ** -0.5).softmax(-1)[:, None]
        # Scores are right to 2^-16 of sizes up to some tens, weights to 2^-18.
        assert ((out[b].double() - (p @ vv)[:, 0]).abs() <= 2.0 ** -11 * (p @ vv.abs())[:, 0]).all()
    assert pool.status() == 0
