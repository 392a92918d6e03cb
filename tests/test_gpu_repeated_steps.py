"""The same steps of an 8-bit pool give the same bits however often they are run: no result depends on the order in which beams came to a
shared segment's list."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 4), (8, 2), (16, 2)])
@pytest.mark.parametrize("slots", [40, 150])
def test_shared_steps_from_fresh_pools(cuda, hq, hkv, slots):
    """Lists whose last query rows are 8 to 56 of 64; a fork makes a second level of them."""
    from paper_2608_08020_gb300.pool import BeamPool
    g = torch.Generator(device="cuda").manual_seed(slots)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    prompt, chunk = rand(2, 1, 1000, hkv, 128), rand(2, 300, slots, hkv, 128)
    steps = [(rand(slots, hq, 128), rand(slots, hkv, 128), rand(slots, hkv, 128)) for _ in range(2)]
    parents = torch.tensor([b if b % 5 < 2 else b - b % 5 for b in range(slots)], dtype=torch.int32, device="cuda")
    first = None
    for _ in range(6):
        pool = BeamPool(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, page_size=16, kv_dtype="fp8",
                        num_pages=63 + 25 * slots, max_beams=slots, max_pages_per_beam=90)
        pool.seed(slots, 1000, prompt[0], prompt[1])
        pool.append_kv(0, 300, chunk[0], chunk[1])
        pool.fork_slots(parents)
        out = torch.zeros(2, slots, hq, 128, device="cuda")
        for i, (q, k, v) in enumerate(steps):
            pool.decode_attention(0, q, k, v, 128 ** -0.5, out[i], 2)
        assert pool.status() == 0
        first = out if first is None else first
        assert torch.equal(out, first)
