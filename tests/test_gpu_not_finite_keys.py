"""Keys that are not finite in a decode step's context.  A key that makes a score NaN makes every head that sees it NaN, wherever in the
context it lies and however the context is split; a key that scores minus infinity weighs nothing, whatever was met before it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HKV = 2


class Step:
    """A pool of `slots` traces that share their first length - 1 tokens, and one step's rows."""

    def __init__(self, dtype, hq, slots, length, seed=0):
        from paper_2608_08020_gb300.pool import TORCH_DT
        self.dtype, self.hq, self.slots, self.length = dtype, hq, slots, length
        self.d, self.dt = (64 if dtype == "f32" else 128), TORCH_DT[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(self.dt)  # noqa: E731
        self.kv = self.rand(2, 1, max(1, length - 1), HKV, self.d)
        self.q, self.new = self.rand(slots, hq, self.d), self.rand(2, slots, HKV, self.d)

    def run(self, flags):
        from paper_2608_08020_gb300.pool import BeamPool
        pages = -(-self.length // 16) + 1
        pool = BeamPool(num_layers=1, num_q_heads=self.hq, num_kv_heads=HKV, head_dim=self.d, page_size=16, kv_dtype=self.dtype,
                        num_pages=pages + 2 * self.slots, max_beams=self.slots, max_pages_per_beam=pages)
        pool.seed(self.slots, self.kv.shape[2], self.kv[0], self.kv[1])
        if self.length == 1:
            pool.truncate(torch.zeros(self.slots, dtype=torch.int32, device="cuda"))
        out = torch.full((self.slots, self.hq, self.d), 7.0, device="cuda")
        pool.decode_attention(0, self.q, self.new[0], self.new[1], self.d ** -0.5, out, flags)
        assert pool.status() == 0
        return out


@pytest.mark.parametrize("dtype,hq", [("fp8", 2), ("fp8", 8), ("fp8", 16), ("bf16", 4), ("bf16", 8), ("bf16", 16), ("f32", 4), ("f32", 16)])
@pytest.mark.parametrize("slots,length", [(3, 1), (3, 33), (3, 65), (2, 300), (1, 4000), (40, 1500)])
@pytest.mark.parametrize("flags", [0, 1, 2])
def test_a_key_that_is_not_a_number(cuda, dtype, hq, slots, length, flags):
    """In head 1's K, at the ends of tiles, in the shared part and in one trace's newest token; the other head stays as it was."""
    t = Step(dtype, hq, slots, length)
    clean = t.run(flags)
    assert bool(clean.isfinite().all())
    g = hq // HKV
    for at in sorted({0, 15, 16, 31, 32, length // 2, length - 2, length - 1}):
        if not 0 <= at < length:
            continue
        sees = slice(slots // 2, slots // 2 + 1) if at == length - 1 else slice(None)
        for bad in (float("nan"), float("inf")):
            if bad == float("inf") and dtype != "fp8":       # (8 bits hold it as NaN)
                continue
            row = t.new[0, sees, 1] if at == length - 1 else t.kv[0, 0, at, 1]
            was = row[..., 5].clone()
            row[..., 5] = bad
            out = t.run(flags)
            row[..., 5] = was
            want = torch.zeros_like(out, dtype=torch.bool)
            want[sees, g:] = True
            assert torch.equal(out.isnan(), want), f"token {at}"
            assert torch.equal(out[~want], clean[~want]), f"token {at}"


@pytest.mark.parametrize("dtype,hq", [("bf16", 4), ("bf16", 8), ("bf16", 16), ("f32", 4), ("f32", 16)])
@pytest.mark.parametrize("slots,length", [(3, 33), (3, 65), (2, 300), (1, 4000), (40, 1500)])
@pytest.mark.parametrize("flags", [0, 1, 2])
def test_scores_of_minus_infinity(cuda, dtype, hq, slots, length, flags):
    """The context's first tokens, a range inside it, all but the newest, all: as with scores so low that they weigh nothing."""
    t = Step(dtype, hq, slots, length)
    t.q[..., 0] = t.q[..., 0].abs() + 0.5
    for lo, hi in ((0, 1), (0, 16), (0, 31), (0, length // 2), (length // 3, length - 1), (0, length - 1)):
        was = t.kv[0, 0, lo:hi, :, 0].clone()
        outs = []
        # 0.5 x -1e6 / sqrt(128) is below -40000: its weight is 0 in fp32, too, beside scores of some tens.
        for low in (float("-inf"), -1e6):
            t.kv[0, 0, lo:hi, :, 0] = low
            outs.append(t.run(flags))
        t.kv[0, 0, lo:hi, :, 0] = was
        assert bool(outs[1].isfinite().all()) and torch.equal(*outs), f"tokens {lo} to {hi}"
    t.kv[0, 0, :, :, 0] = t.new[0, :, :, 0] = float("-inf")
    assert bool(t.run(flags).isnan().all())
