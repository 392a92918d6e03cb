"""A Rotation dropped while calls that use it are still to run: its memory goes to nobody else before they have."""
import pytest
import torch

pytestmark = pytest.mark.gpu
N = 4000


def _pool(dtype):
    from paper_2608_08020_gb300.pool import TORCH_DT, BeamPool
    d = 64 if dtype == "f32" else 128
    pool = BeamPool(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=d, page_size=16, kv_dtype=dtype, num_pages=64, max_beams=2,
                    max_pages_per_beam=16)
    pool.seed(2, 30, *torch.zeros(2, 1, 30, 2, d, dtype=TORCH_DT[dtype], device="cuda"))
    return pool, d, TORCH_DT[dtype]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("call", ["append", "decode"])
def test_dropped_before_it_is_used(cuda, dtype, given, call):
    """A side stream, given or the current one, that is still busy when the object goes and its memory is asked for again."""
    from paper_2608_08020_gb300.rotation import Rotation
    held = []
    for early in (False, True):
        torch.cuda.empty_cache()
        pool, d, dt = _pool(dtype)
        k = torch.ones(7, 2, 2, d, dtype=dt, device="cuda")
        q, out = torch.ones(2, 8, d, dtype=dt, device="cuda"), torch.zeros(2, 8, d, device="cuda")
        rotation = Rotation(d, max_positions=N)
        size = rotation.table.shape
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)               # some 50 ms
        on = {"stream": side} if given else {}
        with torch.cuda.stream(None if given else side):
            if call == "append":
                pool.append_kv(0, 7, k, k, rotation=rotation, **on)
            else:
                pool.decode_attention(0, q, k[0], k[0], 0.1, out, rotation=rotation, **on)
        if early:
            del rotation
            others = [torch.full(size, 9.0, device="cuda") for _ in range(8)]  # noqa: F841  (one has the memory that was the table's)
        torch.cuda.synchronize()
        keys, _ = pool.read_kv(0, torch.full((2,), 30, dtype=torch.int32, device="cuda"), 7)
        held.append((keys, out))
        assert pool.status() == 0
    assert torch.equal(held[0][0], held[1][0]) and torch.equal(held[0][1], held[1][1])
