"""Rotated keys that are infinite, no numbers or so large that a rotation passes the type's range: as the formula gives them."""
import math

import pytest
import torch

from tests.cache8 import rotated
from tests.test_gpu_rotation import BASE, _ints, _pool, _rotation, _round

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_appended_and_decoded_keys(cuda, dtype, interleaved):
    pool, d, dt = _pool(dtype, layers=1, slots=2)
    rot = _rotation(d, interleaved=interleaved)
    z = torch.zeros(1, 1, 2, d, dtype=dt, device="cuda")
    pool.seed(2, 1, z, z)
    pool.truncate(_ints([0, 0]))                          # position 0, whose sines are 0, too
    n, inf = 40, math.inf
    g = torch.Generator().manual_seed(3)
    k = torch.randn(n + 1, 2, 2, d, generator=g)
    odd = torch.tensor([inf, -inf, math.nan, 3.2e38, -3.2e38, 1e-38, 0.0, -0.0])
    at = torch.rand(k.shape, generator=g) < 0.1
    k[at] = odd[torch.randint(0, 8, (int(at.sum()),), generator=g)]
    k = k.to(dt)
    pool.append_kv(0, n, k[:n].cuda(), k[:n].cuda(), rotation=rot)
    pool.decode_attention(0, torch.zeros(2, 8, d, dtype=dt, device="cuda"), k[n].cuda(), k[n].cuda(), 0.1, torch.zeros(2, 8, d, device="cuda"),
                          rotation=rot)
    got = pool.read_kv(0, _ints([0, 0]), n + 1)[0].cpu()
    want = torch.stack([_round(rotated(k[t].double(), t, d, BASE, interleaved), dt) for t in range(n + 1)])
    assert bool(want.isinf().any()) and bool(want.isnan().any())
    assert torch.equal(got.isnan(), want.isnan())
    ok = (got == want) | want.isnan()
    # Values near the least normal one: what the rounding errors' own products fall below is lost, 2^-149 each.
    ok |= (got.double() - want.double()).abs() <= 2.0 ** -146
    assert bool(ok.all()), (got[~ok], want[~ok])
