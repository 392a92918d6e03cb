"""Thoughts of many slots at once, whose heads a team of warps writes one after the other, against the definition."""
import pytest
import torch

from tests.cache8 import rotated
from tests.test_gpu_pool8 import Both, _rand
from tests.test_gpu_rotation import BASE, _ints, _pool, _round

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hkv,n", [(8, 40), (6, 25), (3, 60), (1, 150)])
def test_many_slots_of_8_bits(cuda, hkv, n):
    """Blocks begun by the call before, raised scales, values that are not finite, and slots that hold nothing."""
    slots, live = 230, 200
    t = Both(hq=hkv, hkv=hkv, slots=slots, pages=16 * slots, width=24, seed=hkv)
    t.seed(live, 21)
    t.append(5)
    k, v = (_rand(t.g, n, slots, hkv, 128) for _ in range(2))
    k[n // 2, 3, 0, 7] = float("inf")
    v[0, 5, hkv - 1, 0] = float("nan")
    t.append(n, k, v)
    t.truncate([(b * 7) % (20 + n) + 1 for b in range(slots)])
    t.append(n // 2 + 1)
    t.check_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("hkv", [8, 3])
def test_many_slots_rotated(cuda, dtype, hkv):
    slots, n, at = 240, 45, 21
    pool, d, dt = _pool(dtype, layers=1, hq=2 * hkv, hkv=hkv, slots=slots, pages=8 * slots, width=8)
    from paper_2608_08020_gb300.rotation import Rotation
    g = torch.Generator().manual_seed(hkv)
    rows = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
    seed = rows(2, 1, at, hkv, d)
    pool.seed(slots, at, seed[0].cuda(), seed[1].cuda())
    k, v = rows(n, slots, hkv, d), rows(n, slots, hkv, d)
    pool.append_kv(0, n, k.cuda(), v.cuda(), rotation=Rotation(d, max_positions=300, base=BASE))
    kc, vc = (x.cpu() for x in pool.read_kv(0, _ints([at] * slots), n))
    want = torch.stack([rotated(k[j].double(), at + j, d, BASE) for j in range(n)])
    if dtype == "fp8":       # the model of one pool of slots is slow: a block that no row of the prompt shares, by its largest value
        lo, hi = 32 - at, 48 - at
        for held, exact in ((kc, want.float().double()), (vc, v.double())):
            x = exact[lo:hi]
            top = x.abs().amax((0, 3), keepdim=True)
            e = torch.ceil(torch.log2(top / 448)).clamp(-60, 60)
            e = torch.where(top > 448 * 2.0 ** (e - 1), e, e - 1)
            unit = (x / 2.0 ** e).float().to(torch.float8_e4m3fn).double() * 2.0 ** e
            assert torch.equal(held[lo:hi].double(), unit)
    else:
        assert torch.equal(kc, _round(want, dt)) and torch.equal(vc, v)
    assert pool.status() == 0
