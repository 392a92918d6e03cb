"""The failure path of the 8-bit attention without a fault: a load of each CTA that never comes, waits that run out.

gb_decode_wait_selftest leaves one load a CTA out.  The call must end, record GB_ERR_TIMEOUT, give every output that is right or zero,
and leave the pool usable."""
import time

import pytest
import torch

from tests.cache8 import attention
from tests.test_gpu_pool8 import Both, _rand

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


def stalled_step(t, flags, stalled):
    """One step with a load left out: its rows join the model; (the outputs, which (slot, KV head) are zero, which right)."""
    from paper_2608_08020_gb300 import binding as B
    q, (k, v) = _rand(t.g, t.slots, t.hq, 128, wide=False), (_rand(t.g, t.slots, t.hkv, 128, wide=False) for _ in range(2))
    out = torch.full((t.slots, t.hq, 128), 7.0, device="cuda")
    B.gb_decode_wait_selftest(t.pool.handle, 0, q.cuda(), k.cuda(), v.cuda(), SCALE, out, flags, stalled)
    out, g = out.cpu().double(), t.hq // t.hkv
    zero = torch.zeros(t.slots, t.hkv, dtype=torch.bool)
    right = zero.clone()
    for b in range(t.slots):
        if b not in t.live:
            zero[b] = (out[b] == 0).all()
            continue
        t.model.append(b, 0, k[b:b + 1].double(), v[b:b + 1].double())
        ref, a, dot, top = attention(q[b].double(), t.model.kv[b][0], SCALE)
        tol = a * (2 * dot[:, None] * 2.0 ** -17 + 2.0 ** -18) + t.model.length(b) * 448 * 2.0 ** -31 * top[:, None]   # (Both.check_out)
        right[b] = ((out[b] - ref).abs() <= tol).view(t.hkv, -1).all(1)
        zero[b] = (out[b] == 0).view(t.hkv, -1).all(1)
    return zero, right


def make(name):
    if name == "one":                                     # its chunks shared out among a few CTAs
        t = Both(slots=1, hq=4, hkv=1, pages=200, width=200)
        t.seed(1, 3000, wide=False)
    elif name == "pairs":                                 # a unit a pair, in a pool with vacant slots
        t = Both(slots=24, hq=16, hkv=4, pages=400, width=20)
        t.seed(20, 100, wide=False)
        t.append(40, wide=False)
    else:                                                 # segments, and tails behind them
        t = Both(slots=40, hq=8, hkv=2, pages=600, width=80)
        t.seed(40, 1000, wide=False)
        t.append(30, wide=False)
    return t


@pytest.mark.parametrize("name", ["one", "pairs", "shared"])
@pytest.mark.parametrize("flags,stalled", [(1, 0), (1, 3), (2, 0), (2, 3), (2, 9)])
def test_a_load_that_never_comes(cuda, name, flags, stalled):
    from paper_2608_08020_gb300 import binding as B
    t = make(name)
    t.decode(flags=flags)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    zero, right = stalled_step(t, flags, stalled)
    took = time.perf_counter() - t0
    status = t.pool.status()
    assert bool((zero | right).all())
    assert status in (B.GB_ERR_TIMEOUT, B.GB_OK)
    if status == B.GB_ERR_TIMEOUT:
        assert 1.5 < took < 30 and bool(zero[t.live].any())
    else:                                                 # no CTA had so many stages
        assert stalled > 0 and bool(right[t.live].all())
    if stalled == 0:
        assert status == B.GB_ERR_TIMEOUT
    t.pool.clear_status()
    t.decode(flags=flags)                                 # asks for status 0
    t.check_cache()


def test_a_stage_that_no_cta_has(cuda):
    t = make("pairs")
    zero, right = stalled_step(t, 0, 10 ** 6)
    assert t.pool.status() == 0 and bool(right[t.live].all())


def test_refusals(cuda):
    from paper_2608_08020_gb300 import binding as B
    from paper_2608_08020_gb300.pool import BeamPool
    t = make("one")
    x = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(1, 4, 128, device="cuda")
    with pytest.raises(B.GambitError, match="GB_ERR_INVALID"):
        B.gb_decode_wait_selftest(t.pool.handle, 0, x, x, x, 0.1, out, 0, -1)
    p = BeamPool(num_layers=1, num_q_heads=4, num_kv_heads=2, head_dim=128, page_size=16, kv_dtype="bf16", num_pages=8, max_beams=1,
                 max_pages_per_beam=4)
    with pytest.raises(B.GambitError, match="GB_ERR_UNSUPPORTED"):
        B.gb_decode_wait_selftest(p.handle, 0, x, x, x, 0.1, out, 0, 0)
    t.decode()
