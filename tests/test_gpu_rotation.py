"""Rows rotated on their way into pools of every type: what the cache then holds, and the attention of rotated steps."""
import pytest
import torch

from tests.cache8 import rotated
from tests.test_gpu_pool8 import Both

pytestmark = pytest.mark.gpu
BASE = 1e6


def _round(x, dtype):
    """float64 to the type of a pool's rows, as the library rounds: once."""
    return x.float().to(dtype)


def _pool(dtype, *, layers=2, hq=8, hkv=2, page=16, slots=5, pages=96, width=16):
    from paper_2608_08020_gb300.pool import TORCH_DT, BeamPool
    d = 64 if dtype == "f32" else 128
    pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=page, kv_dtype=dtype, num_pages=pages,
                    max_beams=slots, max_pages_per_beam=width)
    return pool, d, TORCH_DT[dtype]


def _rotation(d, **kw):
    from paper_2608_08020_gb300.rotation import Rotation
    return Rotation(d, **{"max_positions": 300, "base": BASE, **kw})


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("part", [16, 32, 48, 64, "all"])
def test_appended_keys_turn_values_stay(cuda, dtype, interleaved, part):
    """Slots of different lengths, the first chunk after a seed with a shared tail page, chunks over several pages."""
    pool, d, dt = _pool(dtype)
    r = d if part == "all" else part
    rot = _rotation(d, rotary_dim=r, interleaved=interleaved)
    g = torch.Generator().manual_seed(r)
    rows = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
    seed = rows(2, 2, 21, 2, d)
    pool.seed(4, 21, seed[0].cuda(), seed[1].cuda())
    lengths = [21] * 4
    held = [[(seed[0][i], seed[1][i]) for i in range(2)] for _ in range(4)]
    for n in (1, 5, 40):
        for i in range(2):
            k, v = rows(n, 5, 2, d), rows(n, 5, 2, d)
            pool.append_kv(i, n, k.cuda(), v.cuda(), rotation=rot)
            for b in range(4):
                kr = torch.stack([_round(rotated(k[j, b].double(), lengths[b] + j, r, BASE, interleaved), dt) for j in range(n)])
                held[b][i] = (torch.cat([held[b][i][0], kr]), torch.cat([held[b][i][1], v[:, b]]))
        lengths = [x + n for x in lengths]
        for i in range(2):
            k, v = pool.read_kv(i, _ints([0] * 5), max(lengths))
            for b in range(4):
                assert torch.equal(k[:lengths[b], b].cpu(), held[b][i][0]) and torch.equal(v[:lengths[b], b].cpu(), held[b][i][1])
            assert (k[:, 4] == 0).all() and (v[:, 4] == 0).all()
        cut = [lengths[0] - n // 2, -1, 9, lengths[3], -1]
        pool.truncate(_ints(cut))
        for b in range(4):
            if cut[b] >= 0:
                lengths[b] = cut[b]
                held[b] = [(x[:cut[b]], y[:cut[b]]) for x, y in held[b]]
    assert pool.status() == 0


@pytest.mark.parametrize("dtype,hq,hkv", [("f32", 8, 2), ("bf16", 8, 2), ("bf16", 2, 1), ("bf16", 16, 2)])
@pytest.mark.parametrize("flags", [0, 1, 2])
def test_rotated_steps_are_steps_on_rotated_rows(cuda, dtype, hq, hkv, flags):
    pool, d, dt = _pool(dtype, hq=hq, hkv=hkv)
    twin, _, _ = _pool(dtype, hq=hq, hkv=hkv)
    rot = _rotation(d)
    g = torch.Generator().manual_seed(hq)
    rows = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
    seed = rows(2, 2, 37, hkv, d).cuda()
    for p in (pool, twin):
        p.seed(4, 37, seed[0], seed[1])
    for step in range(4):
        for i in range(2):
            q, k, v = rows(5, hq, d), rows(5, hkv, d), rows(5, hkv, d)
            turned = [_round(rotated(x.double(), 37 + step, d, BASE), dt).cuda() for x in (q, k)]
            q, k, v = q.cuda(), k.cuda(), v.cuda()
            copies = [x.clone() for x in (q, k, v)]
            out, ref = torch.full((2, 5, hq, d), 7.0, device="cuda")
            pool.decode_attention(i, q, k, v, d ** -0.5, out, flags, rotation=rot)
            twin.decode_attention(i, *turned, v, d ** -0.5, ref, flags)
            assert torch.equal(out, ref)
            assert all(torch.equal(x, y) for x, y in zip((q, k, v), copies))
        if step == 1:
            for p in (pool, twin):
                p.fork_slots(_ints([0, 0, 2, 2, -1]))
    for i in range(2):
        for x, y in zip(pool.read_kv(i, _ints([0] * 5), 41), twin.read_kv(i, _ints([0] * 5), 41)):
            assert torch.equal(x, y)
    assert pool.status() == 0


def test_output_over_the_new_rows(cuda):
    """An output that overlaps the new rows, which the library takes care of without a rotation, with one."""
    for dtype in ("bf16", "fp8"):
        outs = []
        for over in (False, True):
            pool, d, dt = _pool(dtype, layers=1, slots=3)
            g = torch.Generator(device="cuda").manual_seed(0)
            rows = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
            pool.seed(3, 20, rows(1, 20, 2, d), rows(1, 20, 2, d))
            buf = torch.zeros(3 * 8 * d, device="cuda")
            kv = rows(2, 3, 2, d)
            k, v = buf.view(dt)[:kv.numel()].view_as(kv) if over else kv
            if over:
                k.copy_(kv[0])
                v.copy_(kv[1])
            out = buf.view(3, 8, d) if over else torch.zeros(3, 8, d, device="cuda")
            pool.decode_attention(0, rows(3, 8, d), k, v, 0.1, out, rotation=_rotation(d))
            outs.append(out.clone())
            assert pool.status() == 0
        assert torch.equal(*outs)


@pytest.mark.parametrize("kw", [{}, {"rotary_dim": 32, "interleaved": True}, {"amplitude": 1.5}])
def test_eight_bits(cuda, kw):
    """Rotated rows of an 8-bit pool are rounded once, from the rotation; its rotated queries to bf16."""
    t = Both(layers=2, slots=4, page=32)
    rot = _rotation(128, **kw)
    r, inter, amp = kw.get("rotary_dim", 128), kw.get("interleaved", False), kw.get("amplitude", 1.0)
    turn = lambda x, pos: rotated(x.double(), pos, r, BASE, inter, amp)  # noqa: E731
    t.seed(3, 29, wide=False)
    at = 29
    rows = lambda *s: torch.randn(s, generator=t.g).to(torch.bfloat16)  # noqa: E731
    for n in (1, 20, 3):
        for i in range(2):
            k, v = rows(n, 4, 2, 128), rows(n, 4, 2, 128)
            t.pool.append_kv(i, n, k.cuda(), v.cuda(), rotation=rot)
            for b in t.live:
                kr = torch.stack([turn(k[j, b], at + j) for j in range(n)]).float().double()
                t.model.append(b, i, kr, v[:, b].double())
        at += n
        t.check_cache()
    for _ in range(3):
        for i in range(2):
            q, k, v = rows(4, 8, 128), rows(4, 2, 128), rows(4, 2, 128)
            out = torch.full((4, 8, 128), 7.0, device="cuda")
            t.pool.decode_attention(i, q.cuda(), k.cuda(), v.cuda(), 0.1, out, rotation=rot)
            for b in t.live:
                t.model.append(b, i, turn(k[b:b + 1], at).float().double(), v[b:b + 1].double())
            t.check_out(out.cpu(), _round(turn(q, at), torch.bfloat16), i, 0.1)
        at += 1
    t.check_cache()


def test_far_positions(cuda):
    """The last positions of a long table: the angles are exact to the rows' last place there."""
    pool, d, dt = _pool("f32", layers=1, slots=1, pages=8300, width=8300)
    n = 131000
    x = torch.zeros(1, 32000, 2, d, device="cuda")
    pool.seed(1, 32000, x, x)
    pool.append_kv(0, n - 32000, x[0, :1, None].expand(n - 32000, 1, 2, d).contiguous(), x[0, :1, None].expand(n - 32000, 1, 2, d).contiguous())
    k = torch.randn(5, 1, 2, d, generator=torch.Generator().manual_seed(1))
    pool.append_kv(0, 5, k.cuda(), k.cuda(), rotation=_rotation(d, max_positions=n + 5))
    got = pool.read_kv(0, _ints([n]), 5)[0].cpu()
    ref = torch.stack([rotated(k[j].double(), n + j, d, BASE) for j in range(5)])
    # One rounding to fp32, and 64-bit angles off by 2^-53 of 131000 radians.
    assert ((got.double() - ref).abs() <= 2.0 ** -24 * ref.abs() * 1.001 + 2.0 ** -35).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_positions_past_the_table(cuda, dtype):
    """They are not rotated, and the status says so; positions before them are."""
    pool, d, dt = _pool(dtype, layers=1, slots=2)
    z = torch.zeros(1, 30, 2, d, dtype=dt, device="cuda")
    pool.seed(2, 30, z, z)
    k = torch.ones(4, 2, 2, d, dtype=dt, device="cuda")
    pool.append_kv(0, 4, k, k, rotation=_rotation(d, max_positions=32))
    got = pool.read_kv(0, _ints([30, 30]), 4)[0]
    assert (got[2:] == 1).all() and not (got[:2] == 1).all()
    assert pool.status() == 1
    pool.clear_status()
    out = torch.zeros(2, 8, d, device="cuda")
    pool.decode_attention(0, torch.ones(2, 8, d, dtype=dt, device="cuda"), k[0], k[0], 0.1, out, rotation=_rotation(d, max_positions=32))
    assert (pool.read_kv(0, _ints([34, 34]), 1)[0] == 1).all() and pool.status() == 1


def test_captured_rotated_steps(cuda):
    """Replayed steps rotate to the positions that they run at."""
    for dtype in ("bf16", "fp8"):
        pools = [_pool(dtype, slots=3) for _ in range(2)]
        rot = _rotation(128)
        g = torch.Generator(device="cuda").manual_seed(2)
        rows = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        seed, q, k, v = rows(2, 2, 20, 2, 128), rows(2, 3, 8, 128), rows(2, 3, 2, 128), rows(2, 3, 2, 128)
        outs = torch.zeros(2, 2, 3, 8, 128, device="cuda")

        def step(pool, out):
            for i in range(2):
                pool.decode_attention(i, q[i], k[i], v[i], 0.1, out[i], rotation=rot)

        for pool, _, _ in pools:
            pool.seed(3, 20, seed[0], seed[1])
            step(pool, outs[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(pools[0][0], outs[0])
        for _ in range(15):
            graph.replay()
            step(pools[1][0], outs[1])
            assert torch.equal(outs[0], outs[1])
        for pool, _, _ in pools:
            assert pool.status() == 0


def test_refusals(cuda):
    from paper_2608_08020_gb300 import binding as B
    pool, d, dt = _pool("bf16", layers=1)
    z = torch.zeros(1, 20, 2, d, dtype=dt, device="cuda")
    pool.seed(5, 20, z, z)
    k = torch.zeros(1, 5, 2, d + 8, dtype=dt, device="cuda").flatten()
    good = _rotation(d)
    with pytest.raises(ValueError):
        pool.append_kv(0, 1, k, k, rotation=_rotation(64))
    for bad in (B.GbRotation(0, 300, 128, 0), B.GbRotation(good.table.data_ptr() + 4, 300, 128, 0), B.GbRotation(good.table.data_ptr(), 0, 128, 0),
                B.GbRotation(good.table.data_ptr(), 300, 24, 0), B.GbRotation(good.table.data_ptr(), 300, 144, 0),
                B.GbRotation(good.table.data_ptr(), 300, 0, 0), B.GbRotation(good.table.data_ptr(), 300, 128, 2)):
        with pytest.raises(B.GambitError, match="GB_ERR_INVALID"):
            B.gb_append_kv_rotated(pool.handle, 0, 1, bad, k, k)
    with pytest.raises(B.GambitError, match="GB_ERR_INVALID"):
        pool.append_kv(0, 1, k[1:], k, rotation=good)
    with pytest.raises(B.GambitError, match="GB_ERR_INVALID"):
        pool.decode_attention(0, k, k[4:], k, 0.1, torch.zeros(5, 8, d, device="cuda"), rotation=good)
    assert pool.status() == 0 and pool.read_state()["seq_len"].tolist() == [20] * 5
