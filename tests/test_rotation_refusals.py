"""What Rotation and the 8-bit pool's sizes refuse or say without a GPU."""
import pytest
import torch


def _lib():
    from paper_2608_08020_gb300 import binding
    if not binding.LIB_PATH.exists():
        pytest.skip("libgambit.so not built")
    return binding


def test_rotation_arguments():
    _lib()
    from paper_2608_08020_gb300.rotation import Rotation
    for kw in ({"rotary_dim": 24}, {"rotary_dim": 144}, {"rotary_dim": 0}, {"max_positions": 0}, {"frequencies": [1.0] * 5}):
        with pytest.raises(ValueError):
            Rotation(128, **{"max_positions": 4, "device": "cpu", **kw})


def test_rotation_table():
    _lib()
    from paper_2608_08020_gb300.rotation import Rotation
    r = Rotation(128, max_positions=70000, base=1e4, rotary_dim=32, amplitude=0.5, device="cpu")
    t = torch.arange(70000, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, 32, 2, dtype=torch.float64) / 32)
    table = r.table.double()
    assert r.table.shape == (70000, 4, 16)
    # Two fp32 terms: the second is rounded to 2^-24 of the first's rounding error, 2^-25 of the value.
    assert ((table[:, 0] + table[:, 1]) - 0.5 * t.cos()).abs().max() <= 2.0 ** -49
    assert ((table[:, 2] + table[:, 3]) - 0.5 * t.sin()).abs().max() <= 2.0 ** -49
    f = Rotation(64, max_positions=3, frequencies=torch.arange(32), device="cpu")
    assert torch.allclose(f.table[2, 0, 3], torch.tensor(6.0).cos())


@pytest.mark.parametrize("g,d,ok", [(1, 128, True), (2, 128, True), (4, 128, True), (8, 128, True), (16, 128, False), (3, 128, False),
                                    (4, 64, False)])
def test_sizes_of_an_eight_bit_pool(g, d, ok):
    B = _lib()
    cfg = B.GbPoolConfig(3, 2 * g, 2, d, 32, B.GB_FP8, 100, 4, 10, 0)
    if not ok:
        with pytest.raises(B.GambitError, match="GB_ERR_UNSUPPORTED"):
            B.gb_pool_workspace_bytes(cfg)
        return
    kv, _ = B.gb_pool_workspace_bytes(cfg)
    rows = 3 * 100 * 2 * 2 * 32
    assert kv == -(-rows * 128 // 256) * 256 + rows // 16
