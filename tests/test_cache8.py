"""The model of an 8-bit cache that the GPU tests compare with, against torch's own e4m3 type and hand-made cases (no GPU)."""
import pytest
import torch

from tests.cache8 import Cache8, least_exponent, nearest_e4m3, rotated


def test_nearest_is_torchs_e4m3():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    held = codes[torch.isfinite(codes)].unique()
    assert torch.equal(nearest_e4m3(held), held)
    mid = (held[1:] + held[:-1]) / 2
    x = torch.cat([mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), torch.randn(4096, dtype=torch.float64) * 10])
    x = x.float().double()      # torch rounds through fp32
    assert torch.equal(nearest_e4m3(x), x.float().to(torch.float8_e4m3fn).double())


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.5, 1), (224.0, -1), (224.5, 0), (0.0, -60), (1e-30, -60), (1e30, 60), (896.0, 1)])
def test_exponent(top, e):
    assert least_exponent(torch.tensor([0.0, top, -top / 2, float("inf"), float("nan")], dtype=torch.float64)) == e


def test_a_row_that_does_not_fit_raises_its_block_alone():
    c = Cache8(1, 1, 1, 2)
    x = torch.tensor([[[448.0, 2.0 ** -9]]], dtype=torch.float64)
    c.append(0, 0, x.repeat(18, 1, 1), x.repeat(18, 1, 1))
    c.append(0, 0, 4 * x, x)
    rows, exps = c.kv[0][0]
    assert exps[:, :, 0].tolist() == [[0, 2], [0, 0]]
    assert rows[0, 15, 0, 1] == 2.0 ** -9 and rows[0, 16, 0, 1] == 0 and rows[0, 18, 0, 1] == 2.0 ** -7   # 2^-9 is under half of 2^-7
    c.truncate(0, 17)
    c.append(0, 0, x, x)
    assert c.kv[0][0][1][0, 1, 0] == 2       # a cut keeps the exponent ..
    c.truncate(0, 16)
    c.append(0, 0, x, x)
    assert c.kv[0][0][1][0, 1, 0] == 0       # .. and a block's first row begins it anew


def test_rotation_depends_on_distance_alone():
    g = torch.Generator().manual_seed(0)
    q, k = torch.randn(2, 32, generator=g, dtype=torch.float64)
    for interleaved in (False, True):
        dots = [rotated(q, t + 7, 32, 100.0, interleaved) @ rotated(k, t, 32, 100.0, interleaved) for t in (0, 5, 900)]
        assert torch.allclose(torch.stack(dots), dots[0].expand(3), atol=1e-12)
    assert torch.equal(rotated(q, 3, 16, 100.0)[16:], q[16:])
