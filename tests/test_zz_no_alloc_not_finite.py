"""Keys that are not finite in caller-owned pages: NaN reaches the heads that see it, scores of minus infinity weigh nothing."""
import numpy as np
import pytest

from tests.test_zz_no_alloc import _call, _case, _device

pytestmark = pytest.mark.gpu


def _run(cuda, c):
    from paper_2608_08020_gb300 import binding as B
    d = _device(c, cuda)
    assert _call(B, c, d) == B.GB_OK
    return d["out"].cpu().numpy()


@pytest.mark.parametrize("dtype,G,P", [("f32", 4, 16), ("f32", 8, 32), ("bf16", 2, 16), ("bf16", 4, 32), ("bf16", 8, 64)])
def test_keys_that_are_not_finite(cuda, dtype, G, P):
    c = _case(dtype, G, P, seed=3)
    clean, L = _run(cuda, c), c["seq_len"]
    for b, t in ((0, 0), (0, int(L[0]) - 1), (1, int(L[1]) - 1), (3, 0), (4, P), (5, P - 2), (6, int(L[6]) - 1)):
        at = (c["tables"][b, t // P], 0, 1, t % P, 5)
        was = c["kv"][at]
        c["kv"][at] = np.nan
        out = _run(cuda, c)
        c["kv"][at] = was
        want = np.zeros(out.shape, bool)
        for r in range(len(L)):
            want[r, G:] = t < L[r] and c["tables"][r, t // P] == at[0]
        assert np.array_equal(np.isnan(out), want) and np.array_equal(out[~want], clean[~want]), (b, t)
    c["q"][..., 0] = np.abs(c["q"][..., 0]) + 0.5
    outs = []
    for low in (-np.inf, -1e6):                           # either weighs nothing beside scores of some tens
        c["kv"][c["tables"][0, :2], 0, :, :, 0] = low
        c["kv"][c["tables"][4, :1], 0, :, :, 0] = low
        outs.append(_run(cuda, c))
    assert np.isfinite(outs[1]).all() and np.array_equal(*outs)
    c["kv"][:, 0, :, :, 0] = -np.inf
    assert np.array_equal(np.isnan(_run(cuda, c)).all((1, 2)), L > 0)
