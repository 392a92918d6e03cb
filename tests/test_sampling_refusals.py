"""What gb_sample refuses before it touches a GPU."""
import ctypes

import pytest


def _args(B, **kw):
    a = dict(logits=4096, row_stride=100, u=4096, token=8192, rows=2, vocab=100, dtype=B.GB_F32, all_temperature=1.0, all_top_p=1.0)
    return B.GbSampleArgs(**{**a, **kw})


@pytest.mark.parametrize("kw,code", [({"rows": -1}, 1), ({"vocab": 0}, 1), ({"dtype": 2}, 1), ({"dtype": -1}, 1), ({"logits": 0}, 1), ({"u": 0}, 1),
                                     ({"token": 0}, 1), ({"row_stride": 99}, 1), ({"logits": 4098}, 1), ({"u": 4097}, 1), ({"top_p": 4098}, 1),
                                     ({"vocab": 524289, "row_stride": 600000}, 6), ({"rows": 0}, 0), ({"rows": 0, "logits": 0}, 0)])
def test_arguments(kw, code):
    from paper_2608_08020_gb300 import binding as B
    if not B.LIB_PATH.exists():
        pytest.skip("libgambit.so not built")
    assert B.load().gb_sample(ctypes.byref(_args(B, **kw)), None) == code
    assert B.load().gb_sample(None, None) == 1
