"""The definition that the GPU tests compare sampled tokens with, on hand-made rows (no GPU)."""
import math

import numpy as np
import pytest

from tests.sampling_reference import kept_mass, pick

LOG = [math.log(p) for p in (0.1, 0.4, 0.2, 0.3)]


def test_draw_by_index():
    for u, i in ((0.0, 0), (0.0999, 0), (0.1001, 1), (0.4999, 1), (0.5001, 2), (0.6999, 2), (0.7001, 3), (0.9999, 3)):
        token, lp = pick(LOG, u)
        assert token == i and abs(lp - LOG[i]) < 1e-12


@pytest.mark.parametrize("kw,kept", [({"top_k": 2}, [1, 3]), ({"top_k": 9}, [0, 1, 2, 3]), ({"top_p": 0.39}, [1]), ({"top_p": 0.41}, [1, 3]),
                                     ({"top_p": 0.95}, [0, 1, 2, 3]), ({"min_p": 0.6}, [1, 3]), ({"min_p": 2.0}, [1]), ({"top_p": 0.0}, [1]),
                                     ({"top_k": 3, "top_p": 0.7}, [1, 3]), ({"min_p": 0.3, "top_p": 0.8}, [1, 2, 3])])
def test_what_is_kept(kw, kept):
    assert np.flatnonzero(kept_mass(LOG, **kw)).tolist() == kept


def test_ties_go_to_the_lowest_index():
    x = [1.0, 2.0, 2.0, 2.0, 1.0]
    assert np.flatnonzero(kept_mass(x, top_k=2)).tolist() == [1, 2]
    assert np.flatnonzero(kept_mass(x, top_k=4)).tolist() == [0, 1, 2, 3]
    assert np.flatnonzero(kept_mass([0.0] * 8, top_p=0.5)).tolist() == [0, 1, 2, 3]
    assert pick(x, 0.9, temperature=0.0) == (1, 0.0)


def test_rows_that_are_not_finite():
    inf, nan = math.inf, math.nan
    assert pick([-inf, nan], 0.5) == (-1, -inf)
    assert pick([1.0, inf, -inf, inf], 0.6)[0] == 3
    assert pick([nan, 0.0, -inf], 0.99) == (1, 0.0)
