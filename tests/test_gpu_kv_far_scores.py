"""Scores far from zero, to the end of float32: all weight goes to the largest score, and the logarithm of the sum is that score."""
import pytest
import torch

from kv_far_helpers import check_largest
from kv_helpers import FMTS, Cache, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2.0 ** 20, 2.0 ** 26, 2.0 ** 30, 1e20, 1e30])
@pytest.mark.parametrize("new", [None, [5, 1, 3], [60, 290, 64]], ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_large_scores(fmt, new, scale):
    c = Cache(fmt, [129, 500, 64], 4, 3, 128, 32, new=new)
    Q = queries(c)
    out, lse = c.call("attention", Q, *c.scales, scale=scale, return_lse=True)
    check_largest(c, Q, out, lse, float(torch.tensor(scale, dtype=torch.float32)))
