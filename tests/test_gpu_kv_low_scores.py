"""Attention of rows whose scores are all far below zero."""
import pytest
import torch

from kv_far_helpers import check_largest
from kv_helpers import FMTS, Cache, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [None, [5, 1, 3], [60, 290, 64]], ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_rows_whose_scores_are_all_far_below_zero(fmt, new):
    """Rows that see one token only, themselves: half of these scores are far below zero, and the result is that token's value."""
    lens = [129, 500, 64]
    c = Cache(fmt, lens, 4, 3, 128, 32, new=new)
    Q = queries(c)
    first = torch.cat([c.rows(b)[1] for b in range(3)]).to(torch.int32)
    out, lse = c.call("attention", Q, *c.scales, scale=1e30, first=first, return_lse=True)
    assert (lse < -1e30).any()
    check_largest(c, Q, out, lse, float(torch.tensor(1e30, dtype=torch.float32)), first=first)
