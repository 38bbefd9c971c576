"""Scores capped by a tanh, caps far below the scores to far above them: attention of few and many rows and both forms of the account."""
import pytest

from kv_helpers import FMTS, Cache, queries
from test_gpu_kv_attention import run
from test_gpu_kv_weights import check_weights

pytestmark = pytest.mark.gpu

# one row, drafts, many rows of a sequence
NEW = [None, [5, 1, 3], [60, 290, 64]]
CAPS = [1e-38, 1e-3, 0.7, 8.0, 50.0, 1e3, 1e5, 1e7, 1e9, 1e30]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("new", NEW, ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("nvfp4", 64), ("mxint4", 256)])
def test_caps_of_every_size(fmt, dim, new, cap):
    c = Cache(fmt, [129, 500, 64], 4, 3, dim, 32, new=new)
    Q = queries(c)
    run(c, Q, softcap=cap)
    check_weights(c, Q, softcap=cap)


@pytest.mark.parametrize("new", NEW, ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_scores_of_every_size_under_one_cap(fmt, new):
    """From far below the cap, over the place where it is computed in another way (a quarter of it), to where it holds all of them."""
    c = Cache(fmt, [129, 500, 64], 4, 3, 128, 32, new=new)
    for size in (1e-4, 0.1, 0.5, 2.0, 40.0):
        Q = queries(c, size=size)
        run(c, Q, softcap=10.0)
        check_weights(c, Q, softcap=10.0)
