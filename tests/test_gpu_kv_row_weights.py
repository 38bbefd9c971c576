"""The account over many rows of a sequence: every kernel that serves it, tiles and groups that are not full, rows that saw nothing."""
import pytest
import torch

from helpers import captured_launches
from kv_helpers import FMTS, Cache, queries
from operator_helpers import DEV, gen
from test_gpu_kv_attention import OPTIONS, options_of
from test_gpu_kv_weights import check_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_prompts(fmt, dim, page):
    c = Cache(fmt, [200, 401, 1300, 0, 64, 127], 3, 4, dim, page, new=[150, 401, 31, 0, 3, 17])
    check_weights(c, queries(c))


@pytest.mark.parametrize("rows", [7, 8, 9, 31, 32, 33, 63, 64, 65])
def test_groups_that_are_not_full(rows):
    c = Cache("nvfp4", [300, 65], 2, 1, 64, 32, new=[rows, rows])
    Q = queries(c)
    check_weights(c, Q)
    lse, w = torch.zeros(c.tokens, 2, device=DEV), torch.zeros(c.pages.shape[0], 2, 32, device=DEV)
    name, = captured_launches(lambda: c.call("weights", Q, lse, w, c.scales[0]))
    assert ("row_weights" in name[0]) == (rows > 8)


@pytest.mark.parametrize("o", OPTIONS, ids=lambda o: "-".join(o))
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 256), ("nvfp4", 128), ("mxint4", 64)])
def test_scoring(fmt, dim, o):
    c = Cache(fmt, [129, 500, 64], 2, 3, dim, 32, new=[60, 290, 64])
    check_weights(c, queries(c), **options_of(c, o))


@pytest.mark.parametrize("new", [[6, 5], [60, 50]], ids=["few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_queries_of_rows_without_a_place_may_be_no_numbers(fmt, new):
    """More new rows than the sequence has tokens: the first rows see nothing, whatever they hold."""
    c = Cache(fmt, [4, 400], 2, 1, 64, 16, new=new)
    Q = queries(c)
    y, lse = c.call("attention", Q, *c.scales, return_lse=True)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(1), device=DEV)
    want = c.call("weights", Q, lse, w.clone(), *c.scales[:1])
    assert torch.isfinite(want).all()
    none = torch.isneginf(lse).all(1)
    assert none.sum() == new[0] - 4
    Q[none] = float("nan")
    z, lse2 = c.call("attention", Q, *c.scales, return_lse=True)
    assert torch.equal(z, y) and torch.equal(lse2, lse)
    assert torch.equal(c.call("weights", Q, lse, w.clone(), *c.scales[:1]), want)
