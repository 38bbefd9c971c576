"""Attention over the 4-bit key/value cache against the definition in 64 bits."""
import pytest
import torch

from kv_helpers import FMTS, Cache, check_attention, queries
from operator_helpers import DEV, gen

pytestmark = pytest.mark.gpu


def run(c, Q, **options):
    out, lse = c.call("attention", Q, *c.scales, return_lse=True, **options)
    check_attention(c, Q, out, lse, **options)
    return out, lse


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_one_token_of_each_sequence(fmt, dim):
    c = Cache(fmt, [1, 77, 300, 0, 16, 17, 129, 1000], 2, 4, dim, 16)
    run(c, queries(c))


@pytest.mark.parametrize("heads,group", [(1, 1), (3, 5), (2, 8), (1, 16), (1, 40), (4, 3)])
@pytest.mark.parametrize("fmt", FMTS)
def test_heads(fmt, heads, group):
    c = Cache(fmt, [513, 64, 31], heads, group, 128, 32)
    run(c, queries(c))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("fmt", FMTS)
def test_pages(fmt, page):
    c = Cache(fmt, [700, 15, 2049], 2, 2, 64, page, new=[3, 1, 2])
    run(c, queries(c))


@pytest.mark.parametrize("new", [[1, 1, 1], [2, 7, 0], [33, 100, 5], [150, 400, 300]])
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("nvfp4", 64), ("mxint4", 256)])
def test_new_tokens(fmt, dim, new):
    c = Cache(fmt, [200, 400, 300], 2, 4, dim, 16, new=new)
    run(c, queries(c))


OPTIONS = [dict(softcap=5.0), dict(window=1), dict(window=40), dict(slopes=True), dict(prefix=True), dict(first=True), dict(scale=0.3),
           dict(softcap=20.0, window=130, slopes=True, prefix=True, first=True)]


def options_of(c, o):
    o = dict(o)
    g = gen(5)
    if "slopes" in o:
        o["slopes"] = torch.rand(c.H * c.G, generator=g, device=DEV) * 0.3
    if "prefix" in o:
        o["prefix"] = torch.tensor([(7 * n) // 8 for n in c.lens], dtype=torch.int32, device=DEV)
    if "first" in o:                                     # the last rows' document begins behind them: they see nothing
        o["first"] = torch.cat([torch.tensor([0 if i < n // 2 else c.lens[b] - (n - i) // 2 for i in range(n)], dtype=torch.int32, device=DEV)
                                for b, n in enumerate(c.new)])
    return o


@pytest.mark.parametrize("o", OPTIONS, ids=lambda o: "-".join(o))
@pytest.mark.parametrize("new", [None, [5, 1, 3], [60, 290, 64]], ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_scoring(fmt, new, o):
    c = Cache(fmt, [129, 500, 64], 2, 3, 128, 32, new=new)
    run(c, queries(c), **options_of(c, o))


def test_more_new_rows_than_the_sequence_has():
    c = Cache("mxfp4", [4, 40], 1, 2, 64, 16, new=[6, 5])
    run(c, queries(c))
