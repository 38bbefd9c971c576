"""Scales of the features of a token far apart: in attention of many rows they are taken relative to the largest of 128 tokens."""
import pytest
import torch

from kv_helpers import Cache, check_attention, parts, queries
from operator_helpers import DEV

pytestmark = pytest.mark.gpu

E8M0 = ("mxfp4", "mxint4")


@pytest.mark.parametrize("gap", [10, 25, 26, 27, 30, 34, 35])
@pytest.mark.parametrize("new", [None, [60, 290, 64]], ids=["one", "many"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", E8M0)
def test_features_far_apart(fmt, dim, new, gap):
    """The first 32 features of keys and values are 2^gap larger than the others.  Most queries have zeros there, so their scores come from the others alone;
    results of the others are what they are beside large ones."""
    c = Cache(fmt, [129, 500, 64], 4, 3, dim, 32, new=new, spread=1, low=110)
    for b, n in enumerate(c.lens):
        page, slot = c.at(b, torch.arange(n, device=DEV))
        for part in (1, 3):
            parts(c.pages, fmt, dim)[part][page, :, slot, 0] = 110 + gap
        c.K[b][..., :32] *= 2.0 ** gap
        c.V[b][..., :32] *= 2.0 ** gap
    # A query has elements in the large features or in the others: float16 keeps 2^-39 of a row's largest, so elements 2^-gap of it times keys 2^gap larger
    # would be off by 2^(gap - 39) of a score, 2^-9 at 30, where check_attention allows 2^-19.
    Q = queries(c).double() * 2.0 ** 16
    large = (torch.arange(c.H * c.G, device=DEV) % 2 == 0).view(-1, 1) & (torch.arange(c.tokens, device=DEV) % 2 == 0).view(-1, 1, 1)
    Q = torch.where(large == (torch.arange(dim, device=DEV) < 32), torch.where(large, Q * 2.0 ** -gap, Q), 0.0).to(torch.bfloat16)
    out, lse = c.call("attention", Q, return_lse=True)
    check_attention(c, Q, out, lse)
