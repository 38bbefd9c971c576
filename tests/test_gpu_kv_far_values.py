"""Values at both ends of E8M0, of sequences that one CTA works on and of sequences that several do."""
import pytest
import torch

from kv_helpers import Cache, check_attention, queries
from test_gpu_kv_far_scales import move_scales

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by", [-110, 100, 110, 125])
@pytest.mark.parametrize("lens,heads,new", [([3000] + [33] * 400, 4, None), ([3000, 900], 2, [4, 5]), ([20000], 1, [300]), ([700, 333, 64], 32, [300, 300, 64])],
                         ids=["one", "few", "many-cut", "many-whole"])
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("mxint4", 64), ("mxint4", 256)])
def test_values_far_from_one(fmt, dim, lens, heads, new, by):
    """Parts of a sequence and whole ones alike: nothing between the values and the result is larger than the values are."""
    c = Cache(fmt, lens, heads, 2, dim, 32, new=new)
    Q = queries(c, size=0.3)                             # weights of many tokens
    move_scales(c, 3, by)
    out, lse = c.call("attention", Q, return_lse=True)
    check_attention(c, Q, out.double() * 2.0 ** -by, lse)
