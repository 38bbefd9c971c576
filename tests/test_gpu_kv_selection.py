"""The selection of an eviction by one, two, four and eight CTAs of a sequence and head, with their weights in shared memory and with more than fit there."""
import pytest
import torch

from kv_helpers import Cache
from operator_helpers import DEV, gen
from test_gpu_kv_weights import check_evict, with_evict

pytestmark = pytest.mark.gpu


# CTAs per sequence and head: as many as the SMs have room for, with 2048 tokens at least; one holds 24576 weights
@pytest.mark.parametrize("lens,heads,keep,recent", [([9000], 80, 5000, 100),           # one
                                                    ([25000], 80, 9000, 100),          # one, more than it holds
                                                    ([9000, 700], 20, 8000, 0),        # two
                                                    ([9000], 20, 4100, 300),           # four
                                                    ([101000], 20, 60000, 1000),       # four, more than they hold
                                                    ([17000, 16400], 2, 9000, 5),      # eight
                                                    ([201000], 1, 100000, 1000),       # eight, more than they hold
                                                    ([201000, 40], 1, 200900, 0)])     # eight, nearly all stay
@pytest.mark.parametrize("kind", ["wide", "few values"])
def test_selection_by_clusters(lens, heads, keep, recent, kind):
    page = 128
    c = with_evict(Cache("mxfp4", lens, heads, 1, 64, page))
    c.K = c.V = None                                     # of no use here, and large
    g = gen(22)
    shape = (c.pages.shape[0], heads, page)
    w = torch.randint(0, 3, shape, generator=g, device=DEV).float() if kind == "few values" else \
        torch.exp(30 * torch.randn(shape, generator=g, device=DEV)).clamp(max=3e38)
    check_evict(c, w, keep, recent)
