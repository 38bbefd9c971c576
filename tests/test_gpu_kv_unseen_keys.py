"""Keys that no row sees, in front of every row's document, beside very small ones that rows see: the same bits whatever they hold."""
import pytest
import torch

from kv_helpers import Cache, check_attention, parts, queries
from operator_helpers import DEV, gen
from test_gpu_kv_far_scales import move_scales, short_queries
from test_gpu_kv_weights import check_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[1, 1], [3, 2], [50, 40]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxint4"])
def test_keys_in_front_of_small_ones(fmt, dim, new):
    c = Cache(fmt, [777, 540], 4, 2, dim, 32, new=new)
    begins = [77, 301]                                   # neither is a multiple of 16
    first = torch.cat([torch.full((n,), begins[b], dtype=torch.int32, device=DEV) for b, n in enumerate(new)])
    move_scales(c, 1, -80)
    c.K = [k * 2.0 ** -80 for k in c.K]
    Q = (short_queries(c) * 2.0 ** 80).to(torch.bfloat16)
    out, lse = c.call("attention", Q, return_lse=True, first=first)
    check_attention(c, Q, out, lse, first=first)
    check_weights(c, Q, first=first)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(4), device=DEV)
    account = c.call("weights", Q, lse, w.clone(), first=first)
    for byte in (0xC0, 0xFD, 0xFE, 0xFF):
        for b in range(2):
            page, slot = c.at(b, torch.arange(begins[b], device=DEV))
            for part in parts(c.pages, fmt, dim):
                part[page, :, slot] = byte
        y, z = c.call("attention", Q, return_lse=True, first=first)
        assert torch.equal(y, out) and torch.equal(z, lse)
        assert torch.equal(c.call("weights", Q, lse, w.clone(), first=first), account)
